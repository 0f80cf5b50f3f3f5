"""8-bit products through the plans that their sizes lead to."""
import numpy as np
import pytest
import torch

from tests.fp8_cases import DEV, TORCH, matrix
from tests.gpu_cases import note
from tests.test_gpu_fp8 import G  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,per,dtype", [(128, 600, 5000, 128, "bf16"), (916, 271, 7208, 1, "f16"), (45, 1500, 7098, 128, "f32"),
                                             (128, 600, 4999, 1, "bf16")])
def test_the_workspace_asked_for_is_all_that_a_product_uses(G, M, N, K, per, dtype):  # noqa: F811
    """As many bytes as were asked for give the bits of any more (sums that are split unevenly; packed rows)."""
    note("fp8 exact workspace %d %d %d" % (M, N, K))
    rng = np.random.default_rng(M)
    a, sa, _, _ = matrix(rng, M, K)
    b, sb, _, _ = matrix(rng, N, K, per)
    n = G.gvr_fp8_matmul_workspace(a, sa, b, sb)
    assert n >= 2 * M * N * 4
    want = G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype], workspace=torch.empty(2 * n + 512, dtype=torch.uint8, device=DEV))
    exact = torch.empty(n, dtype=torch.uint8, device=DEV)
    assert torch.equal(G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype], workspace=exact), want)
    assert torch.equal(G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype]), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(771, 531, 1000), (16, 8300, 700), (30, 1000, 640), (64, 1500, 4096), (2312, 769, 512), (1678, 2309, 512),
                                   (1285, 4400, 301)])
def test_a_scale_for_128_rows_is_one_for_each_of_them(G, M, N, K, dtype):  # noqa: F811
    """The kernels that read a scale of 128 rows once give the bits of those that read it for each row."""
    note("fp8 scales of rows %d %d %d %s" % (M, N, K, dtype))
    rng = np.random.default_rng(M)
    a, sa, _, _ = matrix(rng, M, K, pad=-K % 16)
    b, sb, _, _ = matrix(rng, N, K, 128, pad=-K % 16)
    each = sb.repeat_interleave(128, dim=0)[:N].contiguous()
    assert torch.equal(G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype]), G.gvr_fp8_matmul(a, sa, b, each, dtype=TORCH[dtype]))
