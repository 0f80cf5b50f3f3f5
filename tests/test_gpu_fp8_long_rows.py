"""The 8-bit linear layer on rows longer than a head may be."""
import pytest
import torch

from tests.fp8_cases import DEV
from tests.gpu_cases import note
from tests.test_gpu_fp8 import G  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [1 << 20, (1 << 20) + 130])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_a_million(G, K, dtype):  # noqa: F811
    """With gradients, without them and frozen: the same bits."""
    note("fp8 long rows %d" % K)
    torch.manual_seed(K)
    x = torch.randn((2, K), device=DEV, dtype=dtype)
    w = torch.randn((3, K), device=DEV, dtype=dtype, requires_grad=True)
    y = G.gvr_fp8_linear(x, w)
    gw = torch.autograd.grad(y, w, torch.ones_like(y))[0]
    assert gw.shape == w.shape
    with torch.no_grad():
        assert torch.equal(G.gvr_fp8_linear(x, w), y)
    q, qt = G.gvr_fp8_quantize_matrix(w.detach(), square=True, transposed=True)
    z = x.clone().requires_grad_()
    v = G.gvr_fp8_linear(z, q, qt)
    assert torch.equal(v, y)
    assert torch.autograd.grad(v, z, torch.ones_like(v))[0].shape == x.shape
    m = G.gvr_fp8_quantize_matrix(x)
    assert torch.equal(G.gvr_fp8_matmul(*m, *q, dtype=dtype), y)
