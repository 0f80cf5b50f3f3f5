"""8-bit matrices and products whose elements lie past 32 bits: equal to those of small ones."""
import pytest
import torch

from tests.fp8_cases import DEV
from tests.gpu_cases import note
from tests.test_gpu_fp8 import G  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("square", [False, True])
def test_both_directions_of_a_tall_matrix(G, square):  # noqa: F811
    note("fp8 far matrix %s" % square)
    rows, K, tail = 540000, 8192, 96 + 2 * 128   # (the last block of rows has 96)
    assert rows * K > 1 << 32 and rows % 128 == 96
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device=DEV)
    x[-300:] = torch.randn((300, K), device=DEV).bfloat16()
    a, t = G.gvr_fp8_quantize_matrix(x, square=square, transposed=True)
    sa, st = G.gvr_fp8_quantize_matrix(x[-tail:].contiguous(), square=square, transposed=True)
    assert torch.equal(a.codes[-tail:], sa.codes) and torch.equal(a.scale[-sa.scale.shape[0]:], sa.scale)
    assert torch.equal(t.codes[:, -tail:], st.codes) and torch.equal(t.scale[:, -3:], st.scale)
    assert int(a.codes[:-300].max()) == 0 and int(t.codes[:, :-300].max()) == 0
    assert (a.scale[:-sa.scale.shape[0]] == 2.0 ** -126).all() and (t.scale[:, :-3] == 2.0 ** -126).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_results_past_32_bits(G, dtype):  # noqa: F811
    note("fp8 far results %s" % dtype)
    M, N, K = 66000, 65600, 130   # (a sum of two blocks, which no plan splits)
    assert M * N > 1 << 32
    a = G.gvr_fp8_quantize(torch.randn((M, K), device=DEV))
    b = G.gvr_fp8_quantize_matrix(torch.randn((N, K), device=DEV), square=True)
    out = G.gvr_fp8_matmul(*a, *b, dtype=dtype)
    for at in (0, 32760, 65500, M - 200):
        part = G.gvr_fp8_matmul(a.codes[at:at + 200], a.scale[at:at + 200], *b, dtype=dtype)
        assert torch.equal(out[at:at + 200], part)
