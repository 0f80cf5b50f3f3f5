"""Frozen 8-bit layers whose codes lie as a loaded weight's do: packed rows, shifted views, scales in any order."""
import pytest
import torch

from tests.fp8_cases import DEV
from tests.gpu_cases import note
from tests.test_gpu_fp8 import G  # noqa: F401

pytestmark = pytest.mark.gpu


def packed(m, shift=0):
    """The same matrix in packed rows, the first `shift` bytes behind the storage's start; what lies around is NaN codes."""
    rows, cols = m.codes.shape
    store = torch.full((rows * cols + shift + 40,), 0x7F, dtype=torch.uint8, device=DEV)
    codes = store[shift:shift + rows * cols].view(rows, cols)
    codes.copy_(m.codes)
    return codes, m.scale.T.contiguous().T


@pytest.mark.parametrize("M,N,K,shift", [(128, 600, 4099, 0), (1, 333, 2050, 0), (20, 301, 1003, 0), (300, 1027, 4097, 5), (128, 1024, 2048, 3)])
def test_packed_rows_give_the_layer_of_aligned_ones(G, M, N, K, shift):  # noqa: F811
    """Bit for bit: the codes are copied into line in the layer's workspace, forward and backward."""
    note("fp8 frozen %d %d %d %d" % (M, N, K, shift))
    from paper_2604_22312_amd import fp8
    torch.manual_seed(M + N)
    x = torch.randn((M, K), device=DEV).bfloat16().requires_grad_()
    dy = torch.randn((M, N), device=DEV).bfloat16()
    q, qt = G.gvr_fp8_quantize_matrix(torch.randn((N, K), device=DEV) / K ** 0.5, square=True, transposed=True)
    y = G.gvr_fp8_linear(x, q, qt)
    dx = torch.autograd.grad(y, x, dy)[0]
    p, pt = packed(q, shift), packed(qt, shift)
    z = G.gvr_fp8_linear(x, p, pt)
    assert torch.equal(z, y)
    assert torch.equal(torch.autograd.grad(z, x, dy)[0], dx)
    # as much workspace as the product by itself asks for
    xq, dq = G.gvr_fp8_quantize(x.detach()), G.gvr_fp8_quantize(dy)
    for a, b, sizes in ((xq, p, (M, N, K)), (dq, pt, (M, K, N))):
        struct = fp8._matrix_struct(b, "b", sizes[1], sizes[2], 128, x.device)
        assert fp8._product_workspace(*sizes, 128, x.device.index, fp8._layout(struct)) == G.gvr_fp8_matmul_workspace(*a, *b)
        assert torch.equal(G.gvr_fp8_matmul(*a, *b), y if b is p else dx)
    assert fp8._product_workspace(M, N, K, 128, x.device.index) == G.gvr_fp8_matmul_workspace(*xq, *q)


def test_layers_of_different_layouts_in_turn(G):  # noqa: F811
    """The sizes that a layer remembers go by how its codes lie, not by their sizes alone."""
    note("fp8 frozen in turn")
    torch.manual_seed(1)
    x = torch.randn((128, 4099), device=DEV).bfloat16()
    q = G.gvr_fp8_quantize_matrix(torch.randn((600, 4099), device=DEV), square=True)
    ways = [q, packed(q), packed(q, 16), packed(q, 1), q]
    with torch.no_grad():
        want = G.gvr_fp8_linear(x, q)
        for i in range(3):
            for w in ways:
                assert torch.equal(G.gvr_fp8_linear(x, w), want)


@pytest.mark.parametrize("shape", [(3, 60, 200), (7, 200), (200,), (0, 5, 200)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_layer_without_outputs(G, shape, dtype):  # noqa: F811
    note("fp8 layer without outputs %s" % (shape,))
    x = torch.randn(shape, device=DEV, dtype=dtype, requires_grad=True)
    w = torch.randn((0, 200), device=DEV, requires_grad=True)
    for f in (lambda: G.gvr_fp8_linear(x, w), lambda: G.gvr_fp8_linear(x, *G.gvr_fp8_quantize_matrix(w.detach(), square=True,
                                                                                                   transposed=True))):
        y = f()
        assert y.shape == shape[:-1] + (0,) and y.dtype == dtype
        got = torch.autograd.grad(y, (x, w), torch.ones_like(y), allow_unused=True)
        assert got[0].shape == shape and (got[0] == 0).all() and (got[1] is None or got[1].shape == (0, 200))
