"""Every kernel of the 8-bit products against the oracle, at sizes that the planner itself sends to it
(tests/test_fp8_shapes.py asserts which)."""
import numpy as np
import pytest
import torch

import oracle.fp8 as O
from tests.fp8_cases import DEV, TORCH, close, cut_off, product_bound
from tests.fp8_shapes import EVERY, SIZES
from tests.gpu_cases import note
from tests.test_gpu_fp8 import G  # noqa: F401

pytestmark = pytest.mark.gpu


def operand(gen, rows, K, per, wide=None):
    """Codes [rows][K] in rows of `wide` bytes (a multiple of 16 above K; the rest NaN codes) and scales, on the GPU and the host."""
    x = torch.randn((rows, K), generator=gen, device=DEV) * 120
    x *= torch.exp(0.7 * torch.randn((rows, 1), generator=gen, device=DEV))
    store = torch.full((rows, wide or (K + 15) // 16 * 16), 0x7F, dtype=torch.uint8, device=DEV)
    codes = store[:, :K]
    codes.copy_(x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    scale = torch.exp(0.7 * torch.randn(((rows + per - 1) // per, (K + 127) // 128), generator=gen, device=DEV)) / 448
    return codes, scale


def some(rng, n, count=24):
    """Some of n rows: the first, the last, those beside borders of tiles, and others."""
    edges = [0, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, n - 129, n - 65, n - 17, n - 1]
    return np.unique(np.clip(np.concatenate([edges, rng.integers(0, n, count)]), 0, n - 1))


def check(out, a, sa, b, sb, per, dtype, parts):
    """`out` on the rows and columns of `parts` (made once for all types)."""
    K = a.shape[1]
    if not parts:
        rng = np.random.default_rng(a.shape[0])
        ha, hb = (t.cpu().numpy() for t in (sa, sb))
        for rows, cols in ((some(rng, a.shape[0]), None), (None, some(rng, b.shape[0]))):
            va, vb = O.values(a.cpu().numpy(), ha), O.values(b.cpu().numpy(), hb, per)
            va, vb = (va, vb[cols]) if rows is None else (va[rows], vb)
            parts.append((rows, cols, va @ vb.T, np.abs(va) @ np.abs(vb).T, cut_off(va, vb)))
    for rows, cols, ref, mag, cut in parts:
        got = out[:, torch.from_numpy(cols).to(DEV)] if rows is None else out[torch.from_numpy(rows).to(DEV)]
        close(got, ref, product_bound(mag, ref, K, dtype, cut))


@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("M,N,K,types", SIZES)
def test_products(G, M, N, K, types, per):  # noqa: F811
    gen = torch.Generator(device=DEV)
    gen.manual_seed(M * 5 + N * 3 + K + per)
    a, sa = operand(gen, M, K, 1)
    b, sb = operand(gen, N, K, per)
    parts = []
    for dtype in types:
        note("fp8 shapes %d %d %d per %d %s" % (M, N, K, per, dtype))
        store = torch.full((M, N + 8), 7.0, dtype=TORCH[dtype], device=DEV)
        out = G.gvr_fp8_matmul(a, sa, b, sb, out=store[:, :N])
        check(out, a, sa, b, sb, per, dtype, parts)
        assert (store[:, N:] == 7).all()
        assert torch.equal(G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype]), out)


@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (70, 130, 401), (3, 500, 1100), (129, 65, 128)])
def test_products_where_they_are(G, M, N, K, per):  # noqa: F811
    """Rows of any alignment with no workspace to copy them into."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(M + N + K)
    a, sa = operand(gen, M, K, 1, K + 5)
    b, sb = operand(gen, N, K, per, K + 3)
    none, parts = torch.empty(0, dtype=torch.uint8, device=DEV), []
    for dtype in EVERY:
        note("fp8 shapes in place %d %d %d per %d %s" % (M, N, K, per, dtype))
        check(G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype], workspace=none), a, sa, b, sb, per, dtype, parts)


@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("M,N,K", [(2, 2, 200000), (20, 40, 200000), (70, 200, 200000), (70, 200, 140000), (300, 520, 70000), (2300, 1680, 70000),
                                   (1300, 8900, 20000)])
def test_long_sums_are_held_in_32_bits(G, M, N, K, per):  # noqa: F811
    """All-ones codes: whole numbers below 2^24, so a float32 sum is exact in any order, of splits too, and a 16-bit result
    is the sum rounded once; a sum held in 16 bits would stop growing at 256 or 2048."""
    note("fp8 long sums %d %d %d" % (M, N, K))
    wide = (K + 15) // 16 * 16
    a = torch.full((M, wide), 0x38, dtype=torch.uint8, device=DEV)[:, :K]
    b = torch.full((N, wide), 0x38, dtype=torch.uint8, device=DEV)[:, :K]
    blocks = (K + 127) // 128
    sa, sb = torch.full((M, blocks), 0.125, device=DEV), torch.ones(((N + per - 1) // per, blocks), device=DEV)
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        want = torch.tensor(K / 8, dtype=torch.float64).to(dtype)
        out = G.gvr_fp8_matmul(a, sa, b, sb, dtype=dtype)
        assert (out == want.to(DEV)).all()
