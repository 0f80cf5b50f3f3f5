"""8-bit products of very small and very large matrices: the product of two blocks' scales is a float32 number."""
import numpy as np
import pytest
import torch

import oracle.fp8 as O
from tests.fp8_cases import DEV, TORCH, close, cut_off, product_bound
from tests.gpu_cases import note
from tests.test_gpu_fp8 import G  # noqa: F401

pytestmark = pytest.mark.gpu

SIZES = [(3, 200, 300), (20, 130, 640), (70, 257, 401), (300, 520, 2100), (2003, 1700, 130)]


def pair(rng, M, N, K, per, at):
    """Random matrices around 2^at[0] and 2^at[1], their codes and scales on the GPU and on the host."""
    out = []
    for rows, p, e in ((M, 1, at[0]), (N, per, at[1])):
        codes, scale = O.quantise(rng.standard_normal((rows, K)) * 2.0 ** e, rows=p)
        out += [(torch.from_numpy(codes).to(DEV), torch.from_numpy(scale).to(DEV)), (codes, scale)]
    return out


@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("at", [(-60, -60), (-110, -20), (-30, -108), (60, 40), (100, -100), (-120, 120)])
def test_magnitudes(G, M, N, K, per, at):  # noqa: F811
    """Where the scales' product is below 2^-126 it is rounded to a multiple of 2^-149, so a block is off by 2^-150 times the sum of its
    codes' products besides."""
    note("fp8 magnitudes %s %s" % ((M, N, K, per), at))
    rng = np.random.default_rng(M + K)
    a, (ca, ha), b, (cb, hb) = pair(rng, M, N, K, per, at)
    ref, mag = O.product(ca, ha, cb, hb, per)
    step = 2.0 ** -150 * (np.abs(O.CODES[ca & 0x7F]) @ np.abs(O.CODES[cb & 0x7F]).T)
    cut = cut_off(O.values(ca, ha), O.values(cb, hb, per))
    for dtype in ("f32", "bf16"):
        out = G.gvr_fp8_matmul(*a, *b, dtype=TORCH[dtype])
        close(out, ref, product_bound(mag, ref, K, dtype, cut) + step * 1.01)


@pytest.mark.parametrize("M,N,K", SIZES)
def test_results_past_the_range_are_infinite(G, M, N, K):  # noqa: F811
    note("fp8 past the range %s" % ((M, N, K),))
    rng = np.random.default_rng(M)
    a, (ca, ha), b, (cb, hb) = pair(rng, M, N, K, 128, (100, 60))
    a[0].bitwise_and_(0x7F)
    b[0].bitwise_and_(0x7F)   # (no term is negative, so no two infinities meet)
    a[0].clamp_(min=0x38)
    b[0].clamp_(min=0x38)     # (nor is any zero)
    for dtype in ("f32", "bf16", "f16"):
        assert (G.gvr_fp8_matmul(*a, *b, dtype=TORCH[dtype]) == float("inf")).all()
