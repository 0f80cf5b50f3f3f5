"""Inputs and bounds of the GPU tests of 8-bit matrices."""
import numpy as np
import torch

import oracle.fp8 as O
from tests.kv4_cases import DEV, TORCH, UNIT  # noqa: F401

LEAST = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}   # half the least step of a type


def matrix(rng, rows, cols, per=1, pad=0, spread=1.0, zero_tail=False):
    """Codes [rows][cols] (a view of rows `pad` bytes longer, the rest NaN codes) and scales on the GPU, and on the host."""
    x = rng.standard_normal((rows, cols)) * np.exp(spread * rng.standard_normal((rows, 1)))
    codes, scale = O.quantise(x, rows=per)
    wide = np.full((rows, cols + pad), 0x7F, np.uint8)
    wide[:, :cols] = codes
    return torch.from_numpy(wide).to(DEV)[:, :cols], torch.from_numpy(scale).to(DEV), codes, scale


def cut_off(va, vb):
    """What the FP8 matrix cores may cut off: 7 * 2^-13 of the largest product of every eight consecutive elements
    (values va [M][K], vb [N][K])."""
    a, b = (torch.from_numpy(np.pad(np.abs(v), ((0, 0), (0, -v.shape[1] % 8)))).to(DEV) for v in (va, vb))
    total = torch.zeros((a.shape[0], b.shape[0]), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // max(1, 8 * b.shape[0]))
    for m in range(0, a.shape[0], step):
        for k in range(0, a.shape[1], 8):
            total[m:m + step] += (a[m:m + step, None, k:k + 8] * b[None, :, k:k + 8]).amax(dim=-1)
    return 7 * 2.0 ** -13 * total.cpu().numpy()


def product_bound(mag, ref, K, dtype, cut=None):
    """(K + 2 K / 128 + 4) 2^-24 of the magnitudes: a float32 rounding for each addition of a block's K terms and of the
    blocks, two for the scales of each block; for 16-bit results what the FP8 matrix cores cut off; then the result's own
    rounding."""
    b = (K + 2 * ((K + 127) // 128) + 4) * 2.0 ** -24 * mag
    if dtype != "f32":
        b = b + cut
    return b + UNIT[dtype] * (np.abs(ref) + b) + LEAST[dtype]


def close(got, ref, bound):
    got = got.detach().double().cpu().numpy()
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), "%d of %d off, worst %.3g of its bound at %s" % (
        bad.sum(), bad.size, np.nanmax(np.abs(got - ref) / bound), np.argwhere(bad)[0])
