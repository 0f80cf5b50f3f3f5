"""CPU oracle for 8-bit matrices with a scale per 128 elements -- TEST
INFRASTRUCTURE ONLY.

Only ``tests/`` and ``__graft_entry__.smoke()`` may import this module; the
GPU product path never does, and the two share no code. Plain numpy.

* ``quantise``  -- codes (bytes) and float32 scales of x [..., R, C], blocks of
                   128 columns of one row or of 128 rows: m = max|x| of the block, at
                   least 448 * 2^-126; scale m / 448 (rounded to float32), or the least power of two
                   >= m / 448; the code nearest to 448 x / m (x / scale), ties to the
                   even code; NaN scale and codes for a block that is not finite.
* ``values``    -- what codes and scales stand for (float64).
* ``product``   -- A B^T of two such matrices, and the sum of the terms' magnitudes.

With x = a 2^i and m = b 2^j, a and b below 2^24, and a border t 2^k of two codes,
t below 2^5, the quotient 448 x / m differs from the border by nothing or by an
integer over b and a power of two: relatively by 1 / (448 a) > 2^-33 at least. So
its float64 value is on a border only if the quotient is.

Parity status: pinned by ``tests/test_fp8_pins.py`` (the code table against the
format's bit fields, brute-force nearest codes in fractions, hand-worked blocks,
products by loops, planted mistakes).
"""
from __future__ import annotations

import numpy as np

from .indexer import decode_e4m3

BLOCK, MOST = 128, 448.0
CODES = decode_e4m3(np.arange(127))   # 0 .. 448, ascending


def nearest(y):
    """Bytes of the codes nearest to y (finite, |y| <= 448), ties to the even code."""
    y = np.asarray(y, dtype=np.float64)
    size = np.minimum(np.abs(y), MOST)
    hi = np.clip(np.searchsorted(CODES, size), 1, 126)
    lo = hi - 1
    up, down = CODES[hi] - size, size - CODES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code + np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def scales(top, pow2=False):
    """float32 scales and float64 magnitudes of code 448 of blocks whose largest magnitudes are `top`."""
    m = np.maximum(np.asarray(top, dtype=np.float64), MOST * 2.0 ** -126)
    if not pow2:
        return (m.astype(np.float32) / np.float32(MOST)).astype(np.float32), m
    frac, e = np.frexp(m / MOST)
    e = np.where(frac > 0.5, e, e - 1)
    s = np.exp2(e.astype(np.float64))
    return s.astype(np.float32), s * MOST


def quantise(x, pow2=False, rows=1):
    """Codes [..., R, C] and scales [..., R / rows, C / 128] (rounded up)."""
    x = np.asarray(x, dtype=np.float64)
    R, C = x.shape[-2:]
    nr, nc = -(-R // rows), -(-C // BLOCK)
    full = np.zeros(x.shape[:-2] + (nr * rows, nc * BLOCK))
    full[..., :R, :C] = x
    tiles = full.reshape(x.shape[:-2] + (nr, rows, nc, BLOCK))
    finite = np.isfinite(tiles).all(axis=(-3, -1))
    with np.errstate(invalid="ignore"):
        top = np.where(finite, np.abs(tiles).max(axis=(-3, -1)), 1.0)
    scale, m = scales(top, pow2)
    keep = finite[..., :, None, :, None]
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(keep, tiles * MOST / m[..., :, None, :, None], 0.0)
    codes = np.where(keep, nearest(y), 0x7F).astype(np.uint8)
    codes = codes.reshape(x.shape[:-2] + (nr * rows, nc * BLOCK))[..., :R, :C]
    return codes, np.where(finite, scale, np.float32(np.nan))


def values(codes, scale, rows=1):
    codes, scale = np.asarray(codes), np.asarray(scale, dtype=np.float64)
    R, C = codes.shape[-2:]
    s = np.repeat(np.repeat(scale, BLOCK, axis=-1)[..., :C], rows, axis=-2)[..., :R, :]
    return decode_e4m3(codes) * s


def product(a, a_scale, b, b_scale, rows=1):
    """A B^T and sum |terms| [M][N] (float64); `rows`: B's rows per scale."""
    va, vb = values(a, a_scale), values(b, b_scale, rows)
    return va @ vb.T, np.abs(va) @ np.abs(vb).T
