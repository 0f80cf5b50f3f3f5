"""CPU oracle for rotary positions, the 4-bit key / value cache and attention
over it -- TEST INFRASTRUCTURE ONLY.

Only ``tests/`` and ``__graft_entry__.smoke()`` may import this module; the
GPU product path never does, and the two share no code. Plain numpy, float64
unless a function says otherwise.

* ``rope_table``  -- c, s = gain * cos, gain * sin of p theta'_i (float64).
* ``rotate``      -- a' = a c - b s, b' = b c + a s on the first R elements
                     of every head, pairs (i, i + R/2) or (2i, 2i+1), in the
                     dtype of x: float64 for the definition, float32 for the
                     kernels' own arithmetic (products and sum rounded once).
* ``quantise``    -- blocks of 32: the least e >= -126 with max|x| <= 7 * 2^e
                     and the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^e
                     (ties to the even code); codes 0 .. 15 (bit 3: sign) and
                     scale bytes e + 127, 255 for a block that is not finite.
* ``record`` / ``values`` -- a token's record bytes, and what one stands for.
* ``attention``   -- softmax attention of one query row over given tokens.

Parity status: pinned by ``tests/test_kv4_pins.py`` (the code table against
the format's bit fields, brute-force nearest codes, hand-worked blocks,
complex-number rotation, two-token attention in closed form, record layout,
planted mistakes).
"""
from __future__ import annotations

import numpy as np

from .rope_prior import yarn_theta

BLOCK = 32
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rope_table(n: int, d: int, gain: float = 1.0, **yarn) -> np.ndarray:
    """[n][d/2][2] float64."""
    phase = np.outer(np.arange(n, dtype=np.float64), yarn_theta(d=d, **yarn))
    return gain * np.stack([np.cos(phase), np.sin(phase)], axis=-1)


def rotate(x, positions, table, interleaved=False, transposed=False) -> np.ndarray:
    """x [T][H][D], positions [T], table [P][R/2][2]; a position outside the
    table gives NaN. Computes in x's dtype, one rounding per operation."""
    x = np.asarray(x)
    R = 2 * table.shape[1]
    pos = np.asarray(positions)
    ok = (pos >= 0) & (pos < table.shape[0])
    cs = table[np.where(ok, pos, 0)].astype(x.dtype)
    cs = np.where(ok[:, None, None], cs, np.nan).astype(x.dtype)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    if transposed:
        s = -s
    y = x.copy()
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y[..., 0:R:2], y[..., 1:R:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y[..., :R // 2], y[..., R // 2:R] = a * c - b * s, b * c + a * s
    return y


def quantise(x):
    """Codes and scale bytes of x [..., 32 n]."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(x.shape[:-1] + (-1, BLOCK))
    top = np.abs(blocks).max(axis=-1)
    finite = np.isfinite(top)
    t = np.where(finite & (top > 0), top, 1.0)
    e = np.ceil(np.log2(t / 7.0)).astype(np.int64)
    # log2 may land a step off at the boundaries: settle by comparison
    e = np.where(t <= 7.0 * np.exp2(e - 1.0), e - 1, e)
    e = np.where(t > 7.0 * np.exp2(e * 1.0), e + 1, e)
    e = np.where(finite & (top > 0), np.maximum(e, -126), -126)
    with np.errstate(invalid="ignore"):
        y = np.abs(blocks) / np.exp2(e * 1.0)[..., None]
        dist = np.abs(np.minimum(y, 6.0)[..., None] - VALUES)
    best = dist.min(axis=-1, keepdims=True)
    near = dist == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), near.argmax(axis=-1))
    code = code + 8 * np.signbit(blocks)
    scale = np.where(finite, e + 127, 255)
    return code.reshape(x.shape).astype(np.uint8), scale.astype(np.uint8)


def dequantise(code, scale):
    """float64 values of codes [..., 32 n] and scale bytes [..., n]."""
    v = np.concatenate([VALUES, -VALUES])[code]
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127.0))
    return v * np.repeat(s, BLOCK, axis=-1)


def record(k, v) -> np.ndarray:
    """Record bytes [T][record] of k and v [T][H][D]."""
    parts, scales = [], []
    for x in (k, v):
        code, scale = quantise(x)
        T = code.shape[0]
        code = code.reshape(T, -1, 2)
        parts.append(code[..., 0] | code[..., 1] << 4)
        scales.append(scale.reshape(T, -1))
    return np.concatenate(parts + scales, axis=1).astype(np.uint8)


def values(rec, heads: int, D: int):
    """k, v [T][heads][D] float64 of record bytes [T][record]."""
    rec = np.asarray(rec, dtype=np.uint8)
    T, half, blocks = rec.shape[0], heads * D // 2, heads * D // BLOCK
    out = []
    for i in range(2):
        b = rec[:, i * half:(i + 1) * half]
        code = np.stack([b & 15, b >> 4], axis=-1).reshape(T, heads * D)
        scale = rec[:, 2 * half + i * blocks:2 * half + (i + 1) * blocks]
        out.append(dequantise(code, scale).reshape(T, heads, D))
    return out


def attention(q, k, v, scale: float):
    """One query row q [q_heads][D] over k, v [n][heads][D]: out [q_heads][D],
    lse [q_heads], and sum_t w_t |v_t| [q_heads][D] (for error bounds)."""
    Hq, D = q.shape
    n, H, _ = k.shape
    out, mag, lse = np.zeros((Hq, D)), np.zeros((Hq, D)), np.full(Hq, -np.inf)
    if n == 0:
        return out, lse, mag
    for h in range(Hq):
        s = scale * (k[:, h * H // Hq] @ q[h])
        m = s.max()
        w = np.exp(s - m)
        lse[h] = m + np.log(w.sum())
        w = w / w.sum()
        out[h] = w @ v[:, h * H // Hq]
        mag[h] = w @ np.abs(v[:, h * H // Hq])
    return out, lse, mag
