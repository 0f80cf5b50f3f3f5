"""What pins the oracle of 8-bit matrices (CPU)."""
from fractions import Fraction

import numpy as np
import pytest

import oracle.fp8 as O


def test_code_table():
    assert len(O.CODES) == 127 and O.CODES[0] == 0 and O.CODES[126] == 448 and np.all(np.diff(O.CODES) > 0)
    assert [O.CODES[i] for i in (1, 7, 8, 9, 0x38, 0x39)] == [2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 1.125 * 2.0 ** -6, 1.0, 1.125]


def by_fractions(x, m):
    """The code nearest to 448 x / m, without any rounding."""
    q = abs(Fraction(float(x))) * 448 / Fraction(float(m))
    d = [abs(Fraction(float(c)) - q) for c in O.CODES]
    best = min(d)
    near = [i for i, v in enumerate(d) if v == best]
    return [i for i in near if i % 2 == 0][0] if len(near) > 1 else near[0]


@pytest.mark.parametrize("top", [1.75, 1.0, 448.0, 3.14159, 2.0 ** -130, 0.0, 1.640625, 1e30])
def test_codes_by_fractions(top):
    rng = np.random.default_rng(3)
    top = float(np.float32(top))
    m = max(top, 448 * 2.0 ** -126)
    x = np.float32(rng.standard_normal(60) * m / 3).clip(-m, m)
    x = np.concatenate([x, np.float32([k / 16 * m / 448 for k in range(1, 120, 2)])[:60],
                        np.float32([2.0 ** -10 * m / 448, 3 * 2.0 ** -10 * m / 448, top, -top])])
    x = x[:124][np.abs(x[:124]) <= top]
    row = np.zeros((1, 128), np.float32)
    row[0, :len(x)], row[0, -1] = x, top
    codes, scale = O.quantise(row)
    assert scale[0, 0] == np.float32(m) / np.float32(448)
    for v, c in zip(row[0], codes[0]):
        assert by_fractions(v, m) == c % 128 and (c >= 128) == np.signbit(v), (v, c)


def test_hand_worked():
    row = np.zeros((2, 130))
    row[0, :4] = [448, 1, -1.0625, 17]     # scale 1: 1; 1.0625 is between 1 and 1.125: even is 1; 17: 16 and 18, even is 16
    row[1, 129] = 7.0
    codes, scale = O.quantise(row)
    assert list(codes[0, :4]) == [0x7E, 0x38, 0xB8, 0x58] and scale[0, 0] == 1 and scale[0, 1] == np.float32(2.0 ** -126)
    assert scale[1, 1] == 2.0 ** -6 and codes[1, 129] == 0x7E and codes[1, :128].max() == 0
    codes, scale = O.quantise(row, pow2=True)
    assert scale[1, 1] == 2.0 ** -6 and scale[0, 0] == 1
    row[1, 129] = 7.5   # above 448 * 2^-6: the next power of two
    codes, scale = O.quantise(row, pow2=True)
    assert scale[1, 1] == 2.0 ** -5 and O.values(codes, scale)[1, 129] == 7.5
    codes, scale = O.quantise(row, rows=128)
    assert scale.shape == (1, 2) and scale[0, 0] == 1 and O.values(codes, scale, 128)[0, 3] == 16


def test_not_finite():
    x = np.ones((3, 256))
    x[0, 5], x[1, 200], x[2, 130] = np.inf, np.nan, -np.inf
    codes, scale = O.quantise(x)
    assert np.isnan(scale).tolist() == [[True, False], [False, True], [False, True]]
    assert (codes[0, :128] == 0x7F).all() and (codes[0, 128:] == 0x7E).all()


def test_half_a_step():
    """Every element is at most half a step from its code: 2^-4 of it, or 2^-10 scales, and the scale's rounding."""
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((40, 300)) * np.exp(3 * rng.standard_normal((40, 300)))).astype(np.float32)
    for kw in (dict(), dict(pow2=True), dict(rows=128)):
        c, s = O.quantise(x, **kw)
        unit = O.values(np.full(c.shape, 0x38, np.uint8), s, kw.get("rows", 1))
        assert np.all(np.abs(O.values(c, s, kw.get("rows", 1)) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * unit) + 2.0 ** -23 * np.abs(x))


def test_product_by_loops():
    rng = np.random.default_rng(7)
    a, sa = O.quantise(rng.standard_normal((3, 140)))
    w = rng.standard_normal((131, 140))
    for rows in (1, 128):
        b, sb = O.quantise(w, rows=rows)
        got, mag = O.product(a, sa, b, sb, rows)
        for m, n in ((0, 0), (2, 130), (1, 127), (2, 128)):
            t = [float(O.CODES[a[m, k] & 127]) * (-1) ** int(a[m, k] >> 7) * float(sa[m, k // 128])
                 * float(O.CODES[b[n, k] & 127]) * (-1) ** int(b[n, k] >> 7) * float(sb[n // rows, k // 128]) for k in range(140)]
            assert abs(sum(t) - got[m, n]) < 1e-12 and abs(sum(map(abs, t)) - mag[m, n]) < 1e-12


def test_planted_mistakes():
    """The pins above would catch: truncation, ties away, a scale of 240, the scale dropped, blocks of 64."""
    y = np.array([1.0625, 1.1875, 17.0, 3 * 2.0 ** -10, 448.0])
    good = O.nearest(y)
    trunc = np.searchsorted(O.CODES, y, side="right") - 1
    away = np.array([np.argmin(np.abs(O.CODES - v * (1 + 1e-12))) for v in y])
    assert (trunc != good).any() and (away != good).any()
    x = np.linspace(-3, 3, 256).reshape(1, 256)
    c, s = O.quantise(x)
    assert s[0, 0] != np.float32(3 / 240) and not np.allclose(O.values(c, np.ones_like(s)), x, rtol=0.1)
    narrow = np.abs(x.reshape(1, 4, 64)).max(-1) / 448
    assert not np.allclose(np.repeat(s, 2, axis=1), narrow)
