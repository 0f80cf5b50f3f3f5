"""Pins of the oracle of rotary positions and the 4-bit cache (CPU): the
definition checked by other means, and planted mistakes that must be caught."""
import numpy as np
import pytest

from oracle import kv4 as O
from oracle.rope_prior import yarn_theta


def test_codes_are_the_formats_bit_fields():
    for c in range(16):
        e, m = (c >> 1) & 3, c & 1
        v = (m * 0.5 if e == 0 else 2.0 ** (e - 1) * (1 + m / 2)) * (-1 if c & 8 else 1)
        assert O.dequantise(np.full(32, c, np.uint8), np.array([127], np.uint8))[0] == v


def test_nearest_code_brute_force():
    rng = np.random.default_rng(3)
    x = np.concatenate([rng.standard_normal(32 * 200), rng.standard_normal(32 * 20) * 1e-30,
                        rng.standard_normal(32 * 20) * 1e30]).reshape(-1, 32)
    code, scale = O.quantise(x)
    val = O.dequantise(code, scale)
    step = np.exp2(scale.astype(np.float64) - 127)
    grid = np.concatenate([O.VALUES, -O.VALUES])
    for b in range(x.shape[0]):
        top = np.abs(x[b]).max()
        assert top <= 7 * step[b, 0] and top > 3.5 * step[b, 0]      # the least power of two that serves
        best = np.abs(x[b][:, None] - grid * step[b, 0]).min(axis=1)
        assert np.array_equal(np.abs(x[b] - val[b]), best)


def test_hand_worked_block():
    x = np.zeros(32)
    x[:10] = [7.0, 6.9, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.3]   # e = 0: ties to the even code
    code, scale = O.quantise(x)
    assert scale[0] == 127
    assert O.dequantise(code, scale)[:10].tolist() == [6, 6, 4, 4, 2, 2, 1, 1, 0, -0.5]
    x[0] = np.nextafter(7.0, 8.0)                                      # one step past: the scale doubles
    assert O.quantise(x)[1][0] == 128
    assert O.quantise(np.zeros(32))[1][0] == 1 and not O.quantise(np.zeros(32))[0].any()
    x[0] = np.inf
    assert O.quantise(x)[1][0] == 255
    x[0] = np.nan
    assert O.quantise(x)[1][0] == 255 and np.isnan(O.dequantise(*O.quantise(x))).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(5)
    T, H, D, R = 5, 3, 64, 40
    x = rng.standard_normal((T, H, D))
    pos = rng.integers(0, 100, T)
    y = O.rotate(x, pos, O.rope_table(100, R, gain=1.25), interleaved)
    th = yarn_theta(d=R)
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    z = (a + 1j * b) * 1.25 * np.exp(1j * pos[:, None, None] * th)
    got = (y[..., 0:R:2] + 1j * y[..., 1:R:2]) if interleaved else (y[..., :R // 2] + 1j * y[..., R // 2:R])
    assert np.allclose(got, z, atol=1e-13) and np.array_equal(y[..., R:], x[..., R:])
    # the transposed rotation is the gradient: <R x, g> = <x, R^T g>
    g = rng.standard_normal(x.shape)
    back = O.rotate(g, pos, O.rope_table(100, R, gain=1.25), interleaved, transposed=True)
    assert np.isclose((y * g).sum(), (x * back).sum(), rtol=1e-12)


def test_rotation_outside_the_table_is_nan():
    y = O.rotate(np.ones((3, 1, 8)), [-1, 10, 9], O.rope_table(10, 4))
    assert np.isnan(y[:2, 0, :4]).all() and np.isfinite(y[2]).all() and (y[:, :, 4:] == 1).all()


def test_record_layout():
    H, D = 2, 64
    k, v = np.zeros((1, H, D)), np.zeros((1, H, D))
    k[0, 1, 33] = 3.0      # head 1, second block, odd element: 3 = 6 * 2^-1 -> e = -1, code 7 in the high bits
    v[0, 0, 2] = -1.0      # head 0, first block, even element: -1 = -4 * 2^-2 -> e = -2, code 14
    r = O.record(k, v)[0]
    assert r.size == H * D * 17 // 16
    nz = {i: int(b) for i, b in enumerate(r) if b not in (0, 1)}
    assert nz == {D // 2 + 16: 7 << 4, H * D // 2 + 1: 14, H * D + 3: 126, H * D + 4: 125}
    kk, vv = O.values(r[None], H, D)
    assert np.array_equal(kk, k) and np.array_equal(vv, v)


def test_two_token_attention_closed_form():
    q = np.array([[1.0, 0.0], [0.0, 2.0]])
    k = np.array([[[1.0, 1.0]], [[-1.0, 0.5]]])
    v = np.array([[[1.0, 0.0]], [[0.0, 4.0]]])
    out, lse, mag = O.attention(q, k, v, 0.5)
    for h, (s0, s1) in enumerate([(0.5, -0.5), (1.0, 0.5)]):
        w = 1 / (1 + np.exp(s1 - s0))
        assert np.allclose(out[h], [w, 4 * (1 - w)]) and np.isclose(lse[h], np.log(np.exp(s0) + np.exp(s1)))
    out, lse, _ = O.attention(q, k[:0], v[:0], 0.5)
    assert not out.any() and np.isneginf(lse).all()


def test_planted_mistakes_are_seen():
    """Wrong variants of the definition differ from the oracle on ordinary inputs."""
    rng = np.random.default_rng(9)
    x = rng.standard_normal((4, 2, 64))
    code, scale = O.quantise(x)
    top = np.abs(x.reshape(4, 2, 2, 32)).max(-1)
    floor_rule = np.floor(np.log2(top)) - 2 + 127            # saturates up to 8 instead of moving the scale
    assert (floor_rule.reshape(scale.shape) != scale).any()
    t = O.rope_table(50, 32)
    pos = np.array([3, 11, 20, 49])
    assert not np.allclose(O.rotate(x, pos, t), O.rotate(x, pos, t, interleaved=True))
    assert not np.allclose(O.rotate(x, pos, t), O.rotate(x, pos, t, transposed=True))
    assert not np.allclose(O.rotate(x, pos, t), O.rotate(x, pos + 1 - 2 * (pos > 40), t))
    k, v = O.values(O.record(x, -x), 2, 64)
    swapped = O.values(np.roll(O.record(x, -x), 64, axis=1), 2, 64)
    assert not np.array_equal(np.nan_to_num(swapped[0]), k) and np.array_equal(k, -v)
