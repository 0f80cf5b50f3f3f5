"""Rotary positions on the GPU against the oracle: equal, bit for bit, to its
float32 arithmetic, and within the rounding of the type of the float64
definition; gradients against the formula and against differences; layouts,
strides, sizes and refusals."""
import numpy as np
import pytest
import torch

from oracle import kv4 as O
from tests.gpu_cases import note
from tests.kv4_cases import DEV, TORCH, UNIT, f64

pytestmark = pytest.mark.gpu

P = 700   # positions of the tables


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    return g


def table(rot, gain=1.0):
    return O.rope_table(P, rot, gain).astype(np.float32)


def check(y, x, pos, tab, inter, inv, dtype):
    """Both against the oracle; the float64 bound: two products and a sum in
    float32, then one rounding to the type."""
    x32 = x.detach().cpu().float().numpy()
    want = O.rotate(x32, pos, tab, inter, inv)
    got = y.detach().cpu()
    assert torch.equal(got, torch.from_numpy(want).to(TORCH[dtype])), "differs from the float32 arithmetic"
    ref = O.rotate(x32.astype(np.float64), pos, tab.astype(np.float64), inter, inv)
    size = O.rotate(np.abs(x32).astype(np.float64), pos, np.abs(tab) * [1.0, 1.0], inter, False)
    R = 2 * tab.shape[1]
    size[..., :R] = np.abs(x32).max() * np.abs(tab).max() * 2
    assert (np.abs(f64(y) - ref) <= UNIT[dtype] * np.abs(ref) + 3 * 2.0 ** -24 * size + 2.0 ** -25 * (dtype == "f16")).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (64, 24), (256, 72), (80, 80), (7, 6), (2, 2), (1024, 512)])
def test_rotate(G, dtype, inter, D, rot):
    rng = np.random.default_rng(D * 7 + rot)
    tab = table(rot, gain=1.3)
    for T, H in ((1, 1), (3, 5), (67, 9)):
        for inv in (False, True):
            note("rotate %s inter=%s D=%d rot=%d T=%d H=%d inv=%s" % (dtype, inter, D, rot, T, H, inv))
            x = torch.from_numpy(rng.standard_normal((T, H, D))).to(TORCH[dtype]).to(DEV)
            pos = rng.integers(0, P, T).astype(np.int32)
            y = G.gvr_rope_rotate(x, torch.from_numpy(pos).to(DEV), torch.from_numpy(tab).to(DEV), inter, inv)
            check(y, x, pos, tab, inter, inv, dtype)


def test_many_heads_and_tokens(G):
    """Sizes at which a thread serves several heads, head counts that do not divide."""
    tab = table(64)
    dt = torch.from_numpy(tab).to(DEV)
    for T, H in ((4097, 33), (2048, 100)):
        note("rotate T=%d H=%d" % (T, H))
        g = torch.Generator(device=DEV).manual_seed(T)
        x = torch.randn((T, H, 96), generator=g, device=DEV).bfloat16()
        pos = torch.randint(0, P, (T,), generator=g, device=DEV, dtype=torch.int32)
        y = G.gvr_rope_rotate(x, pos, dt)
        check(y, x, pos.cpu().numpy(), tab, False, False, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_in_place_and_offsets(G, dtype):
    rng = np.random.default_rng(2)
    T, H, D, rot = 21, 3, 64, 32
    tab = table(rot)
    dt, pos = torch.from_numpy(tab).to(DEV), rng.integers(0, P, T).astype(np.int32)
    dpos = torch.from_numpy(pos).to(DEV)
    wide = torch.from_numpy(rng.standard_normal((T, H + 4, D + 8))).to(TORCH[dtype]).to(DEV)
    views = {"aligned": wide[:, 1:1 + H, :D], "odd start": wide[:, :H, 3:3 + D],
             "heads first": wide[:, :H, :D].transpose(0, 1).contiguous().transpose(0, 1)}
    for name, x in views.items():
        note("rotate strided: %s" % name)
        before = wide.clone()
        check(G.gvr_rope_rotate(x, dpos, dt), x, pos, tab, False, False, dtype)
        assert torch.equal(wide, before)
        y = x.clone(memory_format=torch.preserve_format)
        assert G.gvr_rope_rotate(y, dpos, dt, out=y) is y        # in place
        check(y, x, pos, tab, False, False, dtype)
        out = torch.full_like(wide, 9.0)
        G.gvr_rope_rotate(x, dpos, dt, out=out[:, 2:2 + H, 5:5 + D])
        check(out[:, 2:2 + H, 5:5 + D], x, pos, tab, False, False, dtype)
        out[:, 2:2 + H, 5:5 + D] = 9.0
        assert (out == 9.0).all()                                # nothing else was written


def test_positions_outside_the_table(G):
    x = torch.ones((4, 2, 32), device=DEV)
    pos = torch.tensor([-1, P, P - 1, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    for rot, inter in ((16, False), (16, True), (6, False)):
        y = G.gvr_rope_rotate(x, pos, torch.from_numpy(table(rot)).to(DEV), inter).cpu()
        assert torch.isnan(y[[0, 1, 3], :, :rot]).all() and torch.isfinite(y[2]).all() and (y[:, :, rot:] == 1).all()


def test_nothing_to_do(G):
    tab = torch.from_numpy(table(16)).to(DEV)
    assert G.gvr_rope_rotate(torch.empty((0, 4, 32), device=DEV), torch.empty(0, dtype=torch.int32, device=DEV),
                             tab).shape == (0, 4, 32)
    assert G.gvr_rope_rotate(torch.empty((3, 0, 32), device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV),
                             tab).shape == (3, 0, 32)


@pytest.mark.parametrize("inter", [False, True])
def test_gradient(G, inter):
    """inverse=True is the transpose: the formula's gradient, and the
    difference quotient of the rotation (linear, so any step is exact up to
    rounding: float32 products and sums of |x| <= 6, 2^-24 * 60)."""
    rng = np.random.default_rng(8)
    T, H, D, rot = 9, 3, 48, 40
    tab = table(rot, gain=1.2)
    dt = torch.from_numpy(tab).to(DEV)
    pos = torch.from_numpy(rng.integers(0, P, T).astype(np.int32)).to(DEV)
    x, g = (torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(DEV) for _ in range(2))
    gx = G.gvr_rope_rotate(g, pos, dt, inter, inverse=True)
    ref = O.rotate(f64(g), pos.cpu().numpy(), tab.astype(np.float64), inter, True)
    assert np.abs(f64(gx) - ref).max() <= 60 * 2.0 ** -24
    base = f64(G.gvr_rope_rotate(x, pos, dt, inter))
    for j in rng.integers(0, D, 6):
        step = x.clone()
        step[:, 1, j] += 1.0
        moved = (f64(G.gvr_rope_rotate(step, pos, dt, inter)) - base) / (f64(step) - f64(x))[:, 1, j][:, None, None]
        quotient = (moved * f64(g)).sum(axis=(1, 2))
        assert np.abs(quotient - f64(gx)[:, 1, j]).max() <= 8 * 60 * 2.0 ** -24


@pytest.mark.parametrize("kw", [dict(), dict(d_rope=128, scale=1.0), dict(d_rope=2), dict(d_rope=512, base=5e5, scale=8.0)])
def test_table(G, kw):
    """Rounded once from float64: within one unit of float32 of the oracle's."""
    n, gain = 5000, 1.1
    t = f64(G.gvr_rope_table(n, kw or None, gain=gain, device=DEV))
    d = kw.get("d_rope", 64)
    ref = O.rope_table(n, d, gain, **{k: v for k, v in kw.items() if k != "d_rope"})
    assert t.shape == ref.shape and np.abs(t - ref).max() <= gain * 2.0 ** -24 + 1e-11
    assert G.gvr_rope_table(0, device=DEV).shape == (0, 32, 2)


def test_other_stream_and_prepared(G):
    tab = torch.from_numpy(table(64)).to(DEV)
    x = torch.randn((50, 4, 64), device=DEV)
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    want = G.gvr_rope_rotate(x, pos, tab)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = torch.empty_like(x)
    call = G.prepare_gvr_rope_rotate(x, pos, tab, out=got, stream=s)
    assert call() is got and call.out is got
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    x.add_(1.0)
    torch.cuda.synchronize()
    call()
    s.synchronize()
    assert torch.equal(got, G.gvr_rope_rotate(x, pos, tab))


def test_refusals(G):
    x = torch.zeros((4, 2, 64), device=DEV)
    pos, tab = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros((10, 32, 2), device=DEV)
    ok = dict(x=x, positions=pos, table=tab)
    for kw in (dict(x=x.double()), dict(x=x[0]), dict(x=x.cpu()), dict(x=x.transpose(1, 2)), dict(positions=pos.long()),
               dict(positions=pos[:3]), dict(positions=pos.cpu()), dict(table=tab.double()), dict(table=tab[:, :, :1]),
               dict(table=torch.zeros((10, 33, 2), device=DEV)), dict(table=tab[:, :0]), dict(out=torch.zeros_like(x).half()),
               dict(out=torch.zeros((4, 2, 32), device=DEV)), dict(out=torch.zeros((1, 2, 64), device=DEV).expand(4, 2, 64)),
               dict(out=x.cpu())):
        with pytest.raises(ValueError):
            G.gvr_rope_rotate(**{**ok, **kw})
