"""Rotary positions on the GPU at the edges of their sizes: tables of 2^30 positions,
threads that serve several heads, gradients through autograd."""
import numpy as np
import pytest
import torch

from oracle import kv4 as O
from oracle.rope_prior import yarn_theta
from tests.gpu_cases import note
from tests.kv4_cases import DEV, TORCH, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    return g


def test_table_of_more_than_2_30_positions(G):
    """8.6 GB of one pair: the first and last positions and some between."""
    n = 2 ** 30 + 3
    note("table of 2^30 + 3 positions")
    t = G.gvr_rope_table(n, dict(d_rope=2), device=DEV)
    pos = np.unique(np.concatenate([[0, 1, 63, 64, 255, 256, 2 ** 29, 2 ** 30, n - 2, n - 1],
                                    np.random.default_rng(0).integers(0, n, 1000)]))
    got = f64(t[torch.from_numpy(pos).to(DEV)])[:, 0]
    phase = pos * yarn_theta(d=2)[0]
    ref = np.stack([np.cos(phase), np.sin(phase)], axis=-1)
    # float64's own unit of the phase (2^30 * 2^-52), and one rounding to float32
    assert np.abs(got - ref).max() <= 2.0 ** -24 + 2.0 ** -21


def heads_each(T, H, per_head):
    """Heads that a thread serves (plan_items of csrc/rotary_plan.h)."""
    return 2 if H > 1 and T * H * per_head // 2 >= 256 * 2048 else 1


@pytest.mark.parametrize("inv", [False, True])
@pytest.mark.parametrize("dtype,inter,aligned,T", [("bf16", False, True, 8193), ("bf16", True, True, 8193),
                                                   ("f32", False, True, 8193), ("f16", True, True, 8193),
                                                   ("bf16", False, False, 701), ("f32", True, False, 701)])
def test_two_heads_of_a_thread_and_a_last_one(G, dtype, inter, aligned, T, inv):
    """An odd number of heads where threads serve two: the last head is there, and what lies beside the heads is not
    touched. Wide and element-wise kernel."""
    H, D, rot, P = 33, 96, 64, 200
    assert heads_each(T, H, D // 16 if aligned else rot // 2 + D - rot) == 2
    rng = np.random.default_rng(T + inter)
    tab = O.rope_table(P, rot, 1.1).astype(np.float32)
    pos = rng.integers(0, P, T).astype(np.int32)
    at = 8 if aligned else 3
    wide = torch.randn((T, H + 2, D + 16), generator=torch.Generator(device=DEV).manual_seed(T), device=DEV).to(TORCH[dtype])
    x, out = wide[:, 1:1 + H, at:at + D], torch.full_like(wide, 9.0)
    y = out[:, 1:1 + H, at:at + D]
    note("rotate two heads a thread: %s inter=%s aligned=%s T=%d inv=%s" % (dtype, inter, aligned, T, inv))
    G.gvr_rope_rotate(x, torch.from_numpy(pos).to(DEV), torch.from_numpy(tab).to(DEV), inter, inv, out=y)
    want = O.rotate(x.cpu().float().numpy(), pos, tab, inter, inv)
    assert torch.equal(y.cpu(), torch.from_numpy(want).to(TORCH[dtype]))
    y.fill_(9.0)
    assert (out == 9.0).all()


@pytest.mark.parametrize("dtype,rot,inter,aligned", [("bf16", 0, False, True), ("bf16", 64, False, True), ("f32", 32, False, True),
                                                     ("f16", 64, True, True), ("f32", 24, True, False), ("bf16", 64, False, False)])
def test_append_and_read_two_heads_of_a_thread(G, dtype, rot, inter, aligned):
    """As above for the cache: records equal the oracle's, other records stay, and tokens read back stand beside
    untouched heads."""
    T, H, D, P, page = 4097, 33, 64, 200, 64
    assert heads_each(T, H, D // 8) == 2
    rng = np.random.default_rng(rot + aligned)
    tab = O.rope_table(P, rot, 1.1).astype(np.float32) if rot else None
    pos = rng.integers(0, P, T).astype(np.int32)
    at = 8 if aligned else 3
    wide = torch.randn((2, T, H + 1, D + 16), generator=torch.Generator(device=DEV).manual_seed(rot), device=DEV).to(TORCH[dtype])
    k, v = wide[0, :, :H, at:at + D], wide[1, :, 1:, at:at + D]
    pages = (T + page - 1) // page + 1
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    cache = torch.full((pages, page, G.gvr_kv4_record_bytes(H, D)), 77, dtype=torch.uint8, device=DEV)
    kw = dict(table=torch.from_numpy(tab).to(DEV), positions=torch.from_numpy(pos).to(DEV), interleaved=inter) if rot else {}
    note("append two heads a thread: %s rot=%d inter=%s aligned=%s" % (dtype, rot, inter, aligned))
    G.gvr_kv4_append(k, v, torch.from_numpy(slots).to(DEV), cache, **kw)
    k32 = k.cpu().float().numpy()
    rec = O.record(O.rotate(k32, pos, tab, inter) if rot else k32, v.cpu().float().numpy())
    want = np.full((pages * page, rec.shape[1]), 77, np.uint8)
    want[slots] = rec
    assert np.array_equal(cache.cpu().numpy().reshape(want.shape), want)
    back = torch.full_like(wide, 9.0)
    bk, bv = back[0, :, :H, at:at + D], back[1, :, 1:, at:at + D]
    G.gvr_kv4_read(cache, torch.from_numpy(slots).to(DEV), H, D, dtype=TORCH[dtype], k=bk, v=bv)
    ek, ev = O.values(rec, H, D)
    assert np.array_equal(f64(bk), ek) and np.array_equal(f64(bv), ev)
    bk.fill_(9.0)
    bv.fill_(9.0)
    assert (back == 9.0).all()


# ---- gradients through autograd

def rotary(rng, T=9, H=3, D=48, rot=40, dtype="f32", gain=1.2, P=100):
    tab = O.rope_table(P, rot, gain).astype(np.float32)
    pos = rng.integers(0, P, T).astype(np.int32)
    x, g = (torch.from_numpy(rng.standard_normal((T, H, D))).to(TORCH[dtype]).to(DEV) for _ in range(2))
    return x, g, torch.from_numpy(pos).to(DEV), torch.from_numpy(tab).to(DEV), pos, tab


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("inv", [False, True])
def test_backward(G, dtype, inter, inv):
    """The gradient is the transposed rotation of the result's, bit for bit, and the formula's."""
    x, g, pos, tab, pn, tn = rotary(np.random.default_rng(71), dtype=dtype)
    x.requires_grad_()
    y = G.gvr_rope_rotate(x, pos, tab, inter, inv)
    assert y.requires_grad and torch.equal(y.detach(), G.gvr_rope_rotate(x.detach(), pos, tab, inter, inv))
    y.backward(g)
    assert torch.equal(x.grad, G.gvr_rope_rotate(g, pos, tab, inter, not inv))
    want = O.rotate(g.cpu().float().numpy(), pn, tn, inter, not inv)
    assert torch.equal(x.grad.cpu(), torch.from_numpy(want).to(TORCH[dtype]))


def test_backward_against_differences(G):
    """sum(w * rotate(x)): the gradient against difference quotients (linear: exact up to rounding of float32 products
    and sums of |x| <= 6, as in the gradient's other test)."""
    x, w, pos, tab, _, _ = rotary(np.random.default_rng(72))
    x.requires_grad_()
    (w * G.gvr_rope_rotate(x, pos, tab)).sum().backward()
    base = f64(G.gvr_rope_rotate(x.detach(), pos, tab))
    for j in (0, 3, 19, 20, 39, 40, 47):
        step = x.detach().clone()
        step[:, 1, j] += 1.0
        moved = (f64(G.gvr_rope_rotate(step, pos, tab)) - base) / (f64(step) - f64(x))[:, 1, j][:, None, None]
        assert np.abs((moved * f64(w)).sum(axis=(1, 2)) - f64(x.grad)[:, 1, j]).max() <= 8 * 60 * 2.0 ** -24


def test_backward_of_layouts(G):
    """Gradients that are one element expanded (a sum's), strided inputs, and a second derivative."""
    x, g, pos, tab, _, _ = rotary(np.random.default_rng(73))
    wide = torch.randn((9, 5, 60), device=DEV, requires_grad=True)
    G.gvr_rope_rotate(wide[:, 1:4, 3:51], pos, tab).sum().backward()
    want = torch.zeros_like(wide)
    want[:, 1:4, 3:51] = G.gvr_rope_rotate(torch.ones_like(x), pos, tab, inverse=True)
    assert torch.equal(wide.grad, want)
    x.requires_grad_()
    g.requires_grad_()
    gx, = torch.autograd.grad(G.gvr_rope_rotate(x, pos, tab), x, g, create_graph=True)
    gg, = torch.autograd.grad(gx, g, x.detach())
    assert torch.equal(gg, G.gvr_rope_rotate(x.detach(), pos, tab))


def test_out_and_autograd(G):
    """Written in place, into another tensor, and without gradients."""
    x, g, pos, tab, _, _ = rotary(np.random.default_rng(74))
    want = G.gvr_rope_rotate(g, pos, tab, inverse=True)
    for other in (False, True):
        leaf = x.clone().requires_grad_()
        y = leaf * 2.0
        out = torch.empty_like(x) if other else y
        z = G.gvr_rope_rotate(y, pos, tab, out=out)
        assert z is out and z.requires_grad and torch.equal(z.detach(), G.gvr_rope_rotate(2.0 * x, pos, tab))
        z.backward(g)
        assert torch.equal(leaf.grad, 2.0 * want)
    leaf = x.clone().requires_grad_()
    with pytest.raises(ValueError):
        G.gvr_rope_rotate(x, pos, tab, out=leaf)
    with pytest.raises(ValueError):
        G.gvr_rope_rotate(leaf, pos, tab, out=leaf)
    assert torch.equal(leaf.detach(), x)
    # a tensor that a graph has saved, written without gradients: autograd notices
    leaf = x.clone().requires_grad_()
    saved = x.clone()
    product = (leaf * saved).sum()
    with torch.no_grad():
        assert not G.gvr_rope_rotate(leaf, pos, tab).requires_grad
        assert G.gvr_rope_rotate(saved, pos, tab, out=saved) is saved
    with pytest.raises(RuntimeError):
        product.backward()
    with torch.inference_mode():
        y = x.clone()
        assert torch.equal(G.gvr_rope_rotate(y, pos, tab, out=y), G.gvr_rope_rotate(x, pos, tab))
    assert not G.prepare_gvr_rope_rotate(leaf, pos, tab)().requires_grad
