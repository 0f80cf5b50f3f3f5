"""8-bit matrices with a scale per 128 elements on the GPU against the oracle: codes and scales bit for bit, products
within rounding."""
import numpy as np
import pytest
import torch

import oracle.fp8 as O
from oracle import kv4 as OK
from tests.fp8_cases import DEV, TORCH, UNIT, close, cut_off, matrix, product_bound
from tests.gpu_cases import note

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    return g


def same(t, a, what=""):
    """Equal bits (NaN where NaN)."""
    t = t.cpu().numpy()
    assert t.shape == a.shape, what
    assert np.array_equal(t, a, equal_nan=t.dtype.kind == "f"), (what, np.argwhere(~((t == a) | ((t != t) & (a != a))))[:3])


def given(rng, shape, dtype, odd=0):
    """Values of the type, some rows large, some tiny, with elements on the borders of codes; `odd`: elements that the
    storage is shifted by."""
    x = rng.standard_normal(shape) * np.exp(2 * rng.standard_normal(shape[:-1] + (1,)))
    flat = x.reshape(-1, shape[-1])
    flat[::3] = np.round(flat[::3] * 8) / 8
    if flat.shape[0] > 4:
        flat[3] = 0.0
        flat[4] *= 2.0 ** -13
    t = torch.from_numpy(x).to(TORCH[dtype])
    n = t.numel()
    store = torch.empty(n + odd, dtype=t.dtype, device=DEV)
    store[odd:] = t.reshape(-1).to(DEV)
    return store[odd:].view(shape), t.float().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1, 128), (5, 3, 64), (7, 1, 1), (4, 2, 130), (3, 64, 128), (33, 5, 96), (9, 1, 1000),
                                   (2, 1, 4104), (6, 2, 256)])
@pytest.mark.parametrize("pow2", [False, True])
def test_heads(G, dtype, shape, pow2):
    note("fp8 heads %s %s %s" % (dtype, shape, pow2))
    rng = np.random.default_rng(sum(shape))
    for odd in (0, 1):
        x, h = given(rng, shape, dtype, odd)
        codes, scale = G.gvr_fp8_quantize(x, pow2=pow2)
        ref = O.quantise(h, pow2)
        same(scale, ref[1], "scale")
        same(codes, ref[0], "codes")
    flat = G.gvr_fp8_quantize(x[:, 0], pow2=pow2)
    same(flat.codes, ref[0][:, 0])
    same(flat.scale, ref[1][:, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot,inter", [(128, 64, False), (128, 128, True), (64, 64, False), (64, 24, True), (192, 40, False),
                                         (256, 256, False), (130, 128, True), (128, 2, False)])
def test_rotated_heads_into_a_cache(G, dtype, D, rot, inter):
    note("fp8 rotated %s %d %d %s" % (dtype, D, rot, inter))
    rng = np.random.default_rng(D + rot)
    T, H, rows = 37, 3, 90
    x, h = given(rng, (T, H + 2, D), dtype)
    x, h = x[:, 1:H + 1], h[:, 1:H + 1]
    table = OK.rope_table(50, rot).astype(np.float32)
    pos = rng.integers(0, 50, T).astype(np.int32)
    pos[3], pos[4] = -1, 50    # outside the table
    slots = rng.permutation(rows)[:T].astype(np.int64)
    slots[::7], slots[5], slots[6] = -1, rows, -(2 ** 40)
    codes = torch.full((rows, H, D), 0x55, dtype=torch.uint8, device=DEV)
    scale = torch.full((rows, H, (D + 127) // 128), 9.0, device=DEV)
    G.gvr_fp8_quantize(x, torch.from_numpy(table).to(DEV), torch.from_numpy(pos).to(DEV), inter, True,
                       torch.from_numpy(slots).to(DEV), codes, scale)
    c, s = O.quantise(OK.rotate(h, pos, table, inter), True)
    want = np.full((rows, H, D), 0x55, np.uint8), np.full(tuple(scale.shape), 9.0, np.float32)
    ok = (slots >= 0) & (slots < rows)
    want[0][slots[ok]], want[1][slots[ok]] = c[ok], s[ok]
    same(scale, want[1])
    same(codes, want[0])


def test_infinities_and_nan_stay_in_their_block(G):
    note("fp8 not finite")
    x = torch.ones((4, 2, 300), device=DEV)
    x[0, 0, 3], x[1, 1, 200], x[2, 0, 299], x[3, 1, 130] = float("inf"), float("nan"), float("-inf"), 3e38
    for kw in (dict(), dict(pow2=True)):
        codes, scale = G.gvr_fp8_quantize(x, **kw)
        ref = O.quantise(x.cpu().numpy(), kw.get("pow2", False))
        same(codes, ref[0])
        same(scale, ref[1])
    m, t = G.gvr_fp8_quantize_matrix(x.view(8, 300), transposed=True)
    for got, a in ((m, x.view(8, 300)), (t, x.view(8, 300).T)):
        ref = O.quantise(a.cpu().numpy())
        same(got.codes, ref[0])
        same(got.scale, ref[1])


def test_strided_outputs_and_what_lies_between(G):
    note("fp8 strided outputs")
    rng = np.random.default_rng(2)
    x, h = given(rng, (11, 3, 100), "bf16")
    store = torch.full((11, 5, 117), 0x55, dtype=torch.uint8, device=DEV)
    scales = torch.full((11, 5, 2), 9.0, device=DEV)
    G.gvr_fp8_quantize(x, codes=store[:, 1:4, 3:103], scale=scales[:, 2:5, 1:])
    ref = O.quantise(h)
    want = np.full(store.shape, 0x55, np.uint8)
    want[:, 1:4, 3:103] = ref[0]
    same(store, want)
    want = np.full(scales.shape, 9.0, np.float32)
    want[:, 2:5, 1:] = ref[1]
    same(scales, want)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R,C", [(1, 1), (1, 300), (300, 1), (127, 129), (128, 128), (256, 384), (131, 1000), (17, 64)])
@pytest.mark.parametrize("square", [False, True])
def test_matrices(G, dtype, R, C, square):
    note("fp8 matrix %s %d %d %s" % (dtype, R, C, square))
    rng = np.random.default_rng(R + C)
    per = 128 if square else 1
    for pow2, more in ((False, 0), (True, 3)):
        wide, h = given(rng, (R, C + more), dtype)
        x, h = wide[:, more:], h[:, more:]
        a, b = G.gvr_fp8_quantize_matrix(x, square=square, transposed=True, pow2=pow2)
        for got, m in ((a, h), (b, h.T)):
            ref = O.quantise(m, pow2, per)
            same(got.scale, ref[1], "scale")
            same(got.codes, ref[0], "codes")
        for kw in (dict(), dict(straight=False, transposed=True)):   # each alone, into rows of odd strides
            n, m = (R, C) if kw.get("straight", True) else (C, R)
            store = torch.full((n + 1, m + 5), 0x55, dtype=torch.uint8, device=DEV)
            scale = torch.full(((m + 127) // 128, (n + per - 1) // per), 9.0, device=DEV).T
            out = (store[:n, 2:m + 2], scale)
            G.gvr_fp8_quantize_matrix(x, square=square, pow2=pow2, **kw, **{"out" if not kw else "out_transposed": out})
            ref = O.quantise(h if not kw else h.T, pow2, per)
            want = np.full(store.shape, 0x55, np.uint8)
            want[:n, 2:m + 2] = ref[0]
            same(store, want)
            same(scale, ref[1])


SIZES = [(1, 1, 1), (1, 16, 128), (1, 4096, 256), (2, 129, 127), (3, 64, 2048), (16, 16, 129), (17, 300, 640), (33, 130, 16),
         (64, 64, 64), (65, 257, 384), (128, 512, 1000), (128, 8, 4096), (130, 128, 130), (200, 1, 512), (256, 256, 256),
         (257, 255, 257), (300, 700, 1153), (513, 520, 128), (1, 257, 8191), (40, 96, 8320)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("per", [1, 128])
def test_products(G, M, N, K, per):
    note("fp8 product %d %d %d %d" % (M, N, K, per))
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    dtype = ["bf16", "f16", "f32"][(M + N + K) % 3]
    for pad in (-K % 16, 0, 5):   # rows of a multiple of 16 bytes, packed ones, and of any other length
        a, sa, ca, ha = matrix(rng, M, K, pad=pad)
        b, sb, cb, hb = matrix(rng, N, K, per, pad=pad)
        out = G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype])
        ref, mag = O.product(ca, ha, cb, hb, per)
        close(out, ref, product_bound(mag, ref, K, dtype, cut_off(O.values(ca, ha), O.values(cb, hb, per))))
        assert torch.equal(out, G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_strides_of_everything(G, dtype):
    note("fp8 product strides %s" % dtype)
    rng = np.random.default_rng(4)
    M, N, K = 70, 150, 400
    a, sa, ca, ha = matrix(rng, M, K, pad=13)
    b, sb, cb, hb = matrix(rng, N, K, 128, pad=32)
    store = torch.full((M, N + 9), 7.0, dtype=TORCH[dtype], device=DEV)
    turned = sa.T.contiguous().T   # scales block after block
    wide = torch.full((2, 9), float("nan"), device=DEV)
    wide[:, 1::2] = sb
    G.gvr_fp8_matmul(a, turned, b, wide[:, 1::2], out=store[:, 3:N + 3])
    ref, mag = O.product(ca, ha, cb, hb, 128)
    close(store[:, 3:N + 3], ref, product_bound(mag, ref, K, dtype, cut_off(O.values(ca, ha), O.values(cb, hb, 128))))
    assert (store[:, :3] == 7).all() and (store[:, N + 3:] == 7).all()
    every = sa[:, :1].expand(M, sa.shape[1])   # one scale for a whole row
    got = G.gvr_fp8_matmul(a, every, b, sb, dtype=TORCH[dtype])
    assert torch.equal(got, G.gvr_fp8_matmul(a, every.contiguous(), b, sb, dtype=TORCH[dtype]))


def test_nan_codes_and_scales_stay_in_their_row_and_column(G):
    note("fp8 product nan")
    rng = np.random.default_rng(6)
    for M, N, K in ((3, 70, 300), (150, 140, 300), (300, 300, 512)):
        a, sa, ca, ha = matrix(rng, M, K)
        b, sb, cb, hb = matrix(rng, N, K)
        a[1, 5] = 0x7F
        b[9, 290] = 0xFF
        sb[20, 1] = float("inf")
        sa[2, 0] = float("nan")
        out = G.gvr_fp8_matmul(a, sa, b, sb, dtype=torch.float32).cpu().numpy()
        nan = np.zeros((M, N), bool)
        nan[1], nan[2], nan[:, 9] = True, True, True
        ref, mag = O.product(ca, ha, cb, hb)
        assert np.array_equal(np.isnan(np.delete(out, 20, 1)), np.delete(nan, 20, 1))
        rest = np.setdiff1d(np.arange(M), [1, 2])
        assert not np.isfinite(out[rest, 20]).any()
        ok = ~nan
        ok[:, 20] = False
        assert np.all(np.abs(out - ref)[ok] <= product_bound(mag, ref, K, "f32")[ok])


def test_empty_sums_and_empty_products(G):
    note("fp8 product empty")
    z = torch.zeros((5, 0), dtype=torch.uint8, device=DEV)
    s = torch.zeros((5, 0), device=DEV)
    out = torch.full((5, 5), 7.0, device=DEV)
    G.gvr_fp8_matmul(z, s, z, s, out=out)
    assert (out == 0).all()
    a, sa, _, _ = matrix(np.random.default_rng(0), 4, 200)
    none, no_scale = a[:0], sa[:0]
    assert G.gvr_fp8_matmul(none, no_scale, a, sa).shape == (0, 4)
    assert G.gvr_fp8_matmul(a, sa, none, no_scale).shape == (4, 0)
    assert G.gvr_fp8_quantize(torch.zeros((0, 3, 128), device=DEV)).codes.shape == (0, 3, 128)
    assert G.gvr_fp8_quantize(torch.zeros((3, 0, 128), device=DEV)).scale.shape == (3, 0, 1)
    assert G.gvr_fp8_quantize_matrix(torch.zeros((0, 100), device=DEV)).scale.shape == (0, 1)


def test_replayed_graph(G):
    note("fp8 graph")
    rng = np.random.default_rng(8)
    x = torch.randn((100, 640), device=DEV).bfloat16()
    w = G.gvr_fp8_quantize_matrix(torch.randn((500, 640), device=DEV), square=True)
    pq = G.prepare_gvr_fp8_quantize(x)
    pm = G.prepare_gvr_fp8_matmul(*pq.out, *w)
    pq(), pm()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pq = G.prepare_gvr_fp8_quantize(x)
        pm = G.prepare_gvr_fp8_matmul(*pq(), *w)
        pm()
    for i in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal((100, 640))))
        g.replay()
        torch.cuda.synchronize()
        eager = G.gvr_fp8_matmul(*G.gvr_fp8_quantize(x), *w)
        assert torch.equal(eager, pm.out), i


def linear_reference(x, w, dy):
    """Formula in float64 from the oracle's codes; bounds of y, dx, dw before their own rounding, and of dx, dw against
    the gradients of the codes' own product."""
    K, N, M = x.shape[1], w.shape[0], x.shape[0]
    qx, qw = O.quantise(x), O.quantise(w, rows=128)
    qd, qdt, qxt = O.quantise(dy), O.quantise(dy.T), O.quantise(x.T)
    y, my = O.product(*qx, *qw, 128)
    vw, vd, vx = O.values(*qw, 128), O.values(*qd), O.values(*qx)
    dx, mx = vd @ vw, np.abs(vd) @ np.abs(vw)
    dw, mw = O.product(*qdt, *qxt)
    return ((y, my, K, cut_off(vx, vw)), (dx, mx, N, cut_off(vd, vw.T)),
            (dw, mw, M, cut_off(O.values(*qdt), O.values(*qxt))), vw, vx)


@pytest.mark.parametrize("M,K,N,dtype,weight", [(1, 128, 128, "bf16", "bf16"), (5, 100, 40, "f32", "f32"), (129, 257, 130, "bf16", "f32"),
                                                 (200, 384, 256, "f16", "f16"), (33, 1, 3, "f32", "f32")])
def test_linear_and_its_gradients(G, M, K, N, dtype, weight):
    note("fp8 linear %d %d %d %s" % (M, K, N, dtype))
    rng = np.random.default_rng(M + K + N)
    x = torch.from_numpy(rng.standard_normal((M, K))).to(DEV, TORCH[dtype]).requires_grad_()
    w = torch.from_numpy(rng.standard_normal((N, K)) / 8).to(DEV, TORCH[weight]).requires_grad_()
    dy = torch.from_numpy(rng.standard_normal((M, N))).to(DEV, TORCH[dtype])
    y = G.gvr_fp8_linear(x, w)
    y.backward(dy)
    hx, hw, hd = (t.detach().double().cpu().numpy() for t in (x, w, dy))
    ry, rx, rw, vw, vx = linear_reference(hx, hw, hd)
    bounds = []
    for got, (ref, mag, n, cut), t in ((y, ry, dtype), (x.grad, rx, dtype), (w.grad, rw, weight)):
        bounds.append(product_bound(mag, ref, n, t, cut))
        close(got, ref, bounds[-1])
    # differences of <dy, X W^T> in the codes' values X and W (linear in each, so a step of one is exact): an element of dy or
    # x that enters a gradient is off by half a step of its code, 2^-4 of it or 2^-10 of its block's scale
    def off(a):
        c, s = O.quantise(a)
        unit = O.values(np.full(c.shape, 0x38, np.uint8), s)
        return np.maximum(2.0 ** -4 * np.abs(a), 2.0 ** -10 * unit) * 1.001
    f = lambda X, W: float((hd * (X @ W.T)).sum())  # noqa: E731
    ix = [(int(i), int(j)) for i, j in zip(rng.integers(0, M, 5), rng.integers(0, K, 5))]
    iw = [(int(i), int(j)) for i, j in zip(rng.integers(0, N, 5), rng.integers(0, K, 5))]
    sx = off(hd) @ np.abs(vw) + bounds[1] + 1e-9
    # (dw = sum_m dy x: both factors are rounded along the tokens, x along its own rows in the product that is differentiated)
    sw = (off(hd.T) @ (np.abs(hx) + off(hx.T).T) + np.abs(hd.T) @ (off(hx.T).T + off(hx))
          + bounds[2] + 1e-9)
    for i, j in ix:
        e = np.zeros_like(vx)
        e[i, j] = 0.5
        assert abs((f(vx + e, vw) - f(vx - e, vw)) - float(x.grad[i, j])) <= sx[i, j]
    for i, j in iw:
        e = np.zeros_like(vw)
        e[i, j] = 0.5
        assert abs((f(vx, vw + e) - f(vx, vw - e)) - float(w.grad[i, j])) <= sw[i, j]


def test_linear_frozen_shapes_and_shared_inputs(G):
    note("fp8 linear frozen")
    torch.manual_seed(1)
    x = torch.randn((3, 7, 200), device=DEV, dtype=torch.bfloat16, requires_grad=True)
    w = torch.randn((150, 200), device=DEV, dtype=torch.bfloat16, requires_grad=True)
    dy = torch.randn((3, 7, 150), device=DEV, dtype=torch.bfloat16)
    y = G.gvr_fp8_linear(x, w)
    gx, gw = torch.autograd.grad(y, (x, w), dy)
    assert y.shape == (3, 7, 150) and gx.shape == x.shape and gw.shape == w.shape
    q, qt = G.gvr_fp8_quantize_matrix(w.detach(), square=True, transposed=True)
    z = G.gvr_fp8_linear(x, q, qt)
    assert torch.equal(z, y)
    assert torch.equal(torch.autograd.grad(z, x, dy)[0], gx)
    # the weight alone; a broadcast gradient; one layer used twice
    assert torch.equal(torch.autograd.grad(G.gvr_fp8_linear(x.detach(), w), w, dy)[0], gw)
    one = torch.autograd.grad(G.gvr_fp8_linear(x, w).sum(), (x, w))
    ones = torch.autograd.grad(G.gvr_fp8_linear(x, w), (x, w), torch.ones_like(dy))
    assert all(torch.equal(a, b) for a, b in zip(one, ones))
    twice = torch.autograd.grad(G.gvr_fp8_linear(x, w) + G.gvr_fp8_linear(x, w), (x, w), dy)
    assert torch.equal(twice[0], gx + gx) and torch.equal(twice[1], gw + gw)
    # transposed and expanded inputs
    xt = torch.randn((200, 21), device=DEV).T
    assert torch.equal(G.gvr_fp8_linear(xt, w.detach().T.contiguous().T), G.gvr_fp8_linear(xt.contiguous(), w.detach()))
    with torch.no_grad():
        assert torch.equal(G.gvr_fp8_linear(x, q), y)
    with pytest.raises(ValueError):
        G.gvr_fp8_linear(x, q)
    g = torch.autograd.grad(G.gvr_fp8_linear(x, w), x, dy, create_graph=True)[0]
    with pytest.raises(RuntimeError):
        g.sum().backward()
    with torch.no_grad():
        w.mul_(2)
    assert G.gvr_fp8_linear(x[:0], w).shape == (0, 7, 150)
    gx0, gw0 = torch.autograd.grad(G.gvr_fp8_linear(x[:0], w).sum(), (x, w))
    assert (gx0 == 0).all() and (gw0 == 0).all()


def test_a_sum_over_many_tokens_is_held_in_32_bits(G):
    """All-ones codes over 200000 columns: bfloat16 or float16 partial sums would stop growing."""
    note("fp8 long sum")
    K = 200000
    a = torch.full((2, K), 0x38, dtype=torch.uint8, device=DEV)
    s = torch.ones((2, (K + 127) // 128), device=DEV)
    out = G.gvr_fp8_matmul(a, s, a, s, dtype=torch.float32)
    assert (out == K).all()   # (whole numbers below 2^24: exact in any order)
    assert UNIT["f32"] < 1


@pytest.mark.parametrize("M,N,K,per", [(1, 300, 1001, 128), (20, 1, 1001, 1), (70, 257, 401, 128), (300, 520, 1153, 1)])
def test_rows_that_are_not_aligned(G, M, N, K, per):
    """Packed and shifted rows of either matrix, copied in a workspace or multiplied where they are; a matrix of one row
    has no row stride; what lies beside rows is not read into results (it is NaN)."""
    note("fp8 unaligned %d %d %d" % (M, N, K))
    rng = np.random.default_rng(M + K)
    b, sb, cb, hb = matrix(rng, N, K, per, pad=-K % 16)
    a, sa, ca, ha = matrix(rng, M, K, pad=-K % 16)

    def shifted(c, by, stride):
        store = torch.full((c.shape[0] * stride + by + 64,), 0x7F, dtype=torch.uint8, device=DEV)
        v = store[by:].as_strided(c.shape, (stride, 1))
        return v.copy_(c)
    for dtype in ("bf16", "f32"):
        ref, mag = O.product(ca, ha, cb, hb, per)
        bound = product_bound(mag, ref, K, dtype, cut_off(O.values(ca, ha), O.values(cb, hb, per)))
        aligned = G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype])
        close(aligned, ref, bound)
        for a2, b2 in ((shifted(a, 0, K), b), (a, shifted(b, 0, K)), (shifted(a, 3, K + 1), shifted(b, 1, K + 22)),
                       (shifted(a, 8, K + 7), shifted(b, 16, K))):
            n = G.gvr_fp8_matmul_workspace(a2, sa, b2, sb)
            for size in (0, n // 2, n):   # (the last as much as it asks for)
                ws = torch.full((size,), 0x7F, dtype=torch.uint8, device=DEV)
                out = G.gvr_fp8_matmul(a2, sa, b2, sb, dtype=TORCH[dtype], workspace=ws)
                close(out, ref, bound)
            assert torch.equal(out, G.gvr_fp8_matmul(a2, sa, b2, sb, dtype=TORCH[dtype]))


def test_linear_keeps_nothing_without_gradients(G):
    note("fp8 linear no grad")
    torch.manual_seed(2)
    x = torch.randn((130, 300), device=DEV, requires_grad=True)
    w = torch.randn((70, 300), device=DEV, requires_grad=True)
    y = G.gvr_fp8_linear(x, w)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            z = G.gvr_fp8_linear(x, w)
        assert not z.requires_grad and torch.equal(z, y.detach())
    with pytest.raises(ValueError):
        G.gvr_fp8_linear(x[:, :0], w[:, :0])


@pytest.mark.parametrize("K", [100, 128, 200, 256, 300, 384, 500, 640, 1153])
def test_many_large_tiles(G, K):
    """More tiles of 256 x 256 than compute units, with every number of steps at a tile's begin and end; a NaN row and a NaN
    column stay in theirs; results in aligned and in other rows are the same."""
    note("fp8 many tiles %d" % K)
    M, N = 8100, 8192
    rng = np.random.default_rng(K)
    a, sa, ca, ha = matrix(rng, M, K, pad=-K % 16)
    b, sb, cb, hb = matrix(rng, N, K, 128, pad=-K % 16)
    a[4000, K - 1] = 0x7F
    b[7000, 0] = 0xFF
    dtype = ["bf16", "f16"][K % 8 // 4]
    out = G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype])
    nan = torch.isnan(out)
    assert nan[4000].all() and nan[:, 7000].all() and int(nan.sum()) == M + N - 1
    rows = np.unique(np.concatenate([rng.integers(0, M, 100), [0, 255, 256, 8063, 8064, 8099]]))
    rows = rows[rows != 4000]
    keep = np.delete(np.arange(N), 7000)
    ref, mag = O.product(ca[rows], ha[rows], cb, hb, 128)
    cut = cut_off(O.values(ca[rows], ha[rows]), O.values(cb, hb, 128))
    got = out[torch.from_numpy(rows).to(DEV)][:, torch.from_numpy(keep).to(DEV)]
    close(got, ref[:, keep], product_bound(mag, ref, K, dtype, cut)[:, keep])
    store = torch.full((M, N + 3), 7.0, dtype=TORCH[dtype], device=DEV)
    G.gvr_fp8_matmul(a, sa, b, sb, out=store[:, 1:N + 1])
    assert torch.equal(store[:, 1:N + 1].nan_to_num(3.0), out.nan_to_num(3.0))
    assert (store[:, 0] == 7).all() and (store[:, N + 1:] == 7).all()
    assert torch.equal(G.gvr_fp8_matmul(a, sa, b, sb, dtype=TORCH[dtype]).nan_to_num(3.0), out.nan_to_num(3.0))
