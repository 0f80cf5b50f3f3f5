"""The 4-bit cache on the GPU: appending, reading back, and attention over it
against the oracle (records bit for bit; attention within a bound derived
from its roundings)."""
import numpy as np
import pytest
import torch

from oracle import kv4 as O
from tests.gpu_cases import note
from tests.kv4_cases import DEV, TORCH, Sequences, check_attention, f64, random_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    return g


# ---- tokens in and out

def append_case(G, rng, T, H, D, dtype, rot, inter, page, skip, make=None):
    tab = O.rope_table(300, rot, 1.2).astype(np.float32) if rot else None
    x = [torch.from_numpy(rng.standard_normal((T, H, D)) * (1 + 30 * rng.random((T, H, 1)))).to(TORCH[dtype]) for _ in range(2)]
    if make:
        make(x)
    pages = (T + page - 1) // page + 3
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    slots[rng.random(T) < skip] = -1
    pos = rng.integers(0, 300, T).astype(np.int32)
    cache = torch.full((pages, page, G.gvr_kv4_record_bytes(H, D)), 77, dtype=torch.uint8, device=DEV)
    k, v = (t.to(DEV) for t in x)
    kw = dict(table=torch.from_numpy(tab).to(DEV), positions=torch.from_numpy(pos).to(DEV), interleaved=inter) if rot else {}
    assert G.gvr_kv4_append(k, v, torch.from_numpy(slots).to(DEV), cache, **kw) is cache
    k32 = x[0].float().numpy()
    if rot:
        k32 = O.rotate(k32, pos, tab, inter)
    want = np.full((pages * page, cache.shape[2]), 77, np.uint8)
    want[slots[slots >= 0]] = O.record(k32, x[1].float().numpy())[slots >= 0]
    got = cache.cpu().numpy().reshape(want.shape)
    return got, want, cache, slots


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D,rot,inter", [(64, 64, False), (64, 24, False), (64, 24, True), (128, 0, False), (128, 128, True),
                                         (128, 64, False), (256, 72, True), (256, 6, True), (128, 2, False)])
def test_append(G, dtype, D, rot, inter):
    for T, H, page, skip in ((1, 1, 1, 0.0), (5, 3, 16, 0.3), (130, 8, 64, 0.1)):
        note("append %s D=%d rot=%d inter=%s T=%d H=%d" % (dtype, D, rot, inter, T, H))
        got, want, cache, slots = append_case(G, np.random.default_rng(T + D), T, H, D, dtype, rot, inter, page, skip)
        assert np.array_equal(got, want)
        for out in ("bf16", "f32"):
            k, v = G.gvr_kv4_read(cache, torch.from_numpy(slots).to(DEV), H, D, dtype=TORCH[out])
            keep = slots >= 0
            ek, ev = O.values(want[np.where(keep, slots, 0)], H, D)
            assert np.array_equal(f64(k), np.where(keep[:, None, None], ek, 0.0))
            assert np.array_equal(f64(v), np.where(keep[:, None, None], ev, 0.0))


def test_append_many(G):
    """Several heads to a thread, a head count that does not divide."""
    for T, H in ((4096, 33), (3000, 50)):
        note("append T=%d H=%d" % (T, H))
        got, want, _, _ = append_case(G, np.random.default_rng(T), T, H, 64, "bf16", 32, False, 128, 0.05)
        assert np.array_equal(got, want)


def test_append_special_values(G):
    def make(x):
        k, v = x
        k[0, 0, :] = 0.0                     # a block of zeros
        k[1, 0, 5] = float("inf")            # NaN blocks
        k[1, 1, 40] = float("nan")
        v[2, 0, 0] = -float("inf")
        v[3, :, :] = 1e-40                   # below the smallest scale
        k[4, 0, :32] = torch.tensor([7.0, 3.5, 2.5, 5.0] * 8)          # ties
        k[4, 1, :32] = torch.tensor([7.0000005, 3.4999998] * 16)       # a unit beside them
        v[5, 0, :] = 3e38                    # the largest scales
        v[5, 1, 0] = 3.4028234e38
        v[6, :, ::2] = -0.0
    got, want, cache, slots = append_case(G, np.random.default_rng(0), 9, 2, 64, "f32", 0, False, 16, 0.0, make)
    nan = np.zeros(want.shape, bool)         # codes under a NaN scale stand for nothing
    for t in range(9):
        s = slots[t]
        for i in range(8):
            if want[s, 128 + i] == 255:
                nan[s, i * 16:(i + 1) * 16] = True
    assert np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want))
    k, v = G.gvr_kv4_read(cache, torch.from_numpy(slots).to(DEV), 2, 64, dtype=torch.float32)
    assert torch.isnan(k[1, 0, :32]).all() and torch.isfinite(k[1, 0, 32:]).all() and torch.isnan(k[1, 1, 32:]).all()
    assert torch.isnan(v[2, 0, :32]).all()
    # 3e38 and the largest float32 are nearer to 4 * 2^126 = 2^128 than to 3 * 2^126, and read as infinity
    ek, ev = O.values(want[slots], 2, 64)
    with np.errstate(over="ignore"):
        for got, ref in ((k, ek), (v, ev)):
            assert np.array_equal(got.cpu().numpy(), ref.astype(np.float32), equal_nan=True)


def test_append_strides_and_places(G):
    """A fused projection, unaligned heads; slots outside the cache and out-of-table positions."""
    rng = np.random.default_rng(4)
    T, H, D = 33, 2, 64
    wide = torch.from_numpy(rng.standard_normal((T, 8, D + 8))).bfloat16().to(DEV)
    tab = torch.from_numpy(O.rope_table(50, 64).astype(np.float32)).to(DEV)
    pos = torch.from_numpy(rng.integers(0, 50, T).astype(np.int32)).to(DEV)
    slots = torch.from_numpy(rng.permutation(64)[:T].astype(np.int64)).to(DEV)
    for off in (0, 8, 3):
        note("append strided at %d" % off)
        k, v = wide[:, 1:3, off:off + D] if off < 8 else wide[:, 1:3, 8:8 + D], wide[:, 5:7, off % 8:off % 8 + D]
        a = G.gvr_kv4_append(k, v, slots, G.new_kv4_cache(4, 16, H, D), tab, pos)
        b = G.gvr_kv4_append(k.contiguous(), v.contiguous(), slots, G.new_kv4_cache(4, 16, H, D), tab, pos)
        assert torch.equal(a, b)
    far = slots.clone()
    far[3], far[4], far[5] = 64, -2, 2 ** 40
    pos2 = pos.clone()
    pos2[7], pos2[8] = 50, -1
    c = G.gvr_kv4_append(k.contiguous(), v.contiguous(), far, G.new_kv4_cache(4, 16, H, D), tab, pos2)
    rk, rv = G.gvr_kv4_read(c, far, H, D)
    assert not rk[3:6].any() and not rv[3:6].any()
    assert torch.isnan(rk[7:9]).all() and torch.isfinite(rv).all()
    rk2, rv2 = G.gvr_kv4_read(b, slots, H, D)
    rest = [t for t in range(T) if t not in (3, 4, 5, 7, 8)]
    assert torch.equal(rk[rest], rk2[rest]) and torch.equal(rv[rest], rv2[rest])


def test_read_float16_and_strides(G):
    rng = np.random.default_rng(6)
    cache = torch.from_numpy(random_cache(rng, 3, 16, 3, 64)).to(DEV)
    slots = torch.from_numpy(rng.integers(0, 48, 40)).to(DEV)
    k, v = G.gvr_kv4_read(cache, slots, 3, 64, dtype=torch.float16)
    ek, ev = O.values(cache.cpu().numpy().reshape(48, -1)[slots.cpu().numpy()], 3, 64)
    assert np.array_equal(f64(k), ek) and np.array_equal(f64(v), ev)      # these scales are exact in float16
    wide = torch.zeros((40, 7, 70), dtype=torch.float16, device=DEV)
    G.gvr_kv4_read(cache, slots, 3, 64, dtype=torch.float16, k=wide[:, :3, 1:65], v=wide[:, 4:7, 2:66])
    assert torch.equal(wide[:, :3, 1:65], k) and torch.equal(wide[:, 4:7, 2:66], v)
    assert not wide[:, 3].any() and not wide[:, :3, 65:].any() and not wide[:, :, 0].any()


# ---- attention

def attention_case(G, rng, ctx, nq, heads=2, group=4, D=64, page=16, dtype="bf16", causal=True, K=0, ws=None, amp=1.0,
                   seqs=None, selection=None, lse=True, **kw):
    """nq: query tokens of each sequence (an int: the same number for all)."""
    uniform = isinstance(nq, int)
    nqs = [nq] * len(ctx) if uniform else list(nq)
    starts = np.concatenate([[0], np.cumsum(nqs)]).astype(np.int32)
    seqs = seqs or Sequences(rng, ctx, page, heads, D)
    T, H = int(starts[-1]), heads * group
    q = (amp * torch.from_numpy(rng.standard_normal((T, H, D)))).to(TORCH[dtype]).to(DEV)
    cache, table, lens = seqs.on_gpu()
    if K:
        selection = np.full((T, K), -1, np.int32)
        for b, c in enumerate(ctx):
            for i in range(nqs[b]):
                see = max(0, c - nqs[b] + 1 + i)
                pick = np.sort(rng.permutation(see)[:K])
                selection[starts[b] + i, :len(pick)] = pick
    sel = None if selection is None else torch.from_numpy(selection).to(DEV)
    scale = kw.pop("scale", D ** -0.5)
    lse = torch.full((T, H), 5.0, device=DEV) if lse else None
    args = dict(selection=sel, causal=causal, q_start=None if uniform else torch.from_numpy(starts).to(DEV),
                max_q=None if uniform else max(nqs))
    need = G.gvr_kv4_attention_workspace(q, cache, table, lens, heads, **args)
    what = "attention ctx=%s nq=%s heads=%d x %d D=%d page=%d %s causal=%s K=%d ws=%s/%d" % (
        ctx, nq, heads, group, D, page, dtype, causal, K, ws, need)
    note(what)
    if ws == "none":
        args["workspace"] = torch.empty(0, dtype=torch.uint8, device=DEV)
    elif ws is not None:
        args["workspace"] = torch.full((max(16, int(need * ws)),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full((T, H, D), 7.0, dtype=TORCH[dtype], device=DEV)
    got = G.gvr_kv4_attention(q, cache, table, lens, heads, scale=scale, out=out, lse=lse, **args, **kw)
    torch.cuda.synchronize()
    assert got is out
    check_attention(out, lse, q, seqs, starts, scale, causal, selection, dtype, what)
    return out, q, seqs


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (3, 5), (8, 8), (1, 16), (2, 17), (1, 128)])
def test_decode_head_layouts(G, dtype, D, heads, group):
    rng = np.random.default_rng(D + heads * 31 + group)
    attention_case(G, rng, [200, 1, 33, 0, 97], 1, heads, group, D, dtype=dtype)


@pytest.mark.parametrize("page", [1, 2, 16, 64, 256])
def test_decode_lengths(G, page):
    """Lengths around the steps, the tiles and the ends of pages."""
    rng = np.random.default_rng(page)
    attention_case(G, rng, [0, 1, 2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513], 1, page=page)
    attention_case(G, rng, [31, 32, 33, 64, 96, 100], 1, heads=1, group=2, D=128, page=page)


@pytest.mark.parametrize("nq", [2, 3, 5, 8, 17])
def test_draft_rows(G, nq):
    """Several query tokens of a sequence, some before its first token."""
    rng = np.random.default_rng(nq)
    attention_case(G, rng, [0, 1, nq - 1, nq, nq + 1, 40, 70, 129], nq, heads=2, group=3, D=64)
    attention_case(G, rng, [1, 40, 70, 129], nq, heads=1, group=8, D=128, causal=False)


@pytest.mark.parametrize("ws", ["none", 0.3, 0.6, 1.0, 2.0, None])
@pytest.mark.parametrize("D,heads,group,nq", [(64, 1, 4, 1), (128, 2, 8, 3), (256, 1, 2, 1), (128, 1, 16, 20)])
def test_splits(G, ws, D, heads, group, nq):
    """Every workspace size gives a right answer; a dirty workspace does not show."""
    rng = np.random.default_rng(D + nq)
    attention_case(G, rng, [3000, 700, 0, 2999, 5], nq, heads, group, D, page=64, ws=ws)


def test_one_long_context(G):
    rng = np.random.default_rng(1)
    attention_case(G, rng, [40001], 1, heads=1, group=8, D=64, page=128, amp=3.0)
    attention_case(G, rng, [20011], 2, heads=2, group=4, D=128, page=16, dtype="f16")


@pytest.mark.parametrize("D,heads,group", [(64, 2, 4), (128, 8, 8), (128, 1, 40), (256, 3, 1), (64, 4, 2)])
@pytest.mark.parametrize("K", [1, 31, 64, 300])
def test_selection(G, D, heads, group, K):
    rng = np.random.default_rng(K + D)
    attention_case(G, rng, [1000, 0, 17, 400, 64], 2, heads, group, D, K=K)
    attention_case(G, rng, [1000, 5, 330], 1, heads, group, D, K=K, ws="none", dtype="f16")


def test_selection_entries(G):
    """Empty lists, entries out of order, twice, below zero, past the end and past the causal limit."""
    rng = np.random.default_rng(12)
    ctx, nq, K = [300, 64, 9], 3, 50
    sel = rng.integers(-5, 320, (9, K)).astype(np.int32)
    sel[0] = -1
    sel[4] = 2 ** 31 - 1
    sel[5] = 7
    sel[6, :] = -2 ** 31
    for causal in (True, False):
        attention_case(G, rng, ctx, nq, 2, 4, 128, selection=sel, causal=causal)


def test_selection_of_everything_is_the_whole(G):
    rng = np.random.default_rng(13)
    seqs = Sequences(rng, [600, 600], 64, 2, 128)
    cache, table, lens = seqs.on_gpu()
    q = torch.randn((2, 8, 128), device=DEV).bfloat16()
    sel = torch.arange(600, dtype=torch.int32, device=DEV).repeat(2, 1)
    a = f64(G.gvr_kv4_attention(q, cache, table, lens, 2, selection=sel))
    b = f64(G.gvr_kv4_attention(q, cache, table, lens, 2))
    assert np.abs(a - b).max() <= 2.0 ** -6 * np.abs(b).max()


def test_selection_through_topk(G):
    """The Top-K's out_idx goes in as it is: short rows (-1 padding) and long ones."""
    rng = np.random.default_rng(14)
    ctx = [5000, 1000, 2049]
    scores = torch.from_numpy(rng.standard_normal((3, 5000)).astype(np.float32)).to(DEV)
    sel = G.gvr_topk(scores, torch.tensor(ctx, dtype=torch.int32, device=DEV), None, 2048)
    attention_case(G, rng, ctx, 1, 2, 4, 64, page=64, selection=sel.cpu().numpy())


@pytest.mark.parametrize("D,heads,group", [(64, 2, 4), (128, 1, 8), (256, 2, 2), (128, 2, 1), (128, 1, 5)])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts(G, D, heads, group, causal):
    """Chunks of hundreds of queries: a whole prompt, a chunk behind a context, odd numbers."""
    rng = np.random.default_rng(D + group)
    attention_case(G, rng, [257, 300], 257, heads, group, D, causal=causal)
    attention_case(G, rng, [700], 130, heads, group, D, page=64, causal=causal, dtype="f16")


def test_ragged_prompts(G):
    rng = np.random.default_rng(21)
    attention_case(G, rng, [300, 0, 140, 90, 1, 513], [300, 0, 33, 1, 1, 100], 2, 4, 64)
    attention_case(G, rng, [300, 7, 140, 90], [64, 0, 140, 129], 1, 8, 128, causal=False)


def test_rows_outside_the_sequences_and_beyond_max_q(G):
    rng = np.random.default_rng(22)
    seqs = Sequences(rng, [50, 60], 16, 1, 64)
    cache, table, lens = seqs.on_gpu()
    q = torch.randn((12, 4, 64), device=DEV).bfloat16()
    start = torch.tensor([2, 5, 10], dtype=torch.int32, device=DEV)
    for ws in (None, torch.empty(0, dtype=torch.uint8, device=DEV)):
        full = G.gvr_kv4_attention(q, cache, table, lens, 1, q_start=start, out=torch.full_like(q, 3.0), workspace=ws)
        part = G.gvr_kv4_attention(q, cache, table, lens, 1, q_start=start, max_q=3, out=torch.full_like(q, 3.0),
                                   workspace=ws)
        assert (full[:2] == 3).all() and (full[10:] == 3).all() and (part[8:] == 3).all()
        assert torch.equal(part[2:8], full[2:8])
        # starts that leave the queries: nothing is read or written outside
        wild = torch.tensor([-4, 20, 11], dtype=torch.int32, device=DEV)
        out = G.gvr_kv4_attention(q, cache, table, lens, 1, q_start=wild, out=torch.full_like(q, 3.0), workspace=ws)
        assert (out == 3).all()


def test_strided_queries(G):
    rng = np.random.default_rng(23)
    seqs = Sequences(rng, [100, 37], 16, 2, 64)
    cache, table, lens = seqs.on_gpu()
    wide = torch.randn((6, 12, 96), device=DEV).bfloat16()
    for q in (wide[:, 2:10, 8:72], wide[:, :8, :64].transpose(0, 1).contiguous().transpose(0, 1)):
        a = G.gvr_kv4_attention(q, cache, table, lens, 2)
        assert torch.equal(a, G.gvr_kv4_attention(q.contiguous(), cache, table, lens, 2))


def test_masked_nan_blocks_do_not_show(G):
    """NaN records behind the causal limit, in unselected tokens, and in pages that are not there."""
    rng = np.random.default_rng(24)
    for group, nq in ((2, 4), (5, 7), (16, 3), (4, 40)):
        seqs = Sequences(rng, [90], 16, 1, 64)
        flat = seqs.cache.reshape(-1, seqs.cache.shape[-1])
        first = 90 - nq + nq // 2 + 1     # tokens that only the later queries see
        dirty = seqs.slots(0, np.arange(first, 90))
        q = torch.from_numpy(rng.standard_normal((nq, group, 64))).bfloat16().to(DEV)
        flat[dirty, 64 + 2:] = 255        # the values' scales
        cache, table, lens = seqs.on_gpu()
        for ws in (None, torch.empty(0, dtype=torch.uint8, device=DEV)):
            out = G.gvr_kv4_attention(q, cache, table, lens, 1, workspace=ws)
            note("masked NaN values: group %d nq %d" % (group, nq))
            assert torch.isfinite(out[:nq // 2 + 1]).all() and torch.isnan(out[nq // 2 + 1:]).all()
        flat[dirty, 64:66] = 255          # and the keys'
        cache, table, lens = seqs.on_gpu()
        out2 = G.gvr_kv4_attention(q, cache, table, lens, 1)
        assert torch.equal(out2[:nq // 2 + 1], G.gvr_kv4_attention(q, cache, table, lens, 1, workspace=ws)[:nq // 2 + 1]) or \
            torch.allclose(out2[:nq // 2 + 1].float(), out[:nq // 2 + 1].float(), atol=2e-2)
        assert torch.isfinite(out2[:nq // 2 + 1]).all() and torch.isnan(out2[nq // 2 + 1:]).all()
        sel = torch.full((nq, 20), -1, dtype=torch.int32, device=DEV)
        sel[:, :10] = torch.arange(10, device=DEV)
        assert torch.isfinite(G.gvr_kv4_attention(q, cache, table, lens, 1, selection=sel)).all()


def test_pages_that_are_not_there(G):
    rng = np.random.default_rng(25)
    seqs = Sequences(rng, [128], 16, 2, 64)
    q = torch.from_numpy(rng.standard_normal((1, 8, 64))).bfloat16().to(DEV)
    cache, table, lens = seqs.on_gpu()
    bad = table.clone()
    bad[0, 2], bad[0, 5] = -1, cache.shape[0]
    got = f64(G.gvr_kv4_attention(q, cache, bad, lens, 2))
    t = np.array([i for i in range(128) if i // 16 not in (2, 5)])
    k, v = seqs.kv(0, t)
    ref, _, mag = O.attention(f64(q)[0], k, v, 64 ** -0.5)
    assert (np.abs(got[0] - ref) <= 2.0 ** -8 * 1.1 * mag + 2.0 ** -8 * np.abs(ref)).all()
    bad[:] = -1
    assert not G.gvr_kv4_attention(q, cache, bad, lens, 2).any()
    # a context longer than the table is cut to it, a negative one is empty
    long = torch.full_like(lens, 10 ** 9)
    full = torch.where(table < 0, torch.zeros_like(table), table)[:, :8].contiguous()
    assert torch.equal(G.gvr_kv4_attention(q, cache, full, long, 2), G.gvr_kv4_attention(q, cache, full, lens, 2))
    assert not G.gvr_kv4_attention(q, cache, full, -lens, 2).any()
    none = torch.empty((0, 16, cache.shape[2]), dtype=torch.uint8, device=DEV)
    assert not G.gvr_kv4_attention(q, none, full, lens, 2).any()


def test_large_scores(G):
    """Scores that grow along the context by far more than the exponential's range."""
    rng = np.random.default_rng(26)
    for amp, scale in ((40.0, 1.0), (1.0, -3.0), (1.0, 0.0)):
        attention_case(G, rng, [500, 90], 2, 2, 4, 64, amp=amp, scale=scale)


def test_offsets_past_32_bits(G):
    """A cache of more than 4 GiB, read and written at its end."""
    pages, page, H, D = 62000, 64, 8, 128
    rec = G.gvr_kv4_record_bytes(H, D)
    assert pages * page * rec > 2 ** 32
    rng = np.random.default_rng(27)
    cache = torch.empty((pages, page, rec), dtype=torch.uint8, device=DEV)
    used = [pages - 1, 0, pages - 2, 61000]
    small = random_cache(rng, 4, page, H, D)
    for i, pg in enumerate(used):
        cache[pg] = torch.from_numpy(small[i]).to(DEV)
    table = torch.tensor([used], dtype=torch.int32, device=DEV)
    local = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device=DEV)
    lens = torch.tensor([250], dtype=torch.int32, device=DEV)
    q = torch.randn((1, 16, D), device=DEV).bfloat16()
    sc = torch.from_numpy(small).to(DEV)
    note("attention at the end of a 4.3 GB cache")
    assert torch.equal(G.gvr_kv4_attention(q, cache, table, lens, H), G.gvr_kv4_attention(q, sc, local, lens, H))
    sel = torch.tensor([[249, 3, 70, 140, -1]], dtype=torch.int32, device=DEV)
    assert torch.equal(G.gvr_kv4_attention(q, cache, table, lens, H, selection=sel),
                       G.gvr_kv4_attention(q, sc, local, lens, H, selection=sel))
    qq = torch.randn((200, 16, D), device=DEV).bfloat16()
    assert torch.equal(G.gvr_kv4_attention(qq, cache, table, lens, H), G.gvr_kv4_attention(qq, sc, local, lens, H))
    k = torch.randn((2, H, D), device=DEV).bfloat16()
    slots = torch.tensor([pages * page - 1, 61000 * page + 5], device=DEV)
    G.gvr_kv4_append(k, k, slots, cache)
    rk, rv = G.gvr_kv4_read(cache, slots, H, D)
    want = O.values(O.record(f64(k), f64(k)), H, D)
    assert np.array_equal(f64(rk), want[0]) and np.array_equal(f64(rv), want[1])


def test_same_bits_every_time_other_stream_and_graph(G):
    rng = np.random.default_rng(28)
    seqs = Sequences(rng, [3000, 1234], 64, 2, 128)
    cache, table, lens = seqs.on_gpu()
    q = torch.randn((2, 8, 128), device=DEV).bfloat16()
    want = G.gvr_kv4_attention(q, cache, table, lens, 2).clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call = G.prepare_gvr_kv4_attention(q, cache, table, lens, 2, stream=s)
    for _ in range(3):
        call()
        s.synchronize()
        assert torch.equal(call.out, want)
    k = torch.randn((2, 2, 128), device=DEV).bfloat16()
    v = torch.randn((2, 2, 128), device=DEV).bfloat16()
    slots = torch.tensor([seqs.slots(0, [2999])[0], seqs.slots(1, [1233])[0]], device=DEV)
    app = G.prepare_gvr_kv4_append(k, v, slots, cache, stream=s)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        app()
        call()
    for i in range(4):
        k.normal_()
        v.normal_()
        q.normal_()
        lens[0] = 3000 - 500 * (i % 2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = call.out.clone()
        G.gvr_kv4_append(k, v, slots, cache)
        assert torch.equal(got, G.gvr_kv4_attention(q, cache, table, lens, 2)), "replay %d" % i
        (got.float() @ torch.ones(128, 1, device=DEV)).sum().item()


def test_nothing_to_do(G):
    cache = G.new_kv4_cache(2, 16, 1, 64)
    e = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    t0 = torch.empty((0, 3), dtype=torch.int32, device=DEV)
    l0 = torch.empty(0, dtype=torch.int32, device=DEV)
    assert G.gvr_kv4_attention(e, cache, t0, l0, 1).shape == e.shape
    assert G.gvr_kv4_attention(e, cache, torch.zeros((2, 3), dtype=torch.int32, device=DEV),
                               torch.ones(2, dtype=torch.int32, device=DEV), 1).shape == e.shape
    q = torch.randn((2, 4, 64), device=DEV).bfloat16()
    no_pages = torch.empty((2, 0), dtype=torch.int32, device=DEV)
    assert not G.gvr_kv4_attention(q, cache, no_pages, torch.ones(2, dtype=torch.int32, device=DEV), 1).any()
    k = torch.empty((0, 1, 64), device=DEV)
    s = torch.empty(0, dtype=torch.int64, device=DEV)
    assert not G.gvr_kv4_append(k, k, s, cache).any()
    assert G.gvr_kv4_read(cache, s, 1, 64)[0].shape == (0, 1, 64)


def test_refusals(G):
    cache = G.new_kv4_cache(4, 16, 2, 64)
    q = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device=DEV)
    tab, lens = torch.zeros((2, 2), dtype=torch.int32, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV)
    ok = dict(q=q, cache=cache, block_table=tab, ctx_len=lens, kv_heads=2)
    G.gvr_kv4_attention(**ok)
    flat = torch.zeros(8 * 64 * 2 + 16, dtype=torch.bfloat16, device=DEV)
    for kw in (dict(q=q.float()), dict(q=q.double()), dict(q=q[0]), dict(q=q.cpu()), dict(q=q[:, :7]), dict(q=q[:, :, :32]),
               dict(q=flat[1:1025].view(2, 8, 64)), dict(cache=cache[:, :, :135].contiguous()), dict(cache=cache.int()),
               dict(cache=cache[:, ::2]), dict(cache=cache[:, :12].contiguous()), dict(block_table=tab.long()),
               dict(block_table=tab[0]), dict(ctx_len=lens[:1]), dict(ctx_len=lens.long()), dict(kv_heads=3),
               dict(selection=torch.zeros((2, 0), dtype=torch.int32, device=DEV)),
               dict(selection=torch.zeros((3, 4), dtype=torch.int32, device=DEV)),
               dict(selection=torch.zeros((2, 4), dtype=torch.int64, device=DEV)),
               dict(q_start=torch.zeros(2, dtype=torch.int32, device=DEV)),
               dict(q_start=torch.zeros(3, dtype=torch.int32, device=DEV), max_q=-1),
               dict(block_table=tab[:1].repeat(3, 1), ctx_len=torch.ones(3, dtype=torch.int32, device=DEV)),
               dict(scale=float("inf")), dict(out=q.half()), dict(out=q[:1]), dict(lse=torch.zeros((2, 4), device=DEV)),
               dict(workspace=torch.zeros(64, dtype=torch.uint8, device=DEV)[8:])):
        with pytest.raises(ValueError):
            G.gvr_kv4_attention(**{**ok, **kw})
    k, s = torch.zeros((3, 2, 64), device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    t = torch.zeros((9, 32, 2), device=DEV)
    p = torch.zeros(3, dtype=torch.int32, device=DEV)
    ok = dict(k=k, v=k, slots=s - 1, cache=cache)
    G.gvr_kv4_append(**ok)
    for kw in (dict(k=k.double()), dict(v=k.half()), dict(v=k[:2]), dict(slots=s.int()), dict(slots=s[:2]), dict(positions=p),
               dict(table=t), dict(table=t, positions=p.long()), dict(table=torch.zeros((9, 33, 2), device=DEV), positions=p),
               dict(k=k[:, :1], v=k[:, :1]), dict(k=k.cpu(), v=k.cpu()), dict(cache=cache.cpu())):
        with pytest.raises(ValueError):
            G.gvr_kv4_append(**{**ok, **kw})
    for kw in (dict(slots=s.int()), dict(dtype=torch.float64), dict(kv_heads=3), dict(head_dim=96),
               dict(k=torch.zeros((3, 2, 64), device=DEV)), dict(v=k.bfloat16()[:2])):
        with pytest.raises(ValueError):
            G.gvr_kv4_read(**{**dict(cache=cache, slots=s, kv_heads=2, head_dim=64), **kw})


@pytest.mark.parametrize("shape", [dict(ctx=[700, 60, 0, 3000], nq=1, heads=2, group=4, D=128),
                                   dict(ctx=[900, 901, 40], nq=3, heads=2, group=8, D=64, dtype="f16"),
                                   dict(ctx=[640], nq=200, heads=2, group=2, D=128),
                                   dict(ctx=[300, 513], nq=130, heads=1, group=4, D=64),
                                   dict(ctx=[500], nq=70, heads=1, group=4, D=256),
                                   dict(ctx=[2500, 90], nq=2, heads=4, group=24, D=128, K=150)])
def test_the_same_call_gives_the_same_bits(G, shape):
    """Eight calls of each kernel, with other work between them, agree bit for bit."""
    rng = np.random.default_rng(31)
    ctx, nq, heads, D = shape["ctx"], shape["nq"], shape["heads"], shape["D"]
    seqs = Sequences(rng, ctx, 16, heads, D)
    cache, table, lens = seqs.on_gpu()
    q = torch.randn((len(ctx) * nq, heads * shape["group"], D), device=DEV).to(TORCH[shape.get("dtype", "bf16")])
    sel = None
    if shape.get("K"):
        sel = torch.randint(-1, min(c for c in ctx), (len(ctx) * nq, shape["K"]), device=DEV, dtype=torch.int32)
    note("same bits: %s" % shape)
    lse = torch.empty((q.shape[0], q.shape[1]), device=DEV)
    want = G.gvr_kv4_attention(q, cache, table, lens, heads, selection=sel, lse=lse).clone()
    first = lse.clone()
    for i in range(8):
        torch.randn((1 << (14 + i % 5),), device=DEV)
        got = G.gvr_kv4_attention(q, cache, table, lens, heads, selection=sel, lse=lse)
        assert torch.equal(got, want) and torch.equal(lse, first)


@pytest.mark.parametrize("n", [2, 63, 64, 65, 130, 700])
def test_many_sequences_of_uneven_lengths(G, n):
    """Splits that the kernel sizes: one long context among short and empty ones,
    more sequences than lanes of a wave, and lengths that are all alike."""
    rng = np.random.default_rng(n)
    lengths = [2000] + [int(x) for x in rng.integers(0, 60, n - 1)]
    rng.shuffle(lengths)
    attention_case(G, rng, lengths, 1, heads=1, group=2, D=64, page=16)
    if n <= 130:
        attention_case(G, rng, [300] * n, 1, heads=2, group=4, D=64, page=64)
        attention_case(G, rng, lengths, 3, heads=2, group=8, D=64, page=16, dtype="f16", ws=0.7)


def test_one_long_sequence_among_empty_ones(G):
    """The kernel sizes the splits: all but a few would go to the one long context,
    more than the kernel that joins them holds, were their number not bounded."""
    rng = np.random.default_rng(41)
    attention_case(G, rng, [0] * 40 + [600000] + [0] * 22 + [3, 0], 1, heads=1, group=2, D=64, page=64)


@pytest.mark.parametrize("nq", [1, 40])
def test_longest_context(G, nq):
    """2^31 - 16 tokens, all but those of three pages invisible: places past the
    last step must not pass the end of 32 bits."""
    page, H, D, group = 16, 1, 64, 2
    width = 2 ** 27 - 1
    rng = np.random.default_rng(42)
    cache = random_cache(rng, 3, page, H, D)
    table = torch.full((1, width), -1, dtype=torch.int32, device=DEV)
    for i, at in enumerate((5, 70000000, width - 1)):
        table[0, at] = i
    lens = torch.tensor([width * page], dtype=torch.int32, device=DEV)
    q = torch.randn((nq, H * group, D), device=DEV).bfloat16()
    note("attention over 2^31 - 16 tokens, %d query tokens" % nq)
    out = G.gvr_kv4_attention(q, torch.from_numpy(cache).to(DEV), table, lens, H, causal=False)
    s = Sequences.__new__(Sequences)
    s.table, s.cache, s.ctx, s.page, s.heads, s.D = np.array([[0, 1, 2]]), cache, [3 * page], page, H, D
    check_attention(out, None, q, s, [0, nq], D ** -0.5, causal=False, what="longest context")


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_around_the_kernels_change(G, D, dtype):
    """127 to 130 rows of a KV head (few-rows kernel up to 128), NaN records beside the
    visible ones, ragged query counts, and a workspace that allows some splits only."""
    rng = np.random.default_rng(51)
    attention_case(G, rng, [333], 127, heads=2, group=1, D=D, dtype=dtype)
    attention_case(G, rng, [333], 129, heads=1, group=1, D=D, dtype=dtype)
    attention_case(G, rng, [500, 70], 26, heads=1, group=5, D=D, dtype=dtype, ws=0.5)
    attention_case(G, rng, [700, 90, 0, 200], [150, 90, 3, 1], heads=2, group=1, D=D, dtype=dtype, ws=0.6)
    attention_case(G, rng, [400, 90], [40, 7], heads=1, group=3, D=D, dtype=dtype, causal=False, page=64)


def test_one_sequence_many_rows_split(G):
    """Many rows over a long context: splits of the many-rows kernel, joined."""
    rng = np.random.default_rng(52)
    attention_case(G, rng, [9000], 40, heads=1, group=4, D=128, page=64)
    attention_case(G, rng, [9000], 40, heads=1, group=4, D=128, page=64, dtype="f16", causal=False, ws=0.4)
