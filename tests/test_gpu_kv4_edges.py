"""Attention over the 4-bit cache at the edges of its numbers: values that are
not finite, weights that underflow, counts of query tokens that name nothing."""
import numpy as np
import pytest
import torch

from oracle import kv4 as O
from tests.gpu_cases import note
from tests.kv4_cases import DEV, TORCH, UNIT, Sequences, check_attention, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_22312_amd as g
    g.lib()
    return g


def held(k, v, page=16):
    """One sequence of k, v [n][heads][D] in consecutive pages: its cache, block table and lengths on the GPU, and what
    the records stand for."""
    n, heads, D = k.shape
    rec = O.record(k, v)
    pages = (n + page - 1) // page
    cache = np.zeros((pages * page, rec.shape[1]), np.uint8)
    cache[:n] = rec
    return (torch.from_numpy(cache.reshape(pages, page, -1)).to(DEV),
            torch.arange(pages, dtype=torch.int32, device=DEV).view(1, -1),
            torch.tensor([n], dtype=torch.int32, device=DEV), *O.values(rec, heads, D))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("nq", [1, 33])
def test_visible_nan_of_a_part_without_weight(G, dtype, D, nq):
    """A value that is NaN, in a token whose weight underflows (768 below the largest score), is visible all the same:
    its 32 dimensions are NaN, split or not, and the others are not touched."""
    rng = np.random.default_rng(61)
    n, group, block = 4000, 4, 1
    k = np.full((n, 1, D), -6.0)
    k[n - nq - 40:n - nq + 1] = 6.0            # every row's largest scores, 768 and more above the others
    v = rng.standard_normal((n, 1, D))
    v[5, 0, 32 * block] = np.nan
    cache, table, lens, kk, vv = held(k, v)
    q = torch.full((nq, group, D), 8.0, dtype=TORCH[dtype], device=DEV)
    scale = 8.0 / D                            # scores of +-384
    assert G.gvr_kv4_attention_workspace(q, cache, table, lens, 1) > 0
    nan = np.zeros(D, bool)
    nan[32 * block:32 * block + 32] = True
    for ws in (torch.empty(0, dtype=torch.uint8, device=DEV), None):
        note("visible NaN without weight: %s D=%d nq=%d %s" % (dtype, D, nq, "split" if ws is None else "whole"))
        out = f64(G.gvr_kv4_attention(q, cache, table, lens, 1, scale=scale, workspace=ws))
        for i in range(nq):
            ref, _, mag = O.attention(f64(q)[i], kk[:n - nq + 1 + i], np.nan_to_num(vv[:n - nq + 1 + i]), scale)
            assert np.isnan(out[i][:, nan]).all(), "row %d lost the NaN" % i
            # the weights are 0 and 1: sums in float32 and one rounding
            tol = UNIT[dtype] * np.abs(ref) + 2 * (n + 64) * 2.0 ** -24 * mag + 2.0 ** -24
            assert (np.abs(out[i] - ref) <= tol)[:, ~nan].all()


def one_ahead(n, D, value, rng):
    """k, v of n tokens: all scores 0 but those of token 7, whose value is given; the others' values lie in 1 .. 6."""
    k, v = np.zeros((n, 1, D)), rng.uniform(1.0, 6.0, (n, 1, D))
    k[7, 0, 0], v[7] = 6.0, value
    return k, v


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("nq", [1, 70])
@pytest.mark.parametrize("ahead", [16.0, 17.5, 20.0])
def test_float16_keeps_the_tail_behind_a_large_score(G, D, nq, ahead):
    """One token far ahead whose value is zero: the result is the sum of the many small weights, each of which may carry
    one float16 rounding and 2^-40 of the largest."""
    rng = np.random.default_rng(62)
    n = 20001
    cache, table, lens, kk, vv = held(*one_ahead(n, D, 0.0, rng), page=64)
    q = torch.zeros((nq, 2, D), dtype=torch.float16, device=DEV)
    q[:, :, 0] = 1.0
    u, eps = UNIT["f16"], ((D + 8) * ahead + n + 64) * 2.0 ** -24
    for ws in (torch.empty(0, dtype=torch.uint8, device=DEV), None):
        note("float16 tail: D=%d nq=%d ahead=%s %s" % (D, nq, ahead, "split" if ws is None else "whole"))
        lse = torch.empty((nq, 2), device=DEV)
        out = f64(G.gvr_kv4_attention(q, cache, table, lens, 1, scale=ahead / 6.0, causal=False, workspace=ws, lse=lse))
        ref, ref_lse, mag = O.attention(f64(q)[0], kk, vv, ahead / 6.0)
        tol = (u + 2 * eps) * (1 + u) * mag + u * np.abs(ref) + n * 2.0 ** -40 * 6.0 + 2.0 ** -25
        assert (tol < 0.01 * ref).all()
        assert (np.abs(out - ref) <= tol).all(), "off by %.3g of the result" % (np.abs(out - ref) / ref).max()
        assert (np.abs(f64(lse) - ref_lse) <= 2 * eps + 4 * 2.0 ** -24 * (ref_lse + 1)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("nq", [1, 70])
def test_scores_of_hundreds_of_millions(G, dtype, nq):
    """One token takes all the weight, whatever the scores' size (3.6e8: units of 2^5 in float32)."""
    rng = np.random.default_rng(63)
    k, v = one_ahead(900, 64, 3.0, rng)
    k[:, 0, 1] = 6.0
    cache, table, lens, _, vv = held(k, v)
    q = torch.zeros((nq, 2, 64), dtype=TORCH[dtype], device=DEV)
    q[:, :, 0] = q[:, :, 1] = 60000.0
    for ws in (torch.empty(0, dtype=torch.uint8, device=DEV), None):
        note("scores of 3.6e8: %s nq=%d" % (dtype, nq))
        out = G.gvr_kv4_attention(q, cache, table, lens, 1, scale=1000.0, causal=False, workspace=ws)
        assert np.array_equal(f64(out), np.broadcast_to(vv[7], out.shape))


@pytest.mark.parametrize("dtype,huge", [("f16", 60000.0), ("bf16", 3.3e38)])
@pytest.mark.parametrize("D,group,nq", [(64, 2, 4), (64, 5, 7), (128, 16, 3), (128, 4, 40), (256, 3, 2), (256, 2, 70), (64, 1, 140)])
def test_masked_infinities_do_not_show(G, dtype, huge, D, group, nq):
    """Values that the 16-bit type cannot hold (60000 is stored as 4 * 2^14, 3.3e38 as 4 * 2^126), in tokens that only
    the later queries see: the earlier ones are right, and the later ones not finite where they see them."""
    rng = np.random.default_rng(64)
    n, split = 400, nq // 2
    first = n - nq + split                      # seen by the queries from `split` on
    k, v = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
    v[first:, 0, 40] = huge
    cache, table, lens, kk, vv = held(k, v)
    assert (vv[first:, 0, 40] > (65519 if dtype == "f16" else 3.39e38)).all()
    q = torch.from_numpy(rng.standard_normal((nq, group, D))).to(TORCH[dtype]).to(DEV)
    u, scale = UNIT[dtype], D ** -0.5
    for ws in (torch.empty(0, dtype=torch.uint8, device=DEV), None):
        note("masked infinities: %s D=%d group %d nq %d %s" % (dtype, D, group, nq, "split" if ws is None else "whole"))
        out = f64(G.gvr_kv4_attention(q, cache, table, lens, 1, workspace=ws))
        for i in range(nq):
            t = n - nq + i + 1
            ref, _, mag = O.attention(f64(q)[i], kk[:t], vv[:t], scale)
            if i < split:
                qk = (np.abs(kk[:t, 0]) @ np.abs(f64(q)[i]).T).max()
                eps = ((D + 8) * scale * qk + t + 64) * 2.0 ** -24
                tol = (u + 2 * eps) * (1 + u) * mag + u * np.abs(ref) + t * 2.0 ** -40 * np.abs(vv[:t]).max() + 2.0 ** -25
                assert (np.abs(out[i] - ref) <= tol).all(), "row %d shows a masked value" % i
            else:
                assert not np.isfinite(out[i][:, 40]).any(), "row %d" % i
                assert np.isfinite(out[i][:, :32]).all()


@pytest.mark.parametrize("max_q", [0, 3, 9, 2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 1])
def test_max_q_of_any_size(G, max_q):
    """At most max_q query tokens of a sequence are served, however large it is."""
    rng = np.random.default_rng(65)
    cache, table, lens, _, _ = held(rng.standard_normal((50, 1, 64)), rng.standard_normal((50, 1, 64)))
    q = torch.randn((9, 4, 64), device=DEV).bfloat16()
    start = torch.tensor([0, 9], dtype=torch.int32, device=DEV)
    note("max_q = %d" % max_q)
    want = G.gvr_kv4_attention(q, cache, table, lens, 1)
    out = G.gvr_kv4_attention(q, cache, table, lens, 1, q_start=start, max_q=max_q, out=torch.full_like(q, 3.0))
    served = min(max_q, 9)
    assert (out[served:] == 3).all() and torch.equal(out[:served], want[:served])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,group", [(64, 2, 4), (128, 1, 8), (128, 1, 40), (256, 2, 2)])
def test_selection_over_a_prompt(G, D, heads, group, dtype):
    """A list for every query token of a prompt: whole ones, short ones (-1 behind), and the first tokens' few."""
    rng = np.random.default_rng(66)
    ctx, nq, K = [300, 70, 0], 70, 48
    seqs = Sequences(rng, ctx, 16, heads, D)
    cache, table, lens = seqs.on_gpu()
    sel = np.full((len(ctx) * nq, K), -1, np.int32)
    for b, c in enumerate(ctx):
        for i in range(nq):
            see = max(0, c - nq + 1 + i)
            pick = np.sort(rng.permutation(see)[:K - 20 * (i % 3 == 2)])
            sel[b * nq + i, :len(pick)] = pick
    q = torch.from_numpy(rng.standard_normal((len(ctx) * nq, heads * group, D))).to(TORCH[dtype]).to(DEV)
    note("selection over a prompt: %s D=%d heads=%d group=%d" % (dtype, D, heads, group))
    lse = torch.empty((q.shape[0], q.shape[1]), device=DEV)
    out = G.gvr_kv4_attention(q, cache, table, lens, heads, selection=torch.from_numpy(sel).to(DEV), lse=lse)
    check_attention(out, lse, q, seqs, [nq * b for b in range(len(ctx) + 1)], D ** -0.5, selection=sel, dtype=dtype,
                    what="selection over a prompt")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group,nq", [(64, 2, 4), (64, 5, 7), (128, 16, 3), (128, 4, 40), (256, 2, 70), (64, 1, 140)])
def test_rows_beside_nan_blocks_are_right(G, dtype, D, group, nq):
    """Value and key blocks that are NaN, in tokens that only the later queries see: the earlier rows equal the oracle's
    within their roundings, split or not."""
    rng = np.random.default_rng(67)
    n, split = 300, nq // 2
    first = n - nq + split
    k, v = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
    v[first:, 0, 40] = np.nan
    k[first + 1:, 0, 3] = np.inf
    cache, table, lens, kk, vv = held(k, v)
    q = torch.from_numpy(rng.standard_normal((nq, group, D))).to(TORCH[dtype]).to(DEV)
    u, scale = UNIT[dtype], D ** -0.5
    for ws in (torch.empty(0, dtype=torch.uint8, device=DEV), None):
        note("rows beside NaN: %s D=%d group %d nq %d %s" % (dtype, D, group, nq, "split" if ws is None else "whole"))
        out = f64(G.gvr_kv4_attention(q, cache, table, lens, 1, workspace=ws))
        for i in range(nq):
            t = n - nq + i + 1
            if i >= split:
                seen = out[i] if i > split else out[i][:, 32:64]     # a NaN key: everything; a NaN value: its block
                assert np.isnan(seen).all() and (i > split or np.isfinite(out[i][:, :32]).all())
                continue
            ref, _, mag = O.attention(f64(q)[i], kk[:t], vv[:t], scale)
            qk = (np.abs(kk[:t, 0]) @ np.abs(f64(q)[i]).T).max()
            eps = ((D + 8) * scale * qk + t + 64) * 2.0 ** -24
            tol = (u + 2 * eps) * (1 + u) * mag + u * np.abs(ref) + t * 2.0 ** -40 * np.abs(vv[:t]).max() + 2.0 ** -25
            assert (np.abs(out[i] - ref) <= tol).all(), "row %d" % i


@pytest.mark.parametrize("dtype", ["f16"])
@pytest.mark.parametrize("D,nq", [(64, 1), (128, 20), (128, 70), (256, 1), (256, 70)])
@pytest.mark.parametrize("scale", [1e6, -1e6, 3e28])
def test_scores_past_2_31(G, dtype, D, nq, scale):
    """One token takes all the weight where the scores pass 2^31, up to 1e34 (float16; bfloat16 is for less, as its
    header says)."""
    rng = np.random.default_rng(68)
    k, v = one_ahead(900, D, 3.0, rng)
    k[:, 0, 1] = 6.0
    if scale < 0:
        k = -k
    cache, table, lens, _, vv = held(k, v)
    q = torch.zeros((nq, 2, D), dtype=TORCH[dtype], device=DEV)
    q[:, :, 0] = q[:, :, 1] = 60000.0
    for ws in (torch.empty(0, dtype=torch.uint8, device=DEV), None):
        note("scores past 2^31: %s D=%d nq=%d scale %g" % (dtype, D, nq, scale))
        out = G.gvr_kv4_attention(q, cache, table, lens, 1, scale=scale, causal=False, workspace=ws)
        assert np.array_equal(f64(out), np.broadcast_to(vv[7], out.shape))


@pytest.mark.parametrize("dtype,huge", [("f16", 60000.0), ("bf16", 3.3e38)])
@pytest.mark.parametrize("D,group,nq", [(64, 4, 1), (128, 16, 3), (128, 4, 40), (256, 2, 70), (64, 1, 140)])
def test_visible_infinities_stay_in_their_dimension(G, dtype, huge, D, group, nq):
    """Values that the 16-bit type cannot hold, in tokens that every query sees (not causal; the first and the last): the
    other dimensions are right, those of the same block of 32 among them."""
    rng = np.random.default_rng(70)
    n = 300
    k, v = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
    v[[3, n - 1], 0, 32:64] = 0.0               # (beside the large value every other is less than half a step)
    v[[3, n - 1], 0, 40] = huge
    cache, table, lens, kk, vv = held(k, v)
    q = torch.from_numpy(rng.standard_normal((nq, group, D))).to(TORCH[dtype]).to(DEV)
    u, scale = UNIT[dtype], D ** -0.5
    rest = np.arange(D) != 40
    for ws in (torch.empty(0, dtype=torch.uint8, device=DEV), None):
        note("visible infinities: %s D=%d group %d nq %d %s" % (dtype, D, group, nq, "split" if ws is None else "whole"))
        out = f64(G.gvr_kv4_attention(q, cache, table, lens, 1, causal=False, workspace=ws))
        assert not np.isfinite(out[..., 40]).any()
        for i in range(nq):
            ref, _, mag = O.attention(f64(q)[i], kk, vv, scale)
            qk = (np.abs(kk[:, 0]) @ np.abs(f64(q)[i]).T).max()
            eps = ((D + 8) * scale * qk + n + 64) * 2.0 ** -24
            tol = (u + 2 * eps) * (1 + u) * mag + u * np.abs(ref) + n * 2.0 ** -40 * np.abs(vv[:, 0, rest]).max() + 2.0 ** -25
            assert (np.abs(out[i] - ref) <= tol)[:, rest].all(), "row %d" % i
