"""Inputs and comparisons of the GPU tests of rotary positions and the 4-bit
cache. The cache's bytes come from the oracle's quantiser or are random."""
import numpy as np
import torch

from oracle import kv4 as O

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def f64(t):
    return t.detach().cpu().double().numpy()


def random_cache(rng, pages, page, heads, D, nan_slots=()):
    """Cache bytes with every code and a spread of scales; given slots hold NaN blocks only."""
    rec = heads * D * 17 // 16
    c = rng.integers(0, 256, (pages * page, rec), dtype=np.uint8)
    c[:, heads * D:] = rng.integers(122, 128, (pages * page, rec - heads * D))
    for s in nan_slots:
        c[s, heads * D:] = 255
    return c.reshape(pages, page, rec)


class Sequences:
    """Paged sequences with shuffled pages; spare pages hold NaN records."""

    def __init__(self, rng, ctx, page, heads, D, width=None, nan_tail=True):
        need = [(c + page - 1) // page for c in ctx]
        pages = sum(need) + 2
        order = rng.permutation(pages)
        width = max(need + [1]) + 1 if width is None else width
        self.table = rng.integers(-3, 0, (len(ctx), width)).astype(np.int32)   # unused entries: no page
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.ctx, self.page, self.heads, self.D = list(ctx), page, heads, D
        self.cache = random_cache(rng, pages, page, heads, D)
        if nan_tail:
            # records that no sequence holds must never show: the spare pages and what follows a sequence's end
            flat = self.cache.reshape(pages * page, -1)
            held = np.zeros(pages * page, bool)
            for b, c in enumerate(ctx):
                held[self.slots(b, np.arange(c))] = True
            flat[~held, heads * D:] = 255

    def slots(self, b, tokens):
        tokens = np.asarray(tokens, dtype=np.int64)
        return self.table[b, tokens // self.page].astype(np.int64) * self.page + tokens % self.page

    def kv(self, b, tokens):
        flat = self.cache.reshape(-1, self.cache.shape[-1])
        return O.values(flat[self.slots(b, tokens)], self.heads, self.D)

    def on_gpu(self):
        return (torch.from_numpy(self.cache).to(DEV), torch.from_numpy(self.table).to(DEV),
                torch.tensor(self.ctx, dtype=torch.int32, device=DEV))


def visible(ctx, nq, i, causal, sel=None):
    last = ctx - nq + i if causal else ctx - 1
    if sel is None:
        return np.arange(max(last + 1, 0))
    return sel[(sel >= 0) & (sel <= last)]


def check_attention(out, lse, q, seqs, starts, scale, causal=True, selection=None, dtype="bf16", what=""):
    """out, lse against the float64 oracle, row by row.

    Weights carry one rounding to the 16-bit type (unit u; float16 weights
    below its normal range 2^-25 instead), the scores an error of at most
    (D + 8) 2^-24 scale sum |q k| from their float32 sum and scaling, the sums
    over n tokens (n + 64) 2^-24 whatever their order, and the result one more
    rounding."""
    u = UNIT[dtype]
    out, qd = f64(out), f64(q)
    lse = None if lse is None else f64(lse)
    D = qd.shape[2]
    for b, c in enumerate(seqs.ctx):
        nq = starts[b + 1] - starts[b]
        for i in range(nq):
            r = starts[b] + i
            t = visible(c, nq, i, causal, None if selection is None else selection[r])
            k, v = seqs.kv(b, t)
            ref, ref_lse, mag = O.attention(qd[r], k, v, scale)
            assert np.isfinite(out[r]).all(), "%s: row %d is not finite" % (what, r)
            n = len(t)
            if n == 0:
                assert not out[r].any(), "%s: row %d sees nothing and is not zero" % (what, r)
                assert lse is None or np.isneginf(lse[r]).all()
                continue
            g = qd.shape[1] // seqs.heads
            qk = np.stack([(np.abs(k[:, h // g]) @ np.abs(qd[r, h])).max() for h in range(qd.shape[1])])
            eps = ((D + 8) * abs(scale) * qk + n + 64) * 2.0 ** -24
            vmax = np.repeat(np.abs(v).max(axis=0), g, axis=0)
            tol = (u + 2 * eps[:, None]) * mag * (1 + u) + u * np.abs(ref) + 1e-30
            if dtype == "f16":
                tol = tol + n * 2.0 ** -25 * vmax + 2.0 ** -24
            bad = np.abs(out[r] - ref) > tol
            assert not bad.any(), "%s: row %d (%d tokens): worst %.3g of its tolerance" % (
                what, r, n, (np.abs(out[r] - ref) / tol).max())
            if lse is not None:
                assert (np.abs(lse[r] - ref_lse) <= 2 * eps + 4 * 2.0 ** -24 * (np.abs(ref_lse) + 1)).all(), what
