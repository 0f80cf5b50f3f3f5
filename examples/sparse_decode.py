"""A layer's sparse attention, from prompt to decode steps, on random tensors.

What a serving program does with one layer of a model whose decode attention
reads only the tokens that an indexer selects:

* the hidden states go through the layer's projections in 8 bits (codes with a
  scale per 128 elements on both sides): queries, keys, values, and the indexer's
  queries and keys;
* a page step hands out the pages of the new tokens and says where each goes;
* a prompt chunk: keys and values go into the paged 4-bit cache (keys rotated on
  the way), the indexer's keys into its FP8 cache, the queries are rotated and
  attend over everything up to themselves;
* a decode step: the same for one token (or a few draft tokens) of each request,
  except that the FP8 indexer and the exact Top-K, guided by the step before,
  say which tokens the queries attend to.

    python examples/sparse_decode.py --requests 8 --prompt 4096 --steps 4
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2604_22312_amd as gvr  # noqa: E402


class Projections:
    """The layer's projections of hidden states, weights [out][hidden] in 8 bits: queries,
    keys, values, the indexer's queries and its key (one for all its heads)."""

    def __init__(self, hidden, q_heads=32, kv_heads=8, head_dim=128, index_heads=64, index_dim=128, device="cuda"):
        self.parts = [(q_heads, head_dim), (kv_heads, head_dim), (kv_heads, head_dim), (index_heads, index_dim), (1, index_dim)]
        weight = torch.randn((sum(h * d for h, d in self.parts), hidden), device=device) / hidden ** 0.5
        self.weight = gvr.gvr_fp8_quantize_matrix(weight.bfloat16(), square=True)

    def __call__(self, x):
        """x [T][hidden]: the five projections [T][heads][dim], strided views of one product."""
        y = gvr.gvr_fp8_matmul(*gvr.gvr_fp8_quantize(x), *self.weight, dtype=x.dtype)
        return [t.unflatten(1, hd) for t, hd in zip(y.split([h * d for h, d in self.parts], dim=1), self.parts)]


class SparseLayer:
    """Cache, pages and rotary table of one layer, for `requests` requests
    of at most `longest` tokens."""

    def __init__(self, requests, longest, q_heads=32, kv_heads=8, head_dim=128, K=2048, page=64, drafts=1,
                 index_heads=64, index_dim=128, device="cuda"):
        self.R, self.drafts, self.K, self.page, self.dev = requests, drafts, K, page, device
        self.q_heads, self.kv_heads, self.D = q_heads, kv_heads, head_dim
        pages = (longest + page - 1) // page
        self.cache = gvr.new_kv4_cache(requests * pages, page, kv_heads, head_dim, device)
        self.pool = gvr.new_page_pool(requests * pages, page, requests, pages, device)
        # any page may belong to any request
        self.pool.free_pages.copy_(torch.randperm(requests * pages, device=device))
        self.blocks, self.length = self.pool.block_table, self.pool.ctx_len
        self.table = gvr.gvr_rope_table(longest, dict(d_rope=head_dim), gain=1.0, device=device)
        self.longest, self.tokens = longest, 0   # (of each request, known without asking the device)
        # the indexer's keys: FP8 bytes and a scale per token
        self.index_k = torch.zeros((requests, longest, index_dim), dtype=torch.uint8, device=device)
        self.index_scale = torch.ones((requests, longest), device=device)
        self.index_w = torch.randn((requests * drafts, index_heads), device=device) / index_heads ** 0.5
        self.selected = None

    def _store(self, k, v, index_k, new):
        """Append `new` tokens of every request; what the step says of them."""
        if self.tokens + new > self.longest:
            raise ValueError("%d tokens a request, of at most %d" % (self.tokens + new, self.longest))
        self.tokens += new
        brought = torch.full((self.R,), new, dtype=torch.int32, device=self.dev)
        step = gvr.gvr_page_step(self.pool, brought, self.R * new, ld=self.longest)
        gvr.gvr_kv4_append(k, v, step.slots, self.cache, table=self.table, positions=step.positions)
        if index_k.dtype == torch.uint8:
            self.index_k.view(self.R * self.longest, -1)[step.dense] = index_k
        else:
            gvr.gvr_fp8_quantize(index_k.view(len(index_k), -1), pow2=True, slots=step.dense, codes=self.index_k.flatten(0, 1),
                                 scale=self.index_scale.view(-1, 1))
        return step

    def prompt(self, q, k, v, index_k):
        """q [R * n][q_heads][D] and k, v [R * n][kv_heads][D] of n prompt tokens
        per request; index_k [R * n][index_dim] FP8 bytes, or values to quantise."""
        step = self._store(k, v, index_k, q.shape[0] // self.R)
        q = gvr.gvr_rope_rotate(q, step.positions, self.table)
        return gvr.gvr_kv4_attention(q, self.cache, self.blocks, self.length, self.kv_heads)

    def decode(self, q, k, v, index_q, index_k):
        """One step of `drafts` tokens per request: q [R * drafts][q_heads][D],
        index_q [R * drafts][index_heads][index_dim] FP8 bytes, or values to quantise."""
        step = self._store(k, v, index_k, self.drafts)
        q = gvr.gvr_rope_rotate(q, step.positions, self.table)
        weights = self.index_w
        if index_q.dtype != torch.uint8:   # (a query's scale goes into its heads' weights)
            index_q, scale = gvr.gvr_fp8_quantize(index_q, pow2=True)
            weights = weights * scale.squeeze(2)
        self.selected, _ = gvr.gvr_indexer_topk(index_q.contiguous(), weights, self.index_k, self.index_scale, step.row_len,
                                                self.selected, self.K)
        return gvr.gvr_kv4_attention(q, self.cache, self.blocks, self.length, self.kv_heads, selection=self.selected)


def fp8(shape, device):
    return torch.randn(shape, device=device).to(torch.float8_e4m3fn).view(torch.uint8)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--drafts", type=int, default=1)
    ap.add_argument("--hidden", type=int, default=4096)
    a = ap.parse_args()
    dev = "cuda"
    layer = SparseLayer(a.requests, a.prompt + a.steps * a.drafts, drafts=a.drafts)
    project = Projections(a.hidden)

    for n, name in [(a.prompt, "prompt")] + [(a.drafts, "step %d" % i) for i in range(a.steps)]:
        x = torch.randn((a.requests * n, a.hidden), device=dev).bfloat16()
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        q, k, v, iq, ik = project(x)
        out = layer.prompt(q, k, v, ik) if name == "prompt" else layer.decode(q, k, v, iq, ik)
        end.record()
        end.synchronize()
        print("%s: %d tokens a request, context %d, mean |out| %.4f, %.1f us" % (
            name, n, int(layer.length[0]), out.float().abs().mean().item(), 1e3 * start.elapsed_time(end)), flush=True)


if __name__ == "__main__":
    main()
