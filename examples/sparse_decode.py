"""A layer's sparse attention, from prompt to decode steps, on random tensors.

What a serving program does with one layer of a model whose decode attention
reads only the tokens that an indexer selects:

* a prompt chunk: keys and values go into the paged 4-bit cache (keys rotated on
  the way), the queries are rotated and attend over everything up to themselves;
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


class SparseLayer:
    """Cache, page table and rotary table of one layer, for `requests` requests
    of at most `longest` tokens."""

    def __init__(self, requests, longest, q_heads=32, kv_heads=8, head_dim=128, K=2048, page=64, drafts=1,
                 index_heads=64, index_dim=128, device="cuda"):
        self.R, self.drafts, self.K, self.page, self.dev = requests, drafts, K, page, device
        self.q_heads, self.kv_heads, self.D = q_heads, kv_heads, head_dim
        pages = (longest + page - 1) // page
        self.cache = gvr.new_kv4_cache(requests * pages, page, kv_heads, head_dim, device)
        # any page may belong to any request
        self.blocks = torch.randperm(requests * pages, device=device).to(torch.int32).view(requests, pages)
        self.table = gvr.gvr_rope_table(longest, dict(d_rope=head_dim), gain=1.0, device=device)
        self.length = torch.zeros(requests, dtype=torch.int32, device=device)
        self.longest, self.tokens = longest, 0   # (of each request, known without asking the device)
        # the indexer's keys: FP8 bytes and a scale per token
        self.index_k = torch.zeros((requests, longest, index_dim), dtype=torch.uint8, device=device)
        self.index_scale = torch.ones((requests, longest), device=device)
        self.index_w = torch.randn((requests * drafts, index_heads), device=device) / index_heads ** 0.5
        self.selected = None

    def _store(self, k, v, index_k, new):
        """Append `new` tokens of every request; their positions (int32 [R * new])."""
        if self.tokens + new > self.longest:
            raise ValueError("%d tokens a request, of at most %d" % (self.tokens + new, self.longest))
        self.tokens += new
        pos = self.length.view(-1, 1) + torch.arange(new, dtype=torch.int32, device=self.dev)
        slots = torch.gather(self.blocks, 1, (pos // self.page).long()).long() * self.page + pos % self.page
        pos = pos.view(-1)
        gvr.gvr_kv4_append(k, v, slots.view(-1), self.cache, table=self.table, positions=pos)
        at = pos.view(self.R, new).long()
        self.index_k.scatter_(1, at.unsqueeze(2).expand(-1, -1, index_k.shape[1]), index_k.view(self.R, new, -1))
        self.length += new
        return pos

    def prompt(self, q, k, v, index_k):
        """q [R * n][q_heads][D] and k, v [R * n][kv_heads][D] of n prompt tokens
        per request; index_k [R * n][index_dim] FP8 bytes."""
        pos = self._store(k, v, index_k, q.shape[0] // self.R)
        q = gvr.gvr_rope_rotate(q, pos, self.table)
        return gvr.gvr_kv4_attention(q, self.cache, self.blocks, self.length, self.kv_heads)

    def decode(self, q, k, v, index_q, index_k):
        """One step of `drafts` tokens per request: q [R * drafts][q_heads][D],
        index_q [R * drafts][index_heads][index_dim] FP8 bytes."""
        pos = self._store(k, v, index_k, self.drafts)
        q = gvr.gvr_rope_rotate(q, pos, self.table)
        self.selected, _ = gvr.gvr_indexer_topk(index_q, self.index_w, self.index_k, self.index_scale, pos + 1,
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
    a = ap.parse_args()
    dev = "cuda"
    layer = SparseLayer(a.requests, a.prompt + a.steps * a.drafts, drafts=a.drafts)

    def heads(n, h):
        return torch.randn((a.requests * n, h, layer.D), device=dev).bfloat16()

    for n, name in [(a.prompt, "prompt")] + [(a.drafts, "step %d" % i) for i in range(a.steps)]:
        q, k, v = heads(n, layer.q_heads), heads(n, layer.kv_heads), heads(n, layer.kv_heads)
        ik = fp8((a.requests * n, 128), dev)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        out = layer.prompt(q, k, v, ik) if name == "prompt" else \
            layer.decode(q, k, v, fp8((a.requests * n, 64, 128), dev), ik)
        end.record()
        end.synchronize()
        print("%s: %d tokens a request, context %d, mean |out| %.4f, %.1f us" % (
            name, n, int(layer.length[0]), out.float().abs().mean().item(), 1e3 * start.elapsed_time(end)), flush=True)


if __name__ == "__main__":
    main()
