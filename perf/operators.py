"""Performance cases of the operators around a selected-token decode step:
rotary positions, appending to a paged 4-bit key / value cache, and attention
over that cache (every token, or a Top-K selection of them).

A serving program rotates its queries, appends the new keys and values (the
keys rotated on the way) and attends over the cache: prompts in chunks of
thousands of queries, decode steps of one to a few draft rows per request, and
with sparse attention over the indices that the Top-K returned.

The cache is a uint8 tensor [pages][page_size][record]. A token's record holds,
for KV heads of D elements, the E2M1 codes of its keys ([heads][D / 2], the even
element in the low four bits), the codes of its values, then one E8M0 scale byte
per 32 elements of the keys ([heads][D / 32]) and of the values.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 32        # elements that share a scale
POSITIONS = 131072
#: Rotary settings of the tables: base, and YaRN's original context, factor and ramp.
ROPE_BASE, ROPE_CTX, ROPE_SCALE, ROPE_FAST, ROPE_SLOW = 10000.0, 4096, 40.0, 32.0, 1.0
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
#: Most work of a drawn case: elements of a rotation or an append, record bytes
#: and query-key products (times heads and dimensions) of an attention.
MAX_ELEMS, MAX_BYTES, MAX_PRODUCTS = 16384 * 16 * 128, 32 * 32768 * 1088, 4096 * 30720 * 32 * 128


def _rope(name, tokens, heads, D, rot, **kw):
    case = {"kind": "rope", "tokens": tokens, "heads": heads, "D": D, "rot": rot, "dtype": "bf16",
            "interleaved": False, "inverse": False, "fused": False, "prompt": False}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def _append(name, tokens, heads, D, rot, **kw):
    case = {"kind": "append", "tokens": tokens, "heads": heads, "D": D, "rot": rot, "dtype": "bf16",
            "interleaved": False, "page": 64, "skip": False, "prompt": False}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def _attention(name, requests, rows, ctx, **kw):
    case = {"kind": "attention", "requests": requests, "rows": rows, "ctx": ctx, "q_heads": 32, "heads": 8, "D": 128,
            "dtype": "bf16", "page": 64, "K": 0, "ragged": False, "causal": True}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the benchmark's decode step (64 requests, two draft rows), 64 heads, half of each head rotated
        _rope("rope_decode_b128", 128, 64, 128, 64),
        # a prompt chunk's queries, whole heads, read out of a fused projection
        _rope("rope_prompt_8k", 8192, 32, 128, 128, fused=True, prompt=True),
        # training: the gradient of interleaved positions in float32, an odd number of tokens
        _rope("rope_grad_4099_f32", 4099, 8, 128, 96, dtype="f32", interleaved=True, inverse=True, prompt=True),
        # one request's next token into the cache: latency is everything
        _append("append_b1", 1, 8, 128, 128),
        # a long prompt into fragmented pages
        _append("append_prompt_16k", 16384, 8, 128, 128, prompt=True),
        # odd heads and tokens, padded rows that are skipped, small pages
        _append("append_odd_f32", 1021, 3, 64, 32, dtype="f32", interleaved=True, page=16, skip=True),
        # one request, a short context: latency is everything
        _attention("decode_1k_b1", 1, 1, 1031),
        # an ordinary decode batch
        _attention("decode_32k_b32", 32, 1, 32768),
        # one very long context, split over the whole chip
        _attention("decode_512k_b1", 1, 1, 524289, q_heads=64),
        # the benchmark's decode step with the Top-K's selection: 64 requests, two draft rows each, 100K tokens
        _attention("selected_100k_b128", 64, 2, 102463, q_heads=64, K=2048),
        # a chunk of a long prompt: the queries see the chunks before them and themselves
        _attention("prompt_4k_of_32k", 1, 4096, 32768),
        # mixed lengths, some requests not started, three draft rows, small heads and pages
        _attention("decode_ragged_b48_f16", 48, 3, 16384, q_heads=16, heads=2, D=64, dtype="f16", page=16, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "append", "append", "decode", "decode", "selected", "selected", "prompt"])
    D = rng.choice([64, 128, 128, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    rot = rng.choice([D, D, D // 2, D // 4 + 8])
    page = rng.choice([16, 64, 128])
    if kind == "rope":
        heads = rng.choice([1, 5, 8, 32, 64])
        return _rope(None, _log_int(rng, 1, min(16384, MAX_ELEMS // (heads * D))), heads, D, rot, dtype=dtype,
                     interleaved=rng.random() < 0.5, inverse=rng.random() < 0.3, fused=rng.random() < 0.3,
                     prompt=rng.random() < 0.5)
    if kind == "append":
        heads = rng.choice([1, 2, 3, 4, 8])
        return _append(None, _log_int(rng, 1, min(16384, MAX_ELEMS // (2 * heads * D))), heads, D, rot, dtype=dtype,
                       interleaved=rng.random() < 0.5, page=page, skip=rng.random() < 0.3, prompt=rng.random() < 0.5)
    heads = rng.choice([1, 2, 4, 8, 8])
    kw = {"heads": heads, "q_heads": heads * rng.choice([1, 4, 5, 8, 16]), "D": D, "page": page,
          "dtype": rng.choice(["bf16", "bf16", "f16"])}
    record = heads * D * 17 // 16
    if kind == "prompt":
        ctx = _log_int(rng, 16, 32768)
        requests = rng.randint(1, 4)
        most = max(1, min(4096, ctx, MAX_PRODUCTS // (requests * ctx * kw["q_heads"] * D)))
        return _attention(None, requests, _log_int(rng, 1, most), ctx, ragged=rng.random() < 0.5,
                          causal=rng.random() < 0.8, **kw)
    if kind == "selected":
        ctx = _log_int(rng, 256, 131072)
        return _attention(None, _log_int(rng, 1, max(1, min(96, 4 * MAX_BYTES // (ctx * record)))), rng.randint(1, 3), ctx,
                          K=rng.choice([2048, 2048, rng.randint(64, 2048)]), ragged=rng.random() < 0.3, **kw)
    ctx = _log_int(rng, 1, 262144)
    most = max(1, min(256, MAX_BYTES // (ctx * record)))
    return _attention(None, _log_int(rng, 1, most), rng.randint(1, 4), ctx, ragged=rng.random() < 0.4, **kw)


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _table(rot, gen):
    """Cosines and sines [POSITIONS][rot / 2][2] of YaRN-scaled positions, times its attention factor."""
    half = rot // 2
    i = torch.arange(half, dtype=torch.float64, device=DEV)
    rate = ROPE_BASE ** (-2.0 * i / rot)

    def edge(rotations):
        return rot * math.log(ROPE_CTX / (2.0 * math.pi * rotations)) / (2.0 * math.log(ROPE_BASE))

    lo, hi = max(math.floor(edge(ROPE_FAST)), 0), min(math.ceil(edge(ROPE_SLOW)), rot - 1)
    ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
    rate = rate * (1.0 - ramp) + rate / ROPE_SCALE * ramp
    phase = torch.arange(POSITIONS, dtype=torch.float64, device=DEV).unsqueeze(1) * rate
    gain = 0.1 * math.log(ROPE_SCALE) + 1.0
    return (torch.stack((torch.cos(phase), torch.sin(phase)), dim=-1) * gain).float().contiguous()


def _positions(case, gen):
    """A prompt's are consecutive, a decode batch's anywhere."""
    n = case["tokens"]
    if case["prompt"]:
        first = torch.randint(0, POSITIONS - n + 1, (1,), generator=gen, device=DEV)
        return (first + torch.arange(n, device=DEV)).to(torch.int32)
    return torch.randint(0, POSITIONS, (n,), generator=gen, device=DEV).to(torch.int32)


def _normal(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(DTYPES[dtype])


def _record(heads, D):
    return heads * (D + D // 16)


def _code_bytes():
    """65536 bytes of two codes each, drawn as a unit normal rounds at a scale of 1/2."""
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64) / 2
    cdf = torch.erf(edges / math.sqrt(2.0))
    u = (torch.arange(256, dtype=torch.float64) + 0.5) / 128.0 - 1.0
    codes = torch.bucketize(u.abs(), cdf) + 8 * (u < 0)
    return (codes.unsqueeze(0) + 16 * codes.unsqueeze(1)).reshape(-1).to(torch.uint8).to(DEV)


def _random_cache(pages, page, heads, D, gen):
    cache = torch.empty((pages, page, _record(heads, D)), dtype=torch.uint8, device=DEV)
    pairs = _code_bytes()
    spread = torch.tensor([126] * 13 + [125] * 2 + [127], dtype=torch.uint8, device=DEV)
    flat = cache.view(pages * page, -1)
    step = max(1, (1 << 27) // flat.shape[1])
    for t in range(0, flat.shape[0], step):
        part = flat[t:t + step]
        part[:, :heads * D] = pairs[torch.randint(0, 65536, (part.shape[0], heads * D), generator=gen, device=DEV,
                                                  dtype=torch.int32)]
        part[:, heads * D:] = spread[torch.randint(0, 16, (part.shape[0], heads * D // 16), generator=gen,
                                                   device=DEV, dtype=torch.int32)]
    return cache


def _lengths(case):
    """Context lengths and query rows of each request, the same for every seed."""
    n, requests, rows = case["ctx"], case["requests"], case["rows"]
    ctx, q = [n] * requests, [rows] * requests
    if case["ragged"]:
        rng = random.Random(requests * 1000003 + n)
        # most lengths spread evenly, one request of eight not started or just started
        ctx = [rng.randint(0, min(n, 1)) if rng.random() < 0.125 else rng.randint(n // 8, n) for _ in range(requests)]
        if rows > 4:
            q = [min(c, rng.randint(rows // 4, rows)) for c in ctx]
        ctx[0], q[0] = n, rows
    return ctx, q


def _prepare_attention(case, seed):
    gen = _generator(seed)
    heads, D, page, rows = case["heads"], case["D"], case["page"], case["rows"]
    ctx, nq = _lengths(case)
    need = [max(1, (c + page - 1) // page) for c in ctx]
    pages = sum(need)
    cache = _random_cache(pages + 1, page, heads, D, gen)
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    blocks = torch.full((len(ctx), max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, m in enumerate(need):
        blocks[b, :m] = order[at:at + m]
        at += m
    starts = [0]
    for m in nq:
        starts.append(starts[-1] + m)
    st = {"case": case, "ctx": ctx, "nq": nq, "starts": starts, "cache": cache, "blocks": blocks,
          "ctx_len": torch.tensor(ctx, dtype=torch.int32, device=DEV), "selection": None, "q_start": None,
          "scale": 1.0 / math.sqrt(D)}
    st["q"] = (1.5 * torch.randn((starts[-1], case["q_heads"], D), generator=gen, device=DEV)).to(DTYPES[case["dtype"]])
    if len(set(nq)) > 1:
        st["q_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    if case["K"]:
        # a request's draft rows keep nearly the same tokens: a tenth of them differ
        K, extra = case["K"], max(1, case["K"] // 10)
        sel = torch.full((len(ctx), rows, K), -1, dtype=torch.int32, device=DEV)
        for b, c in enumerate(ctx):
            for r in range(rows):
                see = max(0, c - rows + 1 + r)
                if see <= K:
                    sel[b, r, :see] = torch.arange(see, dtype=torch.int32, device=DEV)
            if c - rows + 1 > K + extra:
                some = torch.rand(c - rows + 1, generator=gen, device=DEV).topk(K + extra, sorted=False).indices
                some = some[torch.randperm(K + extra, generator=gen, device=DEV)]
                for r in range(rows):
                    keep = some[:K] if r == 0 else torch.cat((some[:K - extra], some[K:]))
                    sel[b, r] = keep.sort().values.to(torch.int32)
            elif c - rows + 1 > K:
                for r in range(rows):
                    sel[b, r] = torch.rand(c - rows + 1, generator=gen, device=DEV).topk(K).indices.sort().values
        st["selection"] = sel.view(len(ctx) * rows, K)
    if own:
        import paper_2604_22312_amd as gvr
        st["call"] = gvr.prepare_gvr_kv4_attention(st["q"], cache, blocks, st["ctx_len"], heads, selection=st["selection"],
                                               q_start=st["q_start"], max_q=max(nq), causal=case["causal"],
                                               scale=st["scale"])
    return st


def prepare(case, seed):
    kind = case["kind"]
    if kind == "attention":
        return _prepare_attention(case, seed)
    gen = _generator(seed)
    n, heads, D, dt = case["tokens"], case["heads"], case["D"], case["dtype"]
    st = {"case": case, "table": _table(case["rot"], gen), "positions": _positions(case, gen)}
    if kind == "rope":
        # of a fused projection: the queries, then a key and a value head for every eight query heads
        wide = heads + 2 * ((heads + 7) // 8) if case["fused"] else heads
        st["x"] = _normal((n, wide, D), dt, gen)[:, :heads]
        if own:
            import paper_2604_22312_amd as gvr
            st["call"] = gvr.prepare_gvr_rope_rotate(st["x"], st["positions"], st["table"], interleaved=case["interleaved"],
                                                 inverse=case["inverse"])
        return st
    page = case["page"]
    pages = 2 * ((n + page - 1) // page) + 1   # the last page belongs to no request
    st["k"], st["v"] = _normal((n, heads, D), dt, gen), _normal((n, heads, D), dt, gen)
    st["cache"] = torch.zeros((pages, page, _record(heads, D)), dtype=torch.uint8, device=DEV)
    order = torch.randperm(pages - 1, generator=gen, device=DEV)
    if case["prompt"]:   # consecutive tokens fill page after page
        t = torch.arange(n, device=DEV)
        st["slots"] = order[t // page] * page + t % page
    else:                # one token each of as many requests
        st["slots"] = torch.randperm((pages - 1) * page, generator=gen, device=DEV)[:n].contiguous()
    if case["skip"]:
        st["slots"] = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.1, -1, st["slots"])
    if own:
        import paper_2604_22312_amd as gvr
        st["append"] = gvr.prepare_gvr_kv4_append(st["k"], st["v"], st["slots"], st["cache"], table=st["table"],
                                              positions=st["positions"], interleaved=case["interleaved"])
        st["read"] = gvr.prepare_gvr_kv4_read(st["cache"], st["slots"], heads, D, dtype=DTYPES[dt])
    return st


def _rotated(x, table, positions, interleaved, inverse):
    """x [n][heads][D] in float32 with its first 2 * table.shape[1] elements rotated."""
    rot = 2 * table.shape[1]
    cs = table[positions.long()].unsqueeze(1)
    c, s = cs[..., 0], cs[..., 1]
    if inverse:
        s = -s
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * c - b * s, b * c + a * s
    turned = torch.stack((ra, rb), dim=-1).flatten(-2) if interleaved else torch.cat((ra, rb), dim=-1)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def _quantised(x):
    """Codes [n][heads * D / 2] and scale bytes [n][heads * D / 32] of x [n][heads][D] float32."""
    n = x.shape[0]
    blocks = x.reshape(n, -1, BLOCK)
    bits = blocks.abs().amax(dim=-1).view(torch.int32)
    # the least power of two that keeps the largest element within 7 steps of it
    scale = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(1, 254)
    unit = ((254 - scale) << 23).view(torch.float32).unsqueeze(-1)
    y = blocks * unit
    m = y.abs()
    code = ((m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
            + 8 * (y < 0))
    code = code.view(n, -1, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scale.to(torch.uint8)


def _unpacked(rec, heads, D):
    """Keys and values [...][heads][D] in float32 of records [...][record]."""
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=rec.device)
    value = torch.cat((value, -value))
    byte = torch.arange(256, device=rec.device)
    pairs = torch.stack((value[byte & 15], value[byte >> 4]), dim=-1)
    half, blocks, out = heads * D // 2, heads * D // BLOCK, []
    for i in range(2):
        codes = pairs[rec[..., i * half:(i + 1) * half].int()].reshape(rec.shape[:-1] + (blocks, BLOCK))
        scale = rec[..., 2 * half + i * blocks:2 * half + (i + 1) * blocks].float() - 127.0
        out.append((codes * torch.exp2(scale).unsqueeze(-1)).reshape(rec.shape[:-1] + (heads, D)))
    return out


def _attend(q, k, v, see, scale):
    """Attention of q [b][m][q heads][D] to k, v [b][n][heads][D], where see [b][m][n]; float32."""
    b, m, hq, D = q.shape
    h, n = k.shape[2], k.shape[1]
    g = hq // h
    qh = q.view(b, m, h, g, D).permute(0, 2, 3, 1, 4).reshape(b * h, g * m, D)
    kh = k.permute(0, 2, 3, 1).reshape(b * h, D, n)
    s = (torch.matmul(qh, kh) * scale).view(b, h, g, m, n)
    s = s.masked_fill(~see.view(b, 1, 1, m, n), float("-inf"))
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(b * h, g * m, n), v.permute(0, 2, 1, 3).reshape(b * h, n, D)).view(b, h, g, m, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(b, m, hq, D)


def _plain_attention(st):
    case = st["case"]
    heads, D, page, rows = case["heads"], case["D"], case["page"], case["rows"]
    q, flat = st["q"], st["cache"].view(-1, st["cache"].shape[-1])
    out = torch.empty_like(q)
    if case["K"]:
        step = max(1, (1 << 25) // (case["K"] * heads * D))
        owner = torch.arange(len(st["ctx"]), device=DEV).repeat_interleave(rows)
        last = (st["ctx_len"].view(-1, 1) - rows + torch.arange(rows, device=DEV)).view(-1)
        for t in range(0, q.shape[0], step):
            sel = st["selection"][t:t + step]
            see = (sel >= 0) & (sel <= last[t:t + step].unsqueeze(1))
            idx = torch.where(see, sel, torch.zeros_like(sel)).long()
            pg = st["blocks"][owner[t:t + step].unsqueeze(1), idx // page].long().clamp(min=0)
            k, v = _unpacked(flat[pg * page + idx % page], heads, D)
            o = _attend(q[t:t + step].float().unsqueeze(1), k, v, see.unsqueeze(1), st["scale"])
            out[t:t + step] = o.squeeze(1).to(out.dtype)
        return out
    for b, c in enumerate(st["ctx"]):
        lo, m = st["starts"][b], st["nq"][b]
        if m == 0:
            continue
        if c == 0:
            out[lo:lo + m] = 0
            continue
        pages = st["blocks"][b, :(c + page - 1) // page].long()
        k, v = _unpacked(st["cache"][pages].view(-1, flat.shape[1])[:c], heads, D)
        t = torch.arange(c, device=DEV)
        step = max(1, (1 << 29) // (c * case["q_heads"]))
        for i in range(0, m, step):
            r = torch.arange(i, min(m, i + step), device=DEV)
            last = c - m + r if case["causal"] else torch.full_like(r, c - 1)
            o = _attend(q[lo + i:lo + i + r.numel()].float().unsqueeze(0), k.unsqueeze(0), v.unsqueeze(0),
                        (t <= last.unsqueeze(1)).unsqueeze(0), st["scale"])
            out[lo + i:lo + i + r.numel()] = o.squeeze(0).to(out.dtype)
    return out


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        if kind == "append":   # the cache's new records, as the values that they stand for
            state["append"]()
            return state["read"]()
        return state["call"]()
    if kind == "attention":
        return _plain_attention(state)
    if kind == "rope":
        y = _rotated(state["x"], state["table"], state["positions"], case["interleaved"], case["inverse"])
        return y.to(state["x"].dtype)
    flat = state["cache"].view(-1, state["cache"].shape[-1])
    k = _rotated(state["k"], state["table"], state["positions"], case["interleaved"], False)
    kc, ks = _quantised(k)
    vc, vs = _quantised(state["v"].float())
    slots = state["slots"]
    skipped = slots < 0
    at = torch.where(skipped, torch.full_like(slots, flat.shape[0] - 1), slots)   # into the page of no request
    flat[at] = torch.cat((kc, vc, ks, vs), dim=1)
    out = _unpacked(flat[at], case["heads"], case["D"])
    return tuple(x.masked_fill(skipped.view(-1, 1, 1), 0.0).to(state["k"].dtype) for x in out)


def _visible(case):
    """Query-key pairs, and tokens of the cache that some query of their request sees."""
    ctx, nq = _lengths(case)
    pairs = tokens = 0
    for c, m in zip(ctx, nq):
        if m == 0:
            continue
        if case["K"]:
            seen = [min(case["K"], max(0, c - m + 1 + i)) for i in range(m)]
            pairs += sum(seen)
            tokens += min(c, int(seen[-1] * (1 + 0.1 * (m - 1))))
        elif case["causal"]:
            pairs += sum(max(0, c - m + 1 + i) for i in range(m))
            tokens += c
        else:
            pairs += c * m
            tokens += c
    return pairs, tokens, sum(nq)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    heads, D = case["heads"], case["D"]
    if case["kind"] == "attention":
        pairs, tokens, rows = _visible(case)
        index = rows * case["K"] * 4 + tokens // case["page"] * 4
        return {"bytes": tokens * _record(heads, D) + 2 * rows * case["q_heads"] * D * size + index,
                "flops": 4 * pairs * case["q_heads"] * D}
    n, rot = case["tokens"], case["rot"]
    table = n * (rot * 4 + 4)
    if case["kind"] == "rope":
        return {"bytes": 2 * n * heads * D * size + table, "flops": 3 * n * heads * rot}
    # in: keys and values; out: their records; read again, and the values that they stand for
    return {"bytes": 4 * n * heads * D * size + 2 * n * _record(heads, D) + table + 16 * n,
            "flops": n * heads * (3 * rot + 8 * D)}


def _exact_value(code):
    mantissa, exponent = (code & 1).double(), (code >> 1) & 3
    size = torch.where(exponent == 0, 0.5 * mantissa, (1.0 + 0.5 * mantissa) * 2.0 ** (exponent - 1).double())
    return torch.where((code & 8) != 0, -size, size)


def _exact_part(rec, first, scales, D):
    """One head's keys or values [n][D] in float64: codes from byte `first`, scales from byte `scales`."""
    b = rec[:, first:first + D // 2].int()
    x = torch.stack((_exact_value(b % 16), _exact_value(b // 16)), dim=2).reshape(rec.shape[0], D)
    s = torch.pow(2.0, rec[:, scales:scales + D // BLOCK].double() - 127.0)
    return x * s.repeat_interleave(BLOCK, dim=1)


def _exact_attention(st):
    case = st["case"]
    heads, D, page, rows, group = case["heads"], case["D"], case["page"], case["rows"], case["q_heads"] // case["heads"]
    flat = st["cache"].view(-1, st["cache"].shape[-1])
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    jobs = []   # tokens of the cache, first query, queries, last visible token of each
    for b, c in enumerate(st["ctx"]):
        lo, m = st["starts"][b], st["nq"][b]
        last = torch.arange(m, device=DEV) + (c - m) if case["causal"] or case["K"] else \
            torch.full((m,), c - 1, device=DEV)
        if case["K"]:
            for i in range(m):
                sel = st["selection"][lo + i].long()
                jobs.append((b, sel[(sel >= 0) & (sel <= last[i])], lo + i, last[i:i + 1]))
        else:
            for i in range(0, m, 256):
                jobs.append((b, torch.arange(c, device=DEV), lo + i, last[i:i + 256]))
    kept = None
    for b, t, lo, last in jobs:
        if t.numel() == 0 or last.numel() == 0:
            continue
        m = last.numel()
        if case["K"] or kept is None or kept[0] != b:
            rec = flat[st["blocks"][b].long()[t // page] * page + t % page]
            kept = (b, rec)
        rec = kept[1]
        for h in range(heads):
            k = _exact_part(rec, h * D // 2, heads * D + h * D // BLOCK, D)
            v = _exact_part(rec, (heads + h) * D // 2, heads * D + (heads + h) * D // BLOCK, D)
            q = st["q"][lo:lo + m, h * group:(h + 1) * group].double().reshape(m * group, D)
            s = (q @ k.T * st["scale"]).view(m, group, -1)
            s = torch.where((t.view(1, 1, -1) <= last.view(m, 1, 1)), s, float("-inf"))
            w = torch.nan_to_num(torch.softmax(s, dim=-1), nan=0.0)
            out[lo:lo + m, h * group:(h + 1) * group] = (w.view(m * group, -1) @ v).view(m, group, D)
    return out


def _exact_turn(x, st, conjugate):
    case = st["case"]
    rot = case["rot"]
    turn = torch.view_as_complex(st["table"][st["positions"].long()].double()).unsqueeze(1)
    if conjugate:
        turn = turn.conj()
    y = x.double().clone()
    if case["interleaved"]:
        z = torch.view_as_complex(y[..., :rot].reshape(y.shape[0], y.shape[1], rot // 2, 2).contiguous()) * turn
        y[..., :rot] = torch.view_as_real(z).reshape(y.shape[0], y.shape[1], rot)
    else:
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def _exact_rounded(x):
    """x [n][heads][D] as the cache holds it: nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times the block's power of two."""
    blocks = x.reshape(x.shape[0], -1, BLOCK)
    top = blocks.abs().amax(dim=-1, keepdim=True)
    frac, exponent = torch.frexp(top / 7.0)
    unit = torch.pow(2.0, torch.where(frac > 0.5, exponent, exponent - 1).double().clamp(min=-126))
    y = blocks.abs() / unit
    step = torch.where(y < 2.0, 0.5, torch.where(y < 4.0, 1.0, 2.0))
    y = (torch.round(y / step) * step).clamp(max=6.0) * unit
    return torch.where(blocks < 0, -y, y).reshape(x.shape)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(st)
    if case["kind"] == "rope":
        return _exact_turn(st["x"], st, case["inverse"])
    skipped = (st["slots"] < 0).view(-1, 1, 1)
    k = _exact_rounded(_exact_turn(st["k"], st, False))
    v = _exact_rounded(st["v"].double())
    return tuple(x.masked_fill(skipped, 0.0) for x in (k, v))
