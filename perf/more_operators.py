"""Performance cases of what stands before a selected-token decode step: the
pages, slots and positions of a batch, 8-bit codes with a scale per 128
elements, products of such codes, and a linear layer made of them.

A serving program steps its page pool by the tokens that each request brings,
projects the hidden states in 8 bits, quantises the indexer's queries and keys
(rotated on the way, the keys into their cache); a training program runs the
same projections forward and backward.

A block's scale is its largest magnitude over 448 (at least 2^-126; rounded up to
a power of two with `pow2`), its codes are E4M3 of the elements times 448 over
that magnitude (over the scale with `pow2`), to the nearest, ties to even.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 128       # elements that share a scale
MOST = 448.0      # largest E4M3 value
LEAST = 2.0 ** -126
POSITIONS = 131072
ROPE_BASE = 10000.0
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
#: Most work of a drawn case: elements that are quantised, products summed up, tokens of a step's buffers.
MAX_ELEMS, MAX_PRODUCTS, MAX_TOKENS = 8192 * 4096, 8192 * 8192 * 4096, 131072


def _case(name, kind, base, kw):
    case = dict(base, kind=kind)
    case.update(kw)
    if name:
        case["name"] = name
    return case


def _heads(name, tokens, heads, D, **kw):
    return _case(name, "heads", {"tokens": tokens, "heads": heads, "D": D, "rot": 0, "dtype": "bf16", "pow2": False,
                                 "interleaved": False, "fused": False, "cache": 0}, kw)


def _matrix(name, rows, cols, **kw):
    return _case(name, "matrix", {"rows": rows, "cols": cols, "dtype": "bf16", "pow2": False, "square": False}, kw)


def _matmul(name, M, N, K, **kw):
    return _case(name, "matmul", {"M": M, "N": N, "K": K, "dtype": "bf16", "by_row": False}, kw)


def _linear(name, M, N, K, **kw):
    return _case(name, "linear", {"M": M, "N": N, "K": K, "dtype": "bf16", "weight": "bf16", "frozen": False}, kw)


def _pages(name, requests, ctx, new, tokens, **kw):
    return _case(name, "pages", {"requests": requests, "ctx": ctx, "new": new, "tokens": tokens, "page": 64,
                                 "ragged": False, "reject": 0, "short": False}, kw)


def listed():
    return [
        # one request's next indexer key into its cache: latency is everything
        _heads("quantize_key_b1", 1, 1, 128, rot=64, cache=1),
        # the benchmark's decode step (64 requests, two draft rows): the indexer's queries, half of each head rotated
        _heads("quantize_queries_b128", 128, 64, 128, rot=64, pow2=True),
        # a prompt's hidden states before a projection
        _heads("quantize_prompt_8k", 8192, 1, 4096),
        # training: an output's gradient in both directions, an odd number of tokens, float32
        _matrix("quantize_both_4099_f32", 4099, 4096, dtype="f32"),
        # one token through a projection: latency and the weights' bytes
        _matmul("matmul_m1", 1, 4096, 4096),
        # the benchmark's decode step through the indexer's query projection (64 heads of 128)
        _matmul("matmul_b128", 128, 8192, 4096),
        # odd sizes, a scale per row of both sides (a weight's gradient over 2117 tokens), float32
        _matmul("matmul_by_row_odd_f32", 1021, 1000, 2117, dtype="f32", by_row=True),
        # a prompt through the indexer's query projection
        _matmul("matmul_prompt_8k", 8192, 8192, 4096),
        # a training step of a square layer, bfloat16 weights
        _linear("linear_train_4k", 4096, 4096, 4096),
        # odd sizes, float32 weights and activations
        _linear("linear_train_odd_f32", 771, 1000, 531, dtype="f32", weight="f32"),
        # the benchmark's decode step: two draft tokens for each of 64 requests, of two before one was rejected
        _pages("pages_decode_b64", 64, 102400, 2, 128, reject=1),
        # prompts of mixed lengths beside running requests, small pages, padded buffers
        _pages("pages_prompts_b300", 300, 8192, 400, 131072, page=16, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["heads", "heads", "matrix", "matmul", "matmul", "matmul", "linear", "linear", "pages", "pages"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "heads":
        heads = rng.choice([1, 1, 3, 8, 32, 64])
        D = rng.choice([64, 128, 128, 192, 256]) if heads > 1 or rng.random() < 0.5 else _log_int(rng, 64, 8192)
        rot = rng.choice([0, 64, 32, 48]) if D <= 256 else 0
        return _heads(None, _log_int(rng, 1, min(16384, MAX_ELEMS // (heads * D))), heads, D, rot=rot, dtype=dtype,
                      pow2=rng.random() < 0.5, interleaved=rng.random() < 0.5, fused=rng.random() < 0.3,
                      cache=rng.choice([0, 0, 1, 2]) if D <= 256 else 0)
    if kind == "matrix":
        cols = _log_int(rng, 32, 8192)
        return _matrix(None, _log_int(rng, 1, min(8192, MAX_ELEMS // cols // 2)), cols, dtype=dtype,
                       pow2=rng.random() < 0.5, square=rng.random() < 0.5)
    if kind == "matmul":
        N, K = _log_int(rng, 16, 8192), _log_int(rng, 64, 8192)
        return _matmul(None, _log_int(rng, 1, min(8192, MAX_PRODUCTS // (N * K))), N, K, dtype=dtype,
                       by_row=rng.random() < 0.3)
    if kind == "linear":
        N, K = _log_int(rng, 16, 4096), _log_int(rng, 64, 4096)
        return _linear(None, _log_int(rng, 1, 4096), N, K, dtype=dtype, frozen=rng.random() < 0.3,
                       weight=dtype if rng.random() < 0.5 else "f32")
    requests = _log_int(rng, 1, 2048)
    page = rng.choice([16, 64, 128])
    new = rng.choice([1, 2, 4, _log_int(rng, 8, 2048)])
    most = max(1, min(131072, (1 << 22) * page // (2 * requests)))
    tokens = max(requests, min(MAX_TOKENS, int(requests * new * rng.choice([1.0, 1.0, 1.3, 0.8]))))
    return _pages(None, requests, _log_int(rng, 1, most), new, tokens, page=page, ragged=rng.random() < 0.6,
                  reject=rng.choice([0, 0, 1, 3]), short=rng.random() < 0.3)


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 71)
    return g


def _normal(shape, gen, dtype="f32", spread=0.0):
    """Unit normal values; `spread`: channels and rows of different sizes, as hidden states and gradients have."""
    x = torch.randn(shape, generator=gen, device=DEV)
    if spread:
        x = x * torch.exp(spread * torch.randn(shape[-1], generator=gen, device=DEV))
        x = x * torch.exp(spread * torch.randn(tuple(shape[:-1]) + (1,), generator=gen, device=DEV))
    return x.to(DTYPES[dtype])


def _codes(rows, cols, gen):
    """E4M3 codes as a quantised matrix holds them [rows][cols], each row's storage a multiple of 16 bytes."""
    wide = (cols + 15) // 16 * 16
    x = torch.randn((rows, wide), generator=gen, device=DEV).mul_(120.0).clamp_(-MOST, MOST)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)[:, :cols]


def _scales(rows, cols, gen):
    return torch.exp(0.5 * torch.randn((rows, cols), generator=gen, device=DEV)) / MOST


def _prepare_heads(case, gen):
    n, heads, D = case["tokens"], case["heads"], case["D"]
    # of a fused projection: two more heads behind these
    wide = heads + 2 if case["fused"] else heads
    st = {"x": _normal((n, wide, D), gen, case["dtype"], 0.7)[:, :heads], "table": None, "positions": None, "slots": None,
          "codes": None, "scale": None}
    if case["rot"]:
        half = case["rot"] // 2
        rate = ROPE_BASE ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        phase = torch.arange(POSITIONS, dtype=torch.float64, device=DEV).unsqueeze(1) * rate
        st["table"] = torch.stack((torch.cos(phase), torch.sin(phase)), dim=-1).float().contiguous()
        st["positions"] = torch.randint(0, POSITIONS, (n,), generator=gen, device=DEV).to(torch.int32)
    if case["cache"]:   # rows of a cache, some tokens padded away with 2
        rows = 2 * n + 3
        slots = torch.randperm(rows - 1, generator=gen, device=DEV)[:n]
        if case["cache"] == 2:
            slots = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.1, -1, slots)
        st["slots"] = slots.contiguous()
        st["codes"] = torch.zeros((rows, heads, D), dtype=torch.uint8, device=DEV)
        st["scale"] = torch.ones((rows, heads, (D + BLOCK - 1) // BLOCK), device=DEV)
    if own:
        import paper_2604_22312_amd as gvr
        st["call"] = gvr.prepare_gvr_fp8_quantize(st["x"], table=st["table"], positions=st["positions"],
                                                  interleaved=case["interleaved"], pow2=case["pow2"], slots=st["slots"],
                                                  codes=st["codes"], scale=st["scale"])
    return st


def _lengths(case):
    """Tokens held, brought and taken back by each request, the same for every seed."""
    R, rng = case["requests"], random.Random(case["requests"] * 1000003 + case["ctx"])
    ctx, new = [case["ctx"]] * R, [case["new"]] * R
    if case["ragged"]:
        # one request of eight not started, one of sixteen brings nothing
        ctx = [0 if rng.random() < 0.125 else rng.randint(1, case["ctx"]) for _ in range(R)]
        new = [0 if rng.random() < 0.0625 else rng.randint(1, 2 * case["new"]) for _ in range(R)]
    back = [min(c, rng.randint(0, case["reject"])) if case["reject"] else 0 for c in ctx]
    return ctx, new, back


def _page_counts(case):
    P = case["page"]
    ctx, new, back = _lengths(case)
    held = [(c + P - 1) // P for c in ctx]
    want = [(c - b + n + P - 1) // P for c, b, n in zip(ctx, back, new)]
    return held, want


def _prepare_pages(case, gen):
    R, P = case["requests"], case["page"]
    ctx, new, back = _lengths(case)
    held, want = _page_counts(case)
    more = sum(max(0, w - h) for w, h in zip(want, held))
    free = more // 2 if case["short"] else more + 7
    pages = sum(held) + free
    width = max(max(held), max(want), 1)
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    counts = torch.tensor(held, device=DEV)
    first = torch.cumsum(counts, 0) - counts
    col = torch.arange(width, device=DEV)
    at = (first.unsqueeze(1) + col).clamp(max=max(pages - 1, 0))
    table = torch.where(col < counts.unsqueeze(1), order[at], torch.full_like(at, -1, dtype=torch.int32))
    stack = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
    stack[:free] = order[sum(held):]
    ints = dict(dtype=torch.int32, device=DEV)
    st = {"table": table.contiguous(), "len": torch.tensor(ctx, **ints), "free": stack,
          "count": torch.tensor([free], **ints), "new": torch.tensor(new, **ints),
          "keep": torch.tensor([c - b for c, b in zip(ctx, back)], **ints), "back": torch.tensor(back, **ints),
          "ld": max(ctx) + 2 * case["new"], "T": case["tokens"], "T_back": max(1, sum(back))}
    if own:
        import paper_2604_22312_amd as gvr
        pool = gvr.PagePool(st["table"], st["len"], st["free"], st["count"], P)
        st["step"] = gvr.prepare_gvr_page_step(pool, st["new"], st["T"], keep=st["keep"], ld=st["ld"])
        st["undo"] = gvr.prepare_gvr_page_step(pool, st["back"], st["T_back"], keep=st["keep"], ld=st["ld"])
    return st


def prepare(case, seed):
    gen, kind = _generator(seed), case["kind"]
    if kind == "heads":
        st = _prepare_heads(case, gen)
    elif kind == "matrix":
        st = {"x": _normal((case["rows"], case["cols"]), gen, case["dtype"], 0.7)}
        if own:
            import paper_2604_22312_amd as gvr
            st["call"] = gvr.prepare_gvr_fp8_quantize_matrix(st["x"], square=case["square"], transposed=True,
                                                             pow2=case["pow2"])
    elif kind == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        blocks = (K + BLOCK - 1) // BLOCK
        st = {"a": _codes(M, K, gen), "a_scale": _scales(M, blocks, gen), "b": _codes(N, K, gen),
              "b_scale": _scales(N if case["by_row"] else (N + BLOCK - 1) // BLOCK, blocks, gen)}
        if own:
            import paper_2604_22312_amd as gvr
            st["call"] = gvr.prepare_gvr_fp8_matmul(st["a"], st["a_scale"], st["b"], st["b_scale"],
                                                    dtype=DTYPES[case["dtype"]])
    elif kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        st = {"x": _normal((M, K), gen, case["dtype"], 0.7).requires_grad_(),
              "w": (torch.randn((N, K), generator=gen, device=DEV) / math.sqrt(K)).to(DTYPES[case["weight"]]),
              "dy": (1e-3 * _normal((M, N), gen, "f32", 0.7)).to(DTYPES[case["dtype"]])}
        if not case["frozen"]:
            st["w"].requires_grad_()
        elif own:   # a frozen layer keeps its codes and not the weights
            import paper_2604_22312_amd as gvr
            st["frozen"] = gvr.gvr_fp8_quantize_matrix(st["w"], square=True, transposed=True)
    else:
        st = _prepare_pages(case, gen)
    st["case"] = case
    return st


def _rotated(x, table, positions, interleaved):
    """x [n][heads][D] in float32 with its first 2 * table.shape[1] elements rotated."""
    rot = 2 * table.shape[1]
    cs = table[positions.long()].unsqueeze(1)
    c, s = cs[..., 0], cs[..., 1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * c - b * s, b * c + a * s
    turned = torch.stack((ra, rb), dim=-1).flatten(-2) if interleaved else torch.cat((ra, rb), dim=-1)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def _padded(x, axis):
    """x with zeros up to a multiple of BLOCK along `axis` (-1 or -2)."""
    more = -x.shape[axis] % BLOCK
    return torch.nn.functional.pad(x, (0, more) if axis == -1 else (0, 0, 0, more)) if more else x


def _scale_of(top, pow2):
    """Scale of blocks whose largest magnitudes are `top`, and the magnitude that its code 448 stands for."""
    top = top.clamp(min=MOST * LEAST)
    if not pow2:
        return top / MOST, top
    frac, exponent = torch.frexp(top / MOST)
    scale = torch.ldexp(torch.ones_like(top), torch.where(frac > 0.5, exponent, exponent - 1))
    return scale, MOST * scale


def _e4m3(x, full):
    """Codes of 448 x / full; in float64, as the quotients of short numbers often lie on the border of two codes."""
    y = x.double() * MOST / full.double()
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return (torch.round(y / step) * step).to(torch.float8_e4m3fn)


def _quantised(x, pow2, square=False):
    """Codes and scales of x [...][C] in float32 by blocks along the last axis (128 x 128 with `square`)."""
    C, R = x.shape[-1], x.shape[-2]
    y = _padded(x, -1)
    y = y.reshape(y.shape[:-1] + (-1, BLOCK))
    top = y.abs().amax(dim=-1)
    if square:
        t = _padded(top, -2)
        t = t.view(-1, BLOCK, t.shape[-1]).amax(dim=1)
        scale, full = _scale_of(t, pow2)
        full = full.repeat_interleave(BLOCK, dim=0)[:R]
    else:
        scale, full = _scale_of(top, pow2)
    return _e4m3(y, full.unsqueeze(-1)).flatten(-2)[..., :C], scale


def _values(codes, scale, square=False):
    """What codes [R][C] and their scales stand for, in float32."""
    R, C = codes.shape
    s = scale.repeat_interleave(BLOCK, dim=1)[:, :C]
    return codes.float() * (s.repeat_interleave(BLOCK, dim=0)[:R] if square else s)


def _plain_pages(st, T, new):
    """One step of the pool: truncate to `keep`, add `new`; rows of the T tokens."""
    P, R, W = st["case"]["page"], st["len"].shape[0], st["table"].shape[1]
    ctx, n = st["len"].long(), new.long().clamp(min=0)
    keep = torch.minimum(st["keep"].long().clamp(min=0), ctx)
    count = st["count"].long()
    start = torch.cumsum(n, 0) - n
    held, want = (ctx + P - 1) // P, (keep + n + P - 1) // P
    fits = (start + n <= T) & (want <= W)
    need = torch.where(fits, (want - held).clamp(min=0), 0)
    total = torch.cumsum(need, 0)
    served = fits & ((need == 0) | (total <= count))
    after = torch.where(served, keep + n, keep)
    have = (after + P - 1) // P
    taken = torch.where(served, n, 0)
    # pages taken from the top of the stack, freed ones pushed in their place, the first on top
    col = torch.arange(W, device=DEV)
    gets = (col >= held.unsqueeze(1)) & (col < have.unsqueeze(1))
    loses = (col >= have.unsqueeze(1)) & (col < held.unsqueeze(1))
    g = torch.cumsum(gets.view(-1).long(), 0)
    f = torch.cumsum(loses.view(-1).long(), 0)
    top = count - g[-1:]
    pages = st["free"].shape[0]
    page = st["free"][(count - g).clamp(0, max(pages - 1, 0))].view(R, W)
    end = top + f[-1:]
    at = torch.where(loses.view(-1), end - f, pages)
    stack = torch.cat((st["free"], st["free"][:1])).scatter(0, at, st["table"].view(-1))
    st["free"].copy_(stack[:pages])
    st["table"].copy_(torch.where(gets, page, torch.where(loses, -1, st["table"])))
    st["len"].copy_(after)
    st["count"].copy_(end)
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(start + n, t, right=True).clamp(max=R - 1)
    there = (t < start[-1] + n[-1]) & served[r]
    pos = torch.where(there, keep[r] + t - start[r], 0)
    slot = st["table"][r, torch.where(there, pos // P, 0)].long() * P + pos % P
    return {"q_start": torch.cat((start, start[-1:] + n[-1:])).clamp(max=T).int(), "taken": taken.int(),
            "positions": pos.int(), "slots": torch.where(there, slot, -1), "dense": torch.where(there, r * st["ld"] + pos, -1),
            "row_len": torch.where(there, pos + 1, 0).int()}


def _plain_heads(st):
    case, x = st["case"], st["x"].float()
    if st["table"] is not None:
        x = _rotated(x, st["table"], st["positions"], case["interleaved"])
    codes, scale = _quantised(x, case["pow2"])
    if st["slots"] is None:
        return codes, scale
    rows = st["codes"].shape[0]
    at = torch.where(st["slots"] < 0, rows - 1, st["slots"])   # padded tokens into the row of nobody, then cleared
    st["codes"][at], st["scale"][at] = codes.view(torch.uint8), scale
    st["codes"][rows - 1:], st["scale"][rows - 1:] = 0, 1.0
    return st["codes"].view(torch.float8_e4m3fn), st["scale"]


def _plain_linear(st):
    x, w, dy = (st[k].detach().float() for k in ("x", "w", "dy"))
    qw = _values(*_quantised(w, False, square=True), square=True)
    y = torch.matmul(_values(*_quantised(x, False)), qw.T)
    dx = torch.matmul(_values(*_quantised(dy, False)), qw)
    out = [y.to(st["x"].dtype), dx.to(st["x"].dtype)]
    if not st["case"]["frozen"]:
        dw = torch.matmul(_values(*_quantised(dy.T, False)), _values(*_quantised(x.T, False)).T)
        out.append(dw.to(st["w"].dtype))
    return out


def _own_linear(st):
    import paper_2604_22312_amd as gvr
    if st["case"]["frozen"]:
        y = gvr.gvr_fp8_linear(st["x"], st["frozen"][0], st["frozen"][1])
        return [y.detach(), *torch.autograd.grad(y, (st["x"],), st["dy"])]
    y = gvr.gvr_fp8_linear(st["x"], st["w"])
    return [y.detach(), *torch.autograd.grad(y, (st["x"], st["w"]), st["dy"])]


def run(state):
    case = state["case"]
    kind, e4m3 = case["kind"], torch.float8_e4m3fn
    if kind == "linear":
        return _own_linear(state) if own else _plain_linear(state)
    if kind == "pages":   # a step, and the step that takes it back
        if own:
            got = state["step"]()._asdict()
            state["undo"]()
        else:
            got = _plain_pages(state, state["T"], state["new"])
            _plain_pages(state, state["T_back"], state["back"])
        return dict(got, table=state["table"], len=state["len"], free=state["free"], count=state["count"])
    if kind == "matmul":
        if own:
            return state["call"]()
        square = not case["by_row"]
        a = _values(state["a"].view(e4m3), state["a_scale"])
        b = _values(state["b"].view(e4m3), state["b_scale"], square)
        return torch.matmul(a, b.T).to(DTYPES[case["dtype"]])
    if kind == "heads":
        if own:
            codes, scale = state["call"]()
            return codes.view(e4m3), scale
        return _plain_heads(state)
    if own:
        straight, transposed = state["call"]()
        return straight.codes.view(e4m3), straight.scale, transposed.codes.view(e4m3), transposed.scale
    x = state["x"].float()
    codes, scale = _quantised(x, case["pow2"], case["square"])
    if case["square"]:
        return codes, scale, codes.T.contiguous(), scale.T.contiguous()
    turned, turned_scale = _quantised(x.T, case["pow2"])
    return codes, scale, turned, turned_scale


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def work(case):
    kind = case["kind"]
    if kind == "pages":
        held, want = _page_counts(case)
        moved = sum(abs(w - h) for w, h in zip(want, held))
        # each step: lengths in and out, a page number moved once each way, four numbers for every token
        rows = case["tokens"] + max(1, sum(_lengths(case)[2]))
        return {"bytes": 2 * 24 * case["requests"] + 16 * moved + 24 * rows, "flops": 0}
    size = 4 if case["dtype"] == "f32" else 2
    if kind == "heads":
        n, H, D = case["tokens"], case["heads"], case["D"]
        at = (case["rot"] * 4 + 4 if case["rot"] else 0) + (8 if case["cache"] else 0)
        return {"bytes": n * H * (D * (size + 1) + 4 * _blocks(D)) + n * at, "flops": n * H * (2 * D + 3 * case["rot"])}
    if kind == "matrix":
        R, C = case["rows"], case["cols"]
        scales = 2 * _blocks(R) * _blocks(C) if case["square"] else R * _blocks(C) + C * _blocks(R)
        return {"bytes": R * C * (size + 2) + 4 * scales, "flops": 4 * R * C}
    M, N, K = case["M"], case["N"], case["K"]
    if kind == "matmul":
        scales = (M + (N if case["by_row"] else _blocks(N))) * _blocks(K)
        return {"bytes": M * K + N * K + 4 * scales + M * N * size, "flops": 2 * M * N * K}
    wide = 4 if case["weight"] == "f32" else 2
    if case["frozen"]:   # the weight's codes once for each product
        return {"bytes": 2 * size * (M * K + M * N) + 2 * N * K, "flops": 4 * M * N * K}
    return {"bytes": 2 * size * (M * K + M * N) + 2 * wide * N * K, "flops": 6 * M * N * K}


def _exact_codes(x, pow2, tall):
    """Codes, scales and the values they stand for, in float64, of x [R][C] by blocks of `tall` rows and 128 columns."""
    R, C = x.shape
    rows, cols = -(-R // tall), _blocks(C)
    full = torch.zeros((rows * tall, cols * BLOCK), dtype=torch.float64, device=DEV)
    full[:R, :C] = x
    tiles = full.view(rows, tall, cols, BLOCK)
    top = torch.maximum(tiles.abs().amax(dim=(1, 3)), torch.tensor(448.0 * 2.0 ** -126, dtype=torch.float64, device=DEV))
    scale = torch.pow(2.0, torch.ceil(torch.log2(top / 448.0))) if pow2 else top / 448.0
    units = tiles * 448.0 / (448.0 * scale if pow2 else top).view(rows, 1, cols, 1)   # (a tie stays one)
    # three bits behind the leading one, steps of 2^-9 under 2^-6
    step = torch.pow(2.0, torch.floor(torch.log2(units.abs().clamp(min=2.0 ** -6))) - 3.0)
    codes = (torch.round(units / step) * step).clamp(-448.0, 448.0)
    values = (codes * scale.view(rows, 1, cols, 1)).view(rows * tall, cols * BLOCK)[:R, :C]
    return codes.view(rows * tall, cols * BLOCK)[:R, :C], scale, values


def _exact_heads(st):
    case = st["case"]
    n, H, D = st["x"].shape
    x = st["x"].double()
    rot = case["rot"]
    if rot:
        turn = torch.view_as_complex(st["table"][st["positions"].long()].double()).unsqueeze(1)
        if case["interleaved"]:
            z = torch.view_as_complex(x[..., :rot].reshape(n, H, rot // 2, 2).contiguous()) * turn
            front = torch.view_as_real(z).reshape(n, H, rot)
        else:
            z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
            front = torch.cat((z.real, z.imag), dim=-1)
        x = torch.cat((front, x[..., rot:]), dim=-1)
    codes, scale, _ = _exact_codes(x.reshape(n * H, D), case["pow2"], 1)
    codes, scale = codes.reshape(n, H, D), scale.reshape(n, H, -1)
    if st["slots"] is None:
        return codes, scale
    there = st["slots"] >= 0
    whole = st["codes"].double().zero_(), st["scale"].double().fill_(1.0)
    whole[0][st["slots"][there]], whole[1][st["slots"][there]] = codes[there], scale[there]
    return whole


def exact(case, seed):
    kind = case["kind"]
    if kind == "pages":
        return None   # whole numbers
    st = prepare(case, seed)
    if kind == "heads":
        return _exact_heads(st)
    if kind == "matrix":
        x = st["x"].double()
        tall = BLOCK if case["square"] else 1
        codes, scale, _ = _exact_codes(x, case["pow2"], tall)
        turned, turned_scale, _ = _exact_codes(x.T.contiguous(), case["pow2"], tall)
        return codes, scale, turned, turned_scale
    if kind == "matmul":
        K, N = case["K"], case["N"]
        out = torch.zeros((case["M"], N), dtype=torch.float64, device=DEV)
        for i in range(_blocks(K)):
            a, b = (st[k][:, i * BLOCK:min(K, (i + 1) * BLOCK)].contiguous().view(torch.float8_e4m3fn).double() for k in "ab")
            by = st["b_scale"][:, i].double()
            by = by if case["by_row"] else by[torch.arange(N, device=DEV) // BLOCK]
            out += (a @ b.T.contiguous()) * st["a_scale"][:, i].double().unsqueeze(1) * by
        return out
    x, w, dy = (st[k].detach().double() for k in ("x", "w", "dy"))
    qw = _exact_codes(w, False, BLOCK)[2]
    y = _exact_codes(x, False, 1)[2] @ qw.T.contiguous()
    dx = _exact_codes(dy, False, 1)[2] @ qw
    if case["frozen"]:
        return [y, dx]
    return [y, dx, _exact_codes(dy.T.contiguous(), False, 1)[2] @ _exact_codes(x.T.contiguous(), False, 1)[2].T.contiguous()]
