"""ctypes marshalling for the rotary positions and the 4-bit key / value cache
(``include/gvr_rotary.h``, ``include/gvr_kv4.h``): argument checks and
pointers only; the kernels are in ``csrc/rotary.hip``, ``csrc/kv4_cache.hip``
and ``csrc/kv4_attention.hip``. There is no CPU path."""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import GvrError, PreparedCall, RopeParams, _new, _on_device, _ptr, _rope_args, _stream

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
ROPE_INTERLEAVED, ROPE_TRANSPOSED = 1, 2

_ready = False


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _RopeCs(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("positions", ctypes.c_int64), ("rot", ctypes.c_int32),
                ("flags", ctypes.c_int32)]


class _Cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _AttentionArgs(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
                ("ctx_len", ctypes.c_void_p), ("q_start", ctypes.c_void_p), ("selection", ctypes.c_void_p),
                ("T", ctypes.c_int64), ("table_width", ctypes.c_int64), ("sequences", ctypes.c_int32),
                ("max_q", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("K", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


def lib():
    """The library, with this module's entry points declared."""
    global _ready
    L = binding.lib()
    if not _ready:
        vp, i64, i32, p = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER
        L.gvr_rope_table.argtypes = [i64, p(RopeParams), ctypes.c_double, vp, vp]
        L.gvr_rope_rotate.argtypes = [p(_Heads), p(_Heads), i32, i64, i32, i32, vp, p(_RopeCs), vp]
        L.gvr_kv4_record_bytes.argtypes = [i32, i32]
        L.gvr_kv4_append.argtypes = [p(_Cache), p(_Heads), p(_Heads), i32, i64, vp, vp, p(_RopeCs), vp]
        L.gvr_kv4_read.argtypes = [p(_Cache), p(_Heads), p(_Heads), i32, i64, vp, vp]
        L.gvr_kv4_attention_workspace.argtypes = [p(_Cache), p(_AttentionArgs), p(ctypes.c_size_t)]
        L.gvr_kv4_attention.argtypes = [p(_Cache), p(_AttentionArgs), vp, ctypes.c_size_t, vp]
        for name in ("gvr_rope_table", "gvr_rope_rotate", "gvr_kv4_append", "gvr_kv4_read",
                     "gvr_kv4_attention_workspace", "gvr_kv4_attention"):
            getattr(L, name).restype = ctypes.c_int
        L.gvr_kv4_record_bytes.restype = ctypes.c_int64
        _ready = True
    return L


class PreparedOp(PreparedCall):
    """A ``PreparedCall`` of one of this module's operators; calling it
    enqueues the operator again and returns its output(s), also in ``out``."""
    __slots__ = ()

    @property
    def out(self):
        return self.out_idx


def _prepared(name, dev, args, out, keep):
    pc = PreparedOp()
    pc._name, pc._f, pc._args, pc.out_idx, pc._keep = name, getattr(lib(), name), args, out, keep
    pc._dev = dev.index if dev.index is not None else torch.cuda.current_device()
    return pc


def _need(cond, text):
    if not cond:
        raise ValueError(text)


def _heads_tensor(t, name, dtype=None, shape=None, dev=None):
    _need(isinstance(t, torch.Tensor) and t.dim() == 3 and t.dtype in DTYPES,
          "%s must be a bfloat16, float16 or float32 tensor [T][heads][D]" % name)
    _need(t.is_cuda, "%s must be on a GPU (there is no CPU path)" % name)
    _need(t.shape[2] == 0 or t.stride(2) == 1 or t.shape[2] == 1, "%s: a head's elements must be contiguous" % name)
    _need(dtype is None or t.dtype == dtype, "%s must be %s" % (name, dtype))
    _need(shape is None or tuple(t.shape) == tuple(shape), "%s must be %s" % (name, list(shape or ())))
    _need(dev is None or t.device == dev, "%s must be on %s" % (name, dev))
    return _Heads(t.data_ptr(), t.stride(0), t.stride(1))


def _no_overlap(t, name):
    """Every element of a written tensor has a place of its own."""
    reach = 1
    for size, stride in sorted(((t.shape[d], t.stride(d)) for d in range(t.dim())), key=lambda x: x[1]):
        if size > 1:
            _need(stride >= reach, "%s: two of its elements share a place" % name)
            reach = stride * (size - 1) + reach
    return t


def _index(t, name, dtype, shape, dev):
    _need(isinstance(t, torch.Tensor) and t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.device == dev
          and t.is_contiguous(), "%s must be a contiguous %s tensor %s on %s" % (name, dtype, list(shape), dev))


def _cs(table, interleaved, transposed, D, dev):
    _need(isinstance(table, torch.Tensor) and table.dtype == torch.float32 and table.dim() == 3 and table.shape[2] == 2
          and table.device == dev and table.is_contiguous(),
          "table must be a contiguous float32 tensor [positions][rot / 2][2] on %s" % dev)
    _need(1 <= table.shape[1] and 2 * table.shape[1] <= min(D, 512), "table rotates more elements than a head has")
    return _RopeCs(table.data_ptr(), table.shape[0], 2 * table.shape[1],
                   (ROPE_INTERLEAVED if interleaved else 0) | (ROPE_TRANSPOSED if transposed else 0))


def gvr_rope_table(n, params=None, gain=1.0, device="cuda", out=None, stream=None):
    """Cosines and sines [n][d_rope / 2][2] (float32) of the positions 0 .. n-1
    under ``params`` (as ``gvr_rope_prior``), times ``gain``."""
    params, dev = _rope_args(params, device)
    n = int(n)
    shape = (max(n, 0), max(params.d_rope, 0) // 2, 2)
    if out is None:
        out = _new(shape, torch.float32, dev, stream)
    else:
        _index(out, "out", torch.float32, shape, dev)
    with _on_device(dev):
        st = lib().gvr_rope_table(n, ctypes.byref(params), float(gain), _ptr(out), _stream(stream, dev))
    if st != 0:
        raise GvrError("gvr_rope_table", st)
    return out


def prepare_gvr_rope_rotate(x, positions, table, interleaved=False, inverse=False, out=None, stream=None):
    """A ``PreparedOp`` of ``gvr_rope_rotate``. Its calls write the same tensor
    again and are not seen by autograd."""
    xs = _heads_tensor(x, "x")
    T, H, D = x.shape
    dev = x.device
    _need(1 <= D <= 1024, "a head has 1 .. 1024 elements")
    _index(positions, "positions", torch.int32, (T,), dev)
    cs = _cs(table, interleaved, inverse, D, dev)
    if out is None:
        out = _new((T, H, D), x.dtype, dev, stream)
    os = _heads_tensor(_no_overlap(out, "out"), "out", x.dtype, x.shape, dev)
    args = (ctypes.byref(xs), ctypes.byref(os), DTYPES[x.dtype], T, H, D, _ptr(positions), ctypes.byref(cs),
            _stream(stream, dev))
    return _prepared("gvr_rope_rotate", dev, args, out, (x, positions, table, xs, os, cs, stream))


class _Rotate(torch.autograd.Function):
    """The rotation as a node of the graph; ``out`` (x itself or another tensor)
    is written in place. Linear, so its gradient is the transposed rotation."""

    @staticmethod
    def forward(ctx, x, out, positions, table, interleaved, inverse, stream):
        ctx.save_for_backward(positions, table)
        ctx.how = (interleaved, not inverse)
        if out is not None:
            ctx.mark_dirty(out)
        return prepare_gvr_rope_rotate(x, positions, table, interleaved, inverse, out, stream)()

    @staticmethod
    def backward(ctx, grad):
        positions, table = ctx.saved_tensors
        grad = grad if grad.stride(2) == 1 else grad.contiguous()   # (a sum's gradient is one element)
        return (gvr_rope_rotate(grad, positions, table, *ctx.how),) + (None,) * 6


class _RotateInPlace(_Rotate):
    @staticmethod
    def forward(ctx, x, positions, table, interleaved, inverse, stream):
        return _Rotate.forward(ctx, x, x, positions, table, interleaved, inverse, stream)

    @staticmethod
    def backward(ctx, grad):
        return _Rotate.backward(ctx, grad)[:6]


def gvr_rope_rotate(x, positions, table, interleaved=False, inverse=False, out=None, stream=None):
    """x [T][H][D] (bfloat16, float16 or float32; any token and head stride)
    with the first 2 * table.shape[1] elements of each head rotated to its
    token's position (int32 [T]). ``interleaved``: pairs (2i, 2i+1) instead of
    (i, i + rot/2). ``inverse``: the transposed rotation, which takes the
    gradient of the result to the gradient of x. ``out`` may be ``x``. While
    gradients are recorded the call is a node of x's graph (the table gets no
    gradient)."""
    if torch.is_grad_enabled() and isinstance(x, torch.Tensor) and (x.requires_grad or getattr(out, "requires_grad", False)):
        _need(not isinstance(out, torch.Tensor) or not (out.is_leaf and out.requires_grad),
              "out is a leaf that requires a gradient: write into it under torch.no_grad()")
        if out is x:
            return _RotateInPlace.apply(x, positions, table, interleaved, inverse, stream)
        return _Rotate.apply(x, out, positions, table, interleaved, inverse, stream)
    y = prepare_gvr_rope_rotate(x, positions, table, interleaved, inverse, out, stream)()
    if out is not None and not out.is_inference():
        torch.autograd.graph.increment_version(out)   # (a graph may have saved it)
    return y


def gvr_kv4_record_bytes(kv_heads, head_dim) -> int:
    """Bytes of one token in the 4-bit cache."""
    n = int(lib().gvr_kv4_record_bytes(int(kv_heads), int(head_dim)))
    _need(n > 0, "kv_heads 1 .. 1024 and head_dim 64, 128 or 256")
    return n


def new_kv4_cache(pages, page_size, kv_heads, head_dim, device="cuda"):
    """A zeroed cache: uint8 [pages][page_size][record] (every value zero)."""
    return torch.zeros((int(pages), int(page_size), gvr_kv4_record_bytes(kv_heads, head_dim)), dtype=torch.uint8,
                       device=device)


def _cache(cache, kv_heads, head_dim):
    record = gvr_kv4_record_bytes(kv_heads, head_dim)
    _need(isinstance(cache, torch.Tensor) and cache.dtype == torch.uint8 and cache.dim() == 3 and cache.is_contiguous()
          and cache.shape[2] == record, "cache must be a contiguous uint8 tensor [pages][page_size][%d]" % record)
    _need(cache.is_cuda, "cache must be on a GPU (there is no CPU path)")
    page = cache.shape[1]
    _need(1 <= page <= 65536 and page & (page - 1) == 0, "the page size must be a power of two up to 65536")
    return _Cache(cache.data_ptr(), cache.shape[0], page, int(kv_heads), int(head_dim), 0)


def prepare_gvr_kv4_append(k, v, slots, cache, table=None, positions=None, interleaved=False, stream=None):
    """A ``PreparedOp`` of ``gvr_kv4_append``."""
    ks = _heads_tensor(k, "k")
    T, H, D = k.shape
    dev = k.device
    vs = _heads_tensor(v, "v", k.dtype, k.shape, dev)
    _index(slots, "slots", torch.int64, (T,), dev)
    c = _cache(cache, H, D)
    _need(cache.device == dev, "cache must be on %s" % dev)
    cs = None
    if table is not None:
        cs = _cs(table, interleaved, False, D, dev)
        _index(positions, "positions", torch.int32, (T,), dev)
    else:
        _need(positions is None, "positions need a table")
    args = (ctypes.byref(c), ctypes.byref(ks), ctypes.byref(vs), DTYPES[k.dtype], T, _ptr(slots),
            _ptr(positions), ctypes.byref(cs) if cs is not None else None, _stream(stream, dev))
    return _prepared("gvr_kv4_append", dev, args, cache, (k, v, slots, positions, table, c, ks, vs, cs, stream))


def gvr_kv4_append(k, v, slots, cache, table=None, positions=None, interleaved=False, stream=None):
    """Write k and v [T][kv_heads][head_dim] into ``cache`` at ``slots``
    (int64 [T]: page * page_size + place; -1 skips the token), the keys rotated
    by ``table`` at ``positions`` (int32 [T]) on the way; returns ``cache``."""
    return prepare_gvr_kv4_append(k, v, slots, cache, table, positions, interleaved, stream)()


def prepare_gvr_kv4_read(cache, slots, kv_heads, head_dim, dtype=torch.bfloat16, k=None, v=None, stream=None):
    """A ``PreparedOp`` of ``gvr_kv4_read``."""
    c = _cache(cache, kv_heads, head_dim)
    dev = cache.device
    _need(dtype in DTYPES, "dtype must be bfloat16, float16 or float32")
    _need(isinstance(slots, torch.Tensor) and slots.dim() == 1, "slots must be an int64 tensor [T]")
    T = slots.shape[0]
    _index(slots, "slots", torch.int64, (T,), dev)
    shape = (T, c.kv_heads, c.head_dim)
    k = _new(shape, dtype, dev, stream) if k is None else k
    v = _new(shape, dtype, dev, stream) if v is None else v
    ks = _heads_tensor(_no_overlap(k, "k"), "k", dtype, shape, dev)
    vs = _heads_tensor(_no_overlap(v, "v"), "v", dtype, shape, dev)
    args = (ctypes.byref(c), ctypes.byref(ks), ctypes.byref(vs), DTYPES[dtype], T, _ptr(slots), _stream(stream, dev))
    return _prepared("gvr_kv4_read", dev, args, (k, v), (cache, slots, c, ks, vs, stream))


def gvr_kv4_read(cache, slots, kv_heads, head_dim, dtype=torch.bfloat16, k=None, v=None, stream=None):
    """The keys and values [T][kv_heads][head_dim] that the records at
    ``slots`` stand for; zeros for a slot outside the cache."""
    return prepare_gvr_kv4_read(cache, slots, kv_heads, head_dim, dtype, k, v, stream)()


def _attention_args(q, cache, block_table, ctx_len, kv_heads, selection, q_start, max_q, causal, scale, out, lse,
                    stream=None):
    _heads_tensor(q, "q")
    _need(q.dtype != torch.float32, "q must be bfloat16 or float16")
    T, H, D = q.shape
    dev = q.device
    c = _cache(cache, kv_heads, D)
    _need(cache.device == dev, "cache must be on %s" % dev)
    _need(H % c.kv_heads == 0 and 1 <= H // c.kv_heads <= 128, "query heads must be 1 .. 128 times the KV heads")
    _need(q.data_ptr() % 16 == 0 and q.stride(0) % 8 == 0 and q.stride(1) % 8 == 0,
          "q: heads must start 16-byte aligned")
    _need(isinstance(block_table, torch.Tensor) and block_table.dim() == 2, "block_table must be int32 [sequences][pages]")
    B = block_table.shape[0]
    _index(block_table, "block_table", torch.int32, tuple(block_table.shape), dev)
    _index(ctx_len, "ctx_len", torch.int32, (B,), dev)
    if q_start is not None:
        _index(q_start, "q_start", torch.int32, (B + 1,), dev)
        max_q = T if max_q is None else int(max_q)
        _need(0 <= max_q, "max_q must not be negative")
        max_q = min(max_q, T)   # (an int32 in the C call)
    else:
        _need(T % B == 0 if B else T == 0, "without q_start every sequence has as many query tokens")
        max_q = T // B if B else 0
    K = 0
    if selection is not None:
        _need(isinstance(selection, torch.Tensor) and selection.dim() == 2 and selection.shape[1] >= 1,
              "selection must be int32 [T][K]")
        K = selection.shape[1]
        _index(selection, "selection", torch.int32, (T, K), dev)
    if out is None:
        out = _new((T, H, D), q.dtype, dev, stream)
    else:
        _index(out, "out", q.dtype, (T, H, D), dev)
    if lse is not None:
        _index(lse, "lse", torch.float32, (T, H), dev)
    scale = D ** -0.5 if scale is None else float(scale)
    _need(scale == scale and abs(scale) < 3e38, "scale must be finite")
    a = _AttentionArgs(q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(), lse.data_ptr() if lse is not None else None,
                       block_table.data_ptr(), ctx_len.data_ptr(), q_start.data_ptr() if q_start is not None else None,
                       selection.data_ptr() if selection is not None else None, T, block_table.shape[1], B, max_q, H, K,
                       DTYPES[q.dtype], 1 if causal else 0, scale, 0)
    return a, c, out


def gvr_kv4_attention_workspace(q, cache, block_table, ctx_len, kv_heads, selection=None, q_start=None, max_q=None,
                                causal=True) -> int:
    """Bytes of workspace with which ``gvr_kv4_attention`` of these tensors
    splits its contexts over the whole device (0: it does not split)."""
    a, c, _ = _attention_args(q, cache, block_table, ctx_len, kv_heads, selection, q_start, max_q, causal, None,
                              torch.empty_like(q, memory_format=torch.contiguous_format), None)
    n = ctypes.c_size_t(0)
    with _on_device(q.device):
        st = lib().gvr_kv4_attention_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n))
    if st != 0:
        raise GvrError("gvr_kv4_attention_workspace", st)
    return int(n.value)


def prepare_gvr_kv4_attention(q, cache, block_table, ctx_len, kv_heads, selection=None, q_start=None, max_q=None,
                              causal=True, scale=None, out=None, lse=None, workspace=None, stream=None):
    """A ``PreparedOp`` of ``gvr_kv4_attention`` (it keeps the workspace)."""
    a, c, out = _attention_args(q, cache, block_table, ctx_len, kv_heads, selection, q_start, max_q, causal, scale, out,
                                lse, stream)
    dev = q.device
    if workspace is None:
        n = ctypes.c_size_t(0)
        with _on_device(dev):
            st = lib().gvr_kv4_attention_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n))
        if st != 0:
            raise GvrError("gvr_kv4_attention_workspace", st)
        workspace = _new(max(int(n.value), 1), torch.uint8, dev, stream, returned=False)
    _need(isinstance(workspace, torch.Tensor) and workspace.device == dev and workspace.is_contiguous()
          and workspace.data_ptr() % 16 == 0, "workspace must be a contiguous 16-byte aligned tensor on %s" % dev)
    nbytes = workspace.numel() * workspace.element_size()
    args = (ctypes.byref(c), ctypes.byref(a), _ptr(workspace) if nbytes else None, nbytes, _stream(stream, dev))
    return _prepared("gvr_kv4_attention", dev, args, out,
                     (q, cache, block_table, ctx_len, selection, q_start, lse, workspace, a, c, stream))


def gvr_kv4_attention(q, cache, block_table, ctx_len, kv_heads, selection=None, q_start=None, max_q=None, causal=True,
                      scale=None, out=None, lse=None, workspace=None, stream=None):
    """Attention of q [T][q_heads][head_dim] (bfloat16 or float16) over the
    4-bit ``cache``; returns ``out`` [T][q_heads][head_dim].

    block_table (int32 [sequences][pages]) and ctx_len (int32 [sequences])
    describe the sequences; each has T / sequences query tokens, or rows
    q_start[b] .. q_start[b+1]-1 (int32 [sequences + 1], at most ``max_q``
    each; the others' rows of ``out`` and ``lse`` are not written). With
    ``q_start``, give ``max_q``: the launch is planned for that many rows of
    every sequence, and for all T of them if it is None (48 sequences of 3 rows:
    340 us instead of 38). ``selection`` (int32 [T][K], -1 padded: ``gvr_topk``'s result)
    restricts each row to the listed tokens. ``causal``: the queries are the
    last tokens of the context. ``lse`` (float32 [T][q_heads]) receives the
    log of the softmax's sum. ``workspace``: device memory for split contexts
    (``gvr_kv4_attention_workspace`` bytes; allocated for the call if None).
    The cache is a serving store: no gradient is recorded."""
    return prepare_gvr_kv4_attention(q, cache, block_table, ctx_len, kv_heads, selection, q_start, max_q, causal, scale,
                                     out, lse, workspace, stream)()
