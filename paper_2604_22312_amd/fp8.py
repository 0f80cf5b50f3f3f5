"""ctypes marshalling for 8-bit matrices with a scale per 128 elements
(``include/gvr_fp8.h``): argument checks and pointers only; the kernels are in
``csrc/fp8_quantize.hip`` and ``csrc/fp8_matmul.hip``. There is no CPU path."""
from __future__ import annotations

import ctypes
import functools
import math
from typing import NamedTuple

import torch
from torch.autograd.function import once_differentiable

from . import binding, kv4
from .binding import GvrError, _new, _on_device, _ptr, _stream
from .kv4 import DTYPES, _cs, _Heads, _heads_tensor, _index, _need, _no_overlap, _RopeCs

BLOCK = 128
MAX_HEAD = 1 << 20   # elements of a head at most
FP8_POW2, FP8_SQUARE = 1, 2

_ready = False


class _Fp8Heads(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("scale", ctypes.c_void_p), ("scale_token_stride", ctypes.c_int64), ("scale_head_stride", ctypes.c_int64)]


class _Fp8Matrix(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("scale", ctypes.c_void_p),
                ("scale_row_stride", ctypes.c_int64), ("scale_block_stride", ctypes.c_int64),
                ("rows_per_scale", ctypes.c_int32), ("reserved", ctypes.c_int32)]


def lib():
    """The library, with this module's entry points declared."""
    global _ready
    L = binding.lib()
    if not _ready:
        vp, i64, i32, p = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER
        L.gvr_fp8_quantize.argtypes = [p(_Heads), i32, i64, i32, i32, vp, p(_RopeCs), p(_Fp8Heads), vp, i64, i32, vp]
        L.gvr_fp8_quantize_matrix.argtypes = [vp, i64, i32, i64, i64, p(_Fp8Matrix), p(_Fp8Matrix), i32, vp]
        L.gvr_fp8_matmul_workspace.argtypes = [p(_Fp8Matrix), p(_Fp8Matrix), i64, i64, i64, p(ctypes.c_size_t)]
        L.gvr_fp8_matmul.argtypes = [p(_Fp8Matrix), p(_Fp8Matrix), i64, i64, i64, vp, i64, i32, vp, ctypes.c_size_t, vp]
        for name in ("gvr_fp8_quantize", "gvr_fp8_quantize_matrix", "gvr_fp8_matmul_workspace", "gvr_fp8_matmul"):
            getattr(L, name).restype = ctypes.c_int
        _ready = True
    return L


class Fp8Matrix(NamedTuple):
    """E4M3 codes (uint8 [rows][cols]) and their scales (float32 [rows or rows /
    128][cols / 128], rounded up)."""
    codes: torch.Tensor
    scale: torch.Tensor


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def prepare_gvr_fp8_quantize(x, table=None, positions=None, interleaved=False, pow2=False, slots=None, codes=None,
                             scale=None, stream=None):
    """A ``PreparedOp`` of ``gvr_fp8_quantize``."""
    flat = isinstance(x, torch.Tensor) and x.dim() == 2
    x3 = x.unsqueeze(1) if flat else x
    xs = _heads_tensor(x3, "x")
    T, H, D = x3.shape
    dev = x.device
    _need(1 <= D <= MAX_HEAD and H <= 1 << 20, "a token has at most 2^20 heads, a head 1 .. 2^20 elements")
    cs = None
    if table is not None:
        cs = _cs(table, interleaved, False, D, dev)
        _index(positions, "positions", torch.int32, (T,), dev)
    else:
        _need(positions is None, "positions need a table")
    if slots is not None:
        _index(slots, "slots", torch.int64, (T,), dev)
        _need(codes is not None and scale is not None, "slots name rows of given codes and scale")
    tail = (D,) if flat else (H, D)
    if codes is None:
        # (rows of a multiple of 16 bytes, which products load widest)
        wide = (D + 15) // 16 * 16
        codes = _new((T,) + tail[:-1] + (wide,), torch.uint8, dev, stream)[..., :D]
    if scale is None:
        scale = _new((T,) + tail[:-1] + (_blocks(D),), torch.float32, dev, stream)
    _need(isinstance(codes, torch.Tensor) and codes.dtype == torch.uint8 and codes.device == dev
          and tuple(codes.shape[1:]) == tail and (D == 1 or codes.stride(-1) == 1)
          and (slots is not None or codes.shape[0] == T), "codes must be a uint8 tensor of x's shape%s on %s, a head's "
          "elements contiguous" % (" but for its rows" if slots is not None else "", dev))
    _need(isinstance(scale, torch.Tensor) and scale.dtype == torch.float32 and scale.device == dev
          and tuple(scale.shape) == (codes.shape[0],) + tail[:-1] + (_blocks(D),)
          and (_blocks(D) == 1 or scale.stride(-1) == 1), "scale must be a float32 tensor %s on %s, a head's scales contiguous"
          % (list((codes.shape[0],) + tail[:-1] + (_blocks(D),)), dev))
    _no_overlap(codes, "codes")
    _no_overlap(scale, "scale")
    os = _Fp8Heads(codes.data_ptr(), codes.stride(0), 0 if flat else codes.stride(1),
                   scale.data_ptr(), scale.stride(0), 0 if flat else scale.stride(1))
    lib()
    args = (ctypes.byref(xs), DTYPES[x.dtype], T, H, D, _ptr(positions), ctypes.byref(cs) if cs is not None else None,
            ctypes.byref(os), _ptr(slots), codes.shape[0], FP8_POW2 if pow2 else 0, _stream(stream, dev))
    return kv4._prepared("gvr_fp8_quantize", dev, args, Fp8Matrix(codes, scale),
                         (x, positions, table, slots, xs, cs, os, stream))


def gvr_fp8_quantize(x, table=None, positions=None, interleaved=False, pow2=False, slots=None, codes=None, scale=None,
                     stream=None):
    """x [T][H][D] or [T][D] (bfloat16, float16 or float32; any token and head
    stride) as E4M3 codes with a float32 scale per 128 elements of a head: returns
    ``Fp8Matrix`` (codes uint8 of x's shape, scale [T][H][D / 128] or [T][D / 128]).
    With ``table`` and ``positions`` (int32 [T]) the heads are rotated first, as
    ``gvr_rope_rotate`` does it. ``pow2``: scales are powers of two. ``slots``
    (int64 [T], -1 skips the token): the rows of ``codes`` and ``scale``, a cache,
    that the tokens go to, e.g. the indexer's k [C][ld][D] viewed as [C * ld][1][D]
    with k_scale as [C * ld][1][1]. No gradient is recorded
    (``gvr_fp8_linear`` has one)."""
    return prepare_gvr_fp8_quantize(x, table, positions, interleaved, pow2, slots, codes, scale, stream)()


def _matrix_struct(m, name, rows, cols, per, dev, written=False):
    codes, scale = m
    _need(isinstance(codes, torch.Tensor) and codes.dtype == torch.uint8 and tuple(codes.shape) == (rows, cols)
          and codes.device == dev and (cols <= 1 or codes.stride(1) == 1),
          "%s: codes must be a uint8 tensor %s on %s, a row's contiguous" % (name, [rows, cols], dev))
    shape = ((rows + per - 1) // per, _blocks(cols))
    _need(isinstance(scale, torch.Tensor) and scale.dtype == torch.float32 and tuple(scale.shape) == shape
          and scale.device == dev, "%s: scale must be a float32 tensor %s on %s" % (name, list(shape), dev))
    if written:
        _no_overlap(codes, name)
        _no_overlap(scale, name)
    return _Fp8Matrix(codes.data_ptr(), codes.stride(0), scale.data_ptr(), scale.stride(0), scale.stride(1), per, 0)


def prepare_gvr_fp8_quantize_matrix(x, square=False, straight=True, transposed=False, pow2=False, out=None,
                                    out_transposed=None, stream=None):
    """A ``PreparedOp`` of ``gvr_fp8_quantize_matrix``."""
    _need(isinstance(x, torch.Tensor) and x.dim() == 2 and x.dtype in DTYPES,
          "x must be a bfloat16, float16 or float32 tensor [R][C]")
    _need(x.is_cuda, "x must be on a GPU (there is no CPU path)")
    R, C = x.shape
    _need(C <= 1 or x.stride(1) == 1, "x: a row's elements must be contiguous")
    _need(straight or transposed, "straight, transposed or both")
    _need((straight or out is None) and (transposed or out_transposed is None), "an output that was not asked for")
    dev, per = x.device, BLOCK if square else 1

    def made(given, rows, cols, name):
        if given is None:   # (rows of a multiple of 16 bytes, which products load widest)
            given = Fp8Matrix(_new((rows, (cols + 15) // 16 * 16), torch.uint8, dev, stream)[:, :cols],
                              _new(((rows + per - 1) // per, _blocks(cols)), torch.float32, dev, stream))
        return Fp8Matrix(*given), _matrix_struct(given, name, rows, cols, per, dev, True)
    a, sa = made(out, R, C, "out") if straight else (None, None)
    b, sb = made(out_transposed, C, R, "out_transposed") if transposed else (None, None)
    lib()
    args = (_ptr(x), x.stride(0), DTYPES[x.dtype], R, C, ctypes.byref(sa) if straight else None,
            ctypes.byref(sb) if transposed else None, (FP8_POW2 if pow2 else 0) | (FP8_SQUARE if square else 0),
            _stream(stream, dev))
    return kv4._prepared("gvr_fp8_quantize_matrix", dev, args, (a, b) if straight and transposed else a or b,
                         (x, sa, sb, stream))


def gvr_fp8_quantize_matrix(x, square=False, straight=True, transposed=False, pow2=False, out=None, out_transposed=None,
                            stream=None):
    """x [R][C] (bfloat16, float16 or float32; any row stride) as ``Fp8Matrix``:
    its codes (``straight``), those of x^T (``transposed``), or a pair of both from
    one reading of x. Blocks are 128 elements of a row of the result (of x's rows, of
    its columns), or 128 x 128 with ``square``, which both then share (a weight, for
    the product and for its gradient)."""
    return prepare_gvr_fp8_quantize_matrix(x, square, straight, transposed, pow2, out, out_transposed, stream)()


def _matmul_operands(a, a_scale, b, b_scale):
    for t, name in ((a, "a"), (b, "b")):
        _need(isinstance(t, torch.Tensor) and t.dim() == 2 and t.dtype == torch.uint8, "%s must be a uint8 tensor of codes"
              " [rows][K]" % name)
        _need(t.is_cuda, "%s must be on a GPU (there is no CPU path)" % name)
    (M, K), (N, Kb), dev = a.shape, b.shape, a.device
    _need(K == Kb, "a and b have rows of different lengths")
    _need(isinstance(b_scale, torch.Tensor) and b_scale.dim() == 2, "b_scale must be float32 [N or N / 128][K / 128]")
    per = BLOCK if b_scale.shape[0] == _blocks(N) else 1
    sa = _matrix_struct((a, a_scale), "a", M, K, 1, dev)
    return sa, _matrix_struct((b, b_scale), "b", N, K, per, dev), M, N, K


def _matmul_args(a, a_scale, b, b_scale, out, dtype, stream):
    sa, sb, M, N, K = _matmul_operands(a, a_scale, b, b_scale)
    dev = a.device
    if out is None:
        _need(dtype in DTYPES, "dtype must be bfloat16, float16 or float32")
        out = _new((M, N), dtype, dev, stream)
    _need(isinstance(out, torch.Tensor) and out.dtype in DTYPES and tuple(out.shape) == (M, N) and out.device == dev
          and (N <= 1 or out.stride(1) == 1), "out must be a bfloat16, float16 or float32 tensor %s on %s, a row's elements "
          "contiguous" % ([M, N], dev))
    _no_overlap(out, "out")
    return sa, sb, M, N, K, out


def _matmul_workspace(sa, sb, M, N, K, dev):
    n = ctypes.c_size_t(0)
    with _on_device(dev):
        st = lib().gvr_fp8_matmul_workspace(ctypes.byref(sa), ctypes.byref(sb), M, N, K, ctypes.byref(n))
    if st != 0:
        raise GvrError("gvr_fp8_matmul_workspace", st)
    return int(n.value)


def gvr_fp8_matmul_workspace(a, a_scale, b, b_scale) -> int:
    """Bytes of workspace with which ``gvr_fp8_matmul`` of these matrices splits
    its sums over the whole device and brings rows that are not 16-byte aligned into
    line (0: it does neither)."""
    sa, sb, M, N, K = _matmul_operands(a, a_scale, b, b_scale)
    return _matmul_workspace(sa, sb, M, N, K, a.device)


def prepare_gvr_fp8_matmul(a, a_scale, b, b_scale, out=None, dtype=torch.bfloat16, workspace=None, stream=None):
    """A ``PreparedOp`` of ``gvr_fp8_matmul`` (it keeps the workspace)."""
    sa, sb, M, N, K, out = _matmul_args(a, a_scale, b, b_scale, out, dtype, stream)
    dev = a.device
    if workspace is None:
        n = _matmul_workspace(sa, sb, M, N, K, dev)
        workspace = _new(max(n, 1), torch.uint8, dev, stream, returned=False)
    _need(isinstance(workspace, torch.Tensor) and workspace.device == dev and workspace.is_contiguous()
          and workspace.data_ptr() % 16 == 0, "workspace must be a contiguous 16-byte aligned tensor on %s" % dev)
    nbytes = workspace.numel() * workspace.element_size()
    args = (ctypes.byref(sa), ctypes.byref(sb), M, N, K, _ptr(out), out.stride(0), DTYPES[out.dtype],
            _ptr(workspace) if nbytes else None, nbytes, _stream(stream, dev))
    return kv4._prepared("gvr_fp8_matmul", dev, args, out, (a, a_scale, b, b_scale, workspace, sa, sb, stream))


def gvr_fp8_matmul(a, a_scale, b, b_scale, out=None, dtype=torch.bfloat16, workspace=None, stream=None):
    """out [M][N] = A B^T of codes a uint8 [M][K] with a_scale float32 [M][K / 128]
    and codes b [N][K] with b_scale [N / 128][K / 128] (a weight in blocks of
    128 x 128) or [N][K / 128]; any row strides, any strides of the scales.
    ``dtype``: bfloat16, float16 or float32, if ``out`` is not given. Into 16 bits the
    matrix cores cut products off at 2^-13 of the largest of eight neighbours
    (``include/gvr_fp8.h``, Numerics); into float32 every sum is float32, at half the rate.
    ``workspace``: device memory for split sums (``gvr_fp8_matmul_workspace``
    bytes; allocated for the call if None). No gradient is recorded
    (``gvr_fp8_linear`` has one)."""
    return prepare_gvr_fp8_matmul(a, a_scale, b, b_scale, out, dtype, workspace, stream)()


# gvr_fp8_linear makes its matrices in two blocks of memory, one for the call and one
# that the backward pass keeps, and hands the library pointers into them: six calls
# with tensors of their own and their checks took 340 us of host time a step.

class _Block:
    """Places of matrices in one block of memory that is allocated when all are known."""
    __slots__ = ("size", "made")

    def __init__(self):
        self.size, self.made = 0, []

    def matrix(self, rows, cols, per):
        """An ``_Fp8Matrix`` whose pointers count from the block's start until ``place``."""
        wide, blocks = (cols + 15) // 16 * 16, (cols + BLOCK - 1) // BLOCK
        scale = self.size + (rows * wide + 255) // 256 * 256
        m = _Fp8Matrix(self.size, wide, scale, blocks, 1, per, 0)
        self.size = scale + ((rows + per - 1) // per * blocks * 4 + 255) // 256 * 256
        self.made.append(m)
        return m

    def place(self, dev, more=0):
        """The block, with `more` bytes behind its matrices (their address: second)."""
        t = torch.empty(max(self.size + more, 1), dtype=torch.uint8, device=dev)
        start = t.data_ptr()
        for m in self.made:
            m.codes, m.scale = start + (m.codes or 0), start + (m.scale or 0)
        return t, start + self.size


def _check(name, status):
    if status != 0:
        raise GvrError(name, status)


def _layout(m):
    """Of an ``_Fp8Matrix``, what its product's workspace depends on beside its sizes."""
    return (m.codes or 0) % 16, m.row_stride, m.scale_row_stride, m.scale_block_stride


@functools.lru_cache(maxsize=4096)
def _product_workspace(M, N, K, per, device, layout=None):
    """Bytes of workspace of a product of matrices as a ``_Block`` has them (their sizes alone decide), or with a second one
    of the caller's, of this ``_layout``."""
    b = _Block()
    sa, sb = b.matrix(M, K, 1), b.matrix(N, K, per)
    if layout is not None:
        sb = _Fp8Matrix(layout[0], layout[1], 0, layout[2], layout[3], per, 0)
    return _matmul_workspace(sa, sb, M, N, K, torch.device("cuda", device))


def _rows_of(x):
    """x [...][C] as a matrix whose rows are contiguous."""
    m = x if x.dim() == 2 else x.reshape(math.prod(x.shape[:-1]), x.shape[-1])   # (C may be 0)
    return m.contiguous() if m.shape[1] > 1 and m.stride(1) != 1 else m


class _Linear(torch.autograd.Function):
    """y = Q(x) Q(W)^T, dx = Q(dy) Q(W), dW = Q(dy^T) Q(x^T)^T: the rounding to 8 bits
    counts as the identity. Codes of x^T and W^T are what the backward pass keeps."""

    @staticmethod
    def forward(ctx, x, weight, codes, scale, codes_t, scale_t):
        need_x, need_w = ctx.needs_input_grad[:2]
        L, dev = lib(), x.device
        x2 = _rows_of(x)
        (M, K), N = x2.shape, (weight if weight is not None else codes).shape[0]
        y = torch.empty((M, N), dtype=x.dtype, device=dev)
        now, kept = _Block(), _Block()
        xq = now.matrix(M, K, 1)
        xt = kept.matrix(K, M, 1) if need_w else None
        if weight is not None:
            wq, wt = now.matrix(N, K, BLOCK), kept.matrix(K, N, BLOCK) if need_x else None
        else:
            wq, wt = _matrix_struct((codes, scale), "weight", N, K, BLOCK, dev), None
        ws = _product_workspace(M, N, K, BLOCK, dev.index, _layout(wq) if weight is None else None)
        block, ws_at = now.place(dev, ws)
        saved = kept.place(dev)[0] if kept.made else None
        with _on_device(dev):
            stream = _stream(None, dev)
            if need_w or K > MAX_HEAD:   # (the same codes of longer rows than a head may have)
                _check("gvr_fp8_quantize_matrix", L.gvr_fp8_quantize_matrix(
                    x2.data_ptr(), x2.stride(0), DTYPES[x.dtype], M, K, ctypes.byref(xq),
                    ctypes.byref(xt) if need_w else None, 0, stream))
            else:
                _check("gvr_fp8_quantize", L.gvr_fp8_quantize(
                    ctypes.byref(_Heads(x2.data_ptr(), x2.stride(0), 0)), DTYPES[x.dtype], M, 1, K, None, None,
                    ctypes.byref(_Fp8Heads(xq.codes, xq.row_stride, 0, xq.scale, xq.scale_row_stride, 0)), None, M, 0, stream))
            if weight is not None:
                w2 = _rows_of(weight)
                _check("gvr_fp8_quantize_matrix", L.gvr_fp8_quantize_matrix(
                    w2.data_ptr(), w2.stride(0), DTYPES[weight.dtype], N, K, ctypes.byref(wq),
                    ctypes.byref(wt) if need_x else None, FP8_SQUARE, stream))
            _check("gvr_fp8_matmul", L.gvr_fp8_matmul(
                ctypes.byref(xq), ctypes.byref(wq), M, N, K, y.data_ptr(), N, DTYPES[x.dtype],
                ws_at if ws else None, ws, stream))
        ctx.save_for_backward(saved, codes_t, scale_t)
        ctx.sizes = M, N, K
        ctx.types = x.dtype, weight.dtype if weight is not None else None
        ctx.shape = x.shape
        return y.view(x.shape[:-1] + (N,))

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        saved, codes_t, scale_t = ctx.saved_tensors
        need_x, need_w = ctx.needs_input_grad[:2]
        if not need_x and not need_w:
            return (None,) * 6
        (M, N, K), L, dev = ctx.sizes, lib(), dy.device
        d = _rows_of(dy)
        kept, now = _Block(), _Block()   # (the places that forward gave out)
        xt = kept.matrix(K, M, 1) if need_w else None
        if codes_t is not None:
            wt = _matrix_struct((codes_t, scale_t), "weight_t", K, N, BLOCK, dev)
        else:
            wt = kept.matrix(K, N, BLOCK) if need_x else None
        for m in kept.made:
            m.codes, m.scale = saved.data_ptr() + (m.codes or 0), saved.data_ptr() + (m.scale or 0)
        dq, dt = now.matrix(M, N, 1) if need_x else None, now.matrix(N, M, 1) if need_w else None
        dx = torch.empty((M, K), dtype=ctx.types[0], device=dev) if need_x else None
        dw = torch.empty((N, K), dtype=ctx.types[1], device=dev) if need_w else None
        ws_x = _product_workspace(M, K, N, BLOCK, dev.index, _layout(wt) if codes_t is not None else None) if need_x else 0
        ws_w = _product_workspace(N, K, M, 1, dev.index) if need_w else 0
        ws = max(ws_x, ws_w)   # (one after the other)
        block, ws_at = now.place(dev, ws)
        with _on_device(dev):
            stream = _stream(None, dev)
            _check("gvr_fp8_quantize_matrix", L.gvr_fp8_quantize_matrix(
                d.data_ptr(), d.stride(0), DTYPES[d.dtype], M, N, ctypes.byref(dq) if need_x else None,
                ctypes.byref(dt) if need_w else None, 0, stream))
            if need_x:
                _check("gvr_fp8_matmul", L.gvr_fp8_matmul(
                    ctypes.byref(dq), ctypes.byref(wt), M, K, N, dx.data_ptr(), K, DTYPES[dx.dtype],
                    ws_at if ws_x else None, ws_x, stream))
            if need_w:
                _check("gvr_fp8_matmul", L.gvr_fp8_matmul(
                    ctypes.byref(dt), ctypes.byref(xt), N, K, M, dw.data_ptr(), K, DTYPES[dw.dtype],
                    ws_at if ws_w else None, ws_w, stream))
        return dx.view(ctx.shape) if need_x else None, dw, None, None, None, None


def gvr_fp8_linear(x, weight, weight_t=None):
    """y [...][N] = x [...][K] W^T in 8 bits, with gradients, on the current
    stream. ``weight``: [N][K] in bfloat16, float16 or float32, quantised in the
    call (blocks of 128 x 128) and given a gradient, or, of a frozen layer, the
    ``Fp8Matrix`` of it that ``gvr_fp8_quantize_matrix(W, square=True,
    transposed=True)`` made, with that of W^T as ``weight_t``, which the gradient of
    x needs. x and the gradient of y are quantised by 128 elements along the axis
    that each product sums over; the rounding counts as the identity, and there is no
    second derivative. y and the gradients have the types of x and of the weight, and
    their sums are those of ``gvr_fp8_matmul`` into that type.
    A training step may be captured into a graph, on one condition that all autograd
    nodes share: no graph that was recorded eagerly from the same leaves is alive
    (their accumulation belongs to the stream that it was recorded on)."""
    _need(isinstance(x, torch.Tensor) and x.dim() >= 1 and x.dtype in DTYPES and x.is_cuda,
          "x must be a bfloat16, float16 or float32 tensor [...][K] on a GPU (there is no CPU path)")
    _need(x.shape[-1] >= 1, "a row of x needs at least one element")
    if not torch.is_grad_enabled():   # (nothing is kept, and no codes of the transposed are made, for a backward pass that cannot be)
        x = x.detach()
        weight = weight.detach() if isinstance(weight, torch.Tensor) else weight
    if isinstance(weight, torch.Tensor):
        _need(weight.dim() == 2 and weight.dtype in DTYPES and weight.device == x.device and weight.shape[1] == x.shape[-1],
              "weight must be a bfloat16, float16 or float32 tensor [N][%d] on %s" % (x.shape[-1], x.device))
        _need(weight_t is None, "weight_t goes with a weight that is an Fp8Matrix")
        return _Linear.apply(x, weight, None, None, None, None)
    _need(isinstance(weight, tuple) and len(weight) == 2, "weight must be a tensor or an Fp8Matrix")
    N = weight[0].shape[0]
    _matrix_struct(weight, "weight", N, x.shape[-1], BLOCK, x.device)
    if weight_t is not None:
        _matrix_struct(weight_t, "weight_t", x.shape[-1], N, BLOCK, x.device)
    _need(weight_t is not None or not (torch.is_grad_enabled() and x.requires_grad), "the gradient of x needs weight_t")
    return _Linear.apply(x, None, *weight, *(weight_t or (None, None)))
