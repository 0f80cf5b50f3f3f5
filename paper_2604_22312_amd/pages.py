"""ctypes marshalling for the page step (``include/gvr_pages.h``): argument
checks and pointers only; the kernels are in ``csrc/pages.hip``. There is no CPU
path."""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import binding, kv4
from .binding import _new, _ptr, _stream
from .kv4 import _index, _need

_ready = False


class _Pool(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("ctx_len", ctypes.c_void_p), ("free_pages", ctypes.c_void_p),
                ("free_count", ctypes.c_void_p), ("width", ctypes.c_int64), ("pages", ctypes.c_int64),
                ("requests", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class _StepArgs(ctypes.Structure):
    _fields_ = [("new_len", ctypes.c_void_p), ("keep", ctypes.c_void_p), ("T", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("q_start", ctypes.c_void_p), ("taken", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("slots", ctypes.c_void_p), ("dense", ctypes.c_void_p), ("row_len", ctypes.c_void_p)]


def lib():
    """The library, with this module's entry points declared."""
    global _ready
    L = binding.lib()
    if not _ready:
        L.gvr_page_step_workspace.argtypes = [ctypes.c_int32]
        L.gvr_page_step_workspace.restype = ctypes.c_int64
        L.gvr_page_step.argtypes = [ctypes.POINTER(_Pool), ctypes.POINTER(_StepArgs), ctypes.c_void_p, ctypes.c_size_t,
                                    ctypes.c_void_p]
        L.gvr_page_step.restype = ctypes.c_int
        _ready = True
    return L


class PagePool(NamedTuple):
    """The pages of a paged cache and who holds them: block_table int32
    [requests][width] (-1: none), ctx_len int32 [requests], and the stack of free
    pages, free_pages int32 [pages] with free_count int32 [1] entries."""
    block_table: torch.Tensor
    ctx_len: torch.Tensor
    free_pages: torch.Tensor
    free_count: torch.Tensor
    page_size: int


class PageStep(NamedTuple):
    """What a step says of its rows (``gvr_page_step``)."""
    q_start: torch.Tensor            # int32 [requests + 1]
    taken: torch.Tensor              # int32 [requests]
    positions: torch.Tensor          # int32 [T]
    slots: torch.Tensor              # int64 [T]
    dense: Optional[torch.Tensor]    # int64 [T]
    row_len: torch.Tensor            # int32 [T]


def new_page_pool(pages, page_size, requests, width, device="cuda"):
    """A ``PagePool`` whose pages are all free and whose requests are empty."""
    ints = dict(dtype=torch.int32, device=device)
    return PagePool(torch.full((int(requests), int(width)), -1, **ints), torch.zeros(int(requests), **ints),
                    torch.arange(int(pages), **ints), torch.full((1,), int(pages), **ints), int(page_size))


def prepare_gvr_page_step(pool, new_len, tokens, keep=None, ld=None, workspace=None, stream=None):
    """A ``PreparedOp`` of ``gvr_page_step`` (it keeps the workspace and writes
    the same results again)."""
    _need(isinstance(pool, PagePool), "pool must be a PagePool")
    table = pool.block_table
    _need(isinstance(table, torch.Tensor) and table.dim() == 2 and table.dtype == torch.int32 and table.is_contiguous(),
          "block_table must be a contiguous int32 tensor [requests][width]")
    _need(table.is_cuda, "the pool must be on a GPU (there is no CPU path)")
    dev, (R, W) = table.device, table.shape
    _need(R <= 1 << 20, "at most 2^20 requests")
    _index(pool.ctx_len, "ctx_len", torch.int32, (R,), dev)
    _need(isinstance(pool.free_pages, torch.Tensor) and pool.free_pages.dim() == 1, "free_pages must be int32 [pages]")
    _index(pool.free_pages, "free_pages", torch.int32, tuple(pool.free_pages.shape), dev)
    _index(pool.free_count, "free_count", torch.int32, (1,), dev)
    _index(new_len, "new_len", torch.int32, (R,), dev)
    if keep is not None:
        _index(keep, "keep", torch.int32, (R,), dev)
    page, T = int(pool.page_size), int(tokens)
    _need(1 <= page <= 65536 and page & (page - 1) == 0, "the page size must be a power of two up to 65536")
    _need(0 <= T <= (1 << 31) - 16, "tokens must be 0 .. 2^31 - 16")
    _need(ld is None or 0 <= int(ld) <= (1 << 31) - 16, "ld must be 0 .. 2^31 - 16")
    out = PageStep(_new((R + 1,), torch.int32, dev, stream), _new((R,), torch.int32, dev, stream),
                   _new((T,), torch.int32, dev, stream), _new((T,), torch.int64, dev, stream),
                   None if ld is None else _new((T,), torch.int64, dev, stream), _new((T,), torch.int32, dev, stream))
    L = lib()
    if workspace is None:
        workspace = _new(int(L.gvr_page_step_workspace(R)), torch.uint8, dev, stream, returned=False)
    _need(isinstance(workspace, torch.Tensor) and workspace.device == dev and workspace.is_contiguous()
          and workspace.data_ptr() % 16 == 0, "workspace must be a contiguous 16-byte aligned tensor on %s" % dev)
    p = _Pool(table.data_ptr(), pool.ctx_len.data_ptr(), pool.free_pages.data_ptr(), pool.free_count.data_ptr(), W,
              pool.free_pages.shape[0], R, page)
    a = _StepArgs(new_len.data_ptr(), None if keep is None else keep.data_ptr(), T, 0 if ld is None else int(ld),
                  *(None if t is None else t.data_ptr() for t in out))
    args = (ctypes.byref(p), ctypes.byref(a), _ptr(workspace), workspace.numel() * workspace.element_size(),
            _stream(stream, dev))
    return kv4._prepared("gvr_page_step", dev, args, out, (pool, new_len, keep, workspace, p, a, stream))


def gvr_page_step_workspace(requests) -> int:
    """Bytes of workspace of a step of so many requests."""
    n = int(lib().gvr_page_step_workspace(int(requests)))
    _need(n >= 0, "requests must be 0 .. 2^20")
    return n


def gvr_page_step(pool, new_len, tokens, keep=None, ld=None, workspace=None, stream=None):
    """One step of ``pool`` (a ``PagePool``, updated in place): request r is cut
    back to ``keep[r]`` tokens (int32; None: all that it has; 0 ends it) and
    brings ``new_len[r]`` more (int32), in the order of requests, into buffers of
    ``tokens`` rows. Returns a ``PageStep``: ``q_start`` for the attention,
    ``taken`` (new_len, or 0 for a request that was not served: no pages, no
    place in its table or no rows left), and for every row ``positions``,
    ``slots`` for the append, ``dense`` = r * ld + position for a cache
    [requests][ld] (-1 where the position is ld or more; None without ``ld``) and ``row_len`` = position + 1 for the
    indexer. Rows of nobody: 0, -1, -1 and 0. ``workspace``: device memory of
    ``gvr_page_step_workspace`` bytes, allocated for the call if None."""
    return prepare_gvr_page_step(pool, new_len, tokens, keep, ld, workspace, stream)()
