"""Exact decode-time Top-K for MI355X (gfx950): Guess-Verify-Refine and radix select.

Thin Python binding over the C ABI of ``include/gvr_topk.h`` (library
``libgvr_topk.so`` built in-tree by ``paper_2604_22312_amd.build``). This module
only validates tensors and marshals pointers; every step of the Top-K runs in
the HIP kernels of ``csrc/gvr_topk.hip``, ``csrc/rope_prior.hip`` and
``csrc/indexer.hip`` (rotary positions and the 4-bit cache:
``csrc/rotary.hip``, ``csrc/kv4_cache.hip``, ``csrc/kv4_attention.hip``; pages
and 8-bit matrices: ``csrc/pages.hip``, ``csrc/fp8_quantize.hip``,
``csrc/fp8_matmul.hip``). There is no CPU fallback: if the
library is missing, importing the functions raises.

Functions mirror the C entry points:

* ``gvr_topk(scores, row_len, prev_topk, K, out_idx=None, stream=None)``
* ``radix_topk(scores, row_len, prev_topk, K, out_idx=None, stream=None)``
* ``gvr_topk_ex`` / ``radix_topk_ex`` (options, per-row stats)
* ``gvr_topk_ex_noalloc`` -- ``gvr_topk_ex`` with no allocation inside the
  call (split-row workspace in a static device array)
* ``gvr_workspace_size`` / ``gvr_topk_ex_ws`` / ``radix_topk_ex_ws`` /
  ``new_workspace`` -- the split-row workspace owned by the caller (nothing
  allocated inside the call)
* ``prepare_gvr_topk`` / ``prepare_radix_topk`` -- a call checked and
  marshalled once, re-enqueued by calling it (loops over fixed buffers; with
  ``workspace=``, on a caller workspace)
* ``gvr_rope_g(n, params=None, device=...)`` -- g(Delta) of the RoPE/YaRN prior
* ``gvr_rope_prior(n, K, params=None, device=...)`` -- its static index set
  (``include/gvr_rope_prior.h``)
* ``gvr_indexer_scores(q, w, k, k_scale, ...)`` / ``gvr_indexer_topk(...)`` --
  the FP8 indexer scores, and the indexer followed by gvr_topk
  (``include/gvr_indexer.h``)
* ``gvr_rope_table(n, ...)`` / ``gvr_rope_rotate(x, positions, table, ...)`` --
  rotary positions of queries and keys, and of their gradients
  (``include/gvr_rotary.h``)
* ``new_kv4_cache`` / ``gvr_kv4_append`` / ``gvr_kv4_read`` /
  ``gvr_kv4_attention`` -- the paged 4-bit key / value cache: tokens in (keys
  rotated on the way) and out, and attention over all of a context or over
  the tokens a Top-K selected (``include/gvr_kv4.h``)
* ``new_page_pool`` / ``gvr_page_step`` -- block tables, slots, positions and row
  starts from the tokens that requests keep and bring (``include/gvr_pages.h``)
* ``gvr_fp8_quantize`` / ``gvr_fp8_quantize_matrix`` / ``gvr_fp8_matmul`` /
  ``gvr_fp8_linear`` -- E4M3 codes with a scale per 128 elements: of heads (rotated,
  into the indexer's key cache) and matrices, their products, and a linear layer of
  them with its gradients (``include/gvr_fp8.h``)
"""
from .binding import (  # noqa: F401
    GVR_MAX_CANDIDATES,
    GVR_MAX_K,
    PATH_NAMES,
    GvrError,
    Options,
    PreparedCall,
    RopeParams,
    decode_stats,
    gvr_indexer_scores,
    gvr_indexer_topk,
    gvr_rope_g,
    gvr_rope_params,
    gvr_read_floor,
    gvr_rope_prior,
    gvr_topk,
    gvr_topk_ex,
    gvr_topk_ex_noalloc,
    gvr_topk_ex_ws,
    gvr_workspace_size,
    lib,
    library_path,
    new_stats,
    new_workspace,
    prepare_gvr_topk,
    prepare_radix_topk,
    radix_topk,
    radix_topk_ex,
    radix_topk_ex_ws,
    status_string,
    version,
)
from .fp8 import (  # noqa: F401
    Fp8Matrix,
    gvr_fp8_linear,
    gvr_fp8_matmul,
    gvr_fp8_matmul_workspace,
    gvr_fp8_quantize,
    gvr_fp8_quantize_matrix,
    prepare_gvr_fp8_matmul,
    prepare_gvr_fp8_quantize,
    prepare_gvr_fp8_quantize_matrix,
)
from .kv4 import (  # noqa: F401
    PreparedOp,
    gvr_kv4_append,
    gvr_kv4_attention,
    gvr_kv4_attention_workspace,
    gvr_kv4_read,
    gvr_kv4_record_bytes,
    gvr_rope_rotate,
    gvr_rope_table,
    new_kv4_cache,
    prepare_gvr_kv4_append,
    prepare_gvr_kv4_attention,
    prepare_gvr_kv4_read,
    prepare_gvr_rope_rotate,
)
from .pages import (  # noqa: F401
    PagePool,
    PageStep,
    gvr_page_step,
    gvr_page_step_workspace,
    new_page_pool,
    prepare_gvr_page_step,
)
