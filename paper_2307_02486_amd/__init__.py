"""MI355X (gfx950) dilated attention, forward and backward passes (LongNet,
Sec. 2.2-2.3), the head norms of its attention layer, and serving from a paged
cache.

The computation runs in the HIP kernels of libdilated_attn.so behind the C
ABI declared in include/dilated_attn.h, include/dilated_attn_paged.h and
include/dilated_attn_compressed.h; this package only marshals arguments.
"""
from .ops import (StageTimer, bwd_workspace_for, cache_append, cache_scale_shape, dilated_attn,  # noqa: F401
                  dilated_attn_bwd, evict_pages, layer_norm, layer_norm_bwd, page_weights,
                  page_weights_workspace_bytes, paged_attn, paged_workspace_bytes, plan, plan_bwd, plan_raw,
                  qk_norm_xpos, qk_norm_xpos_bwd, wgrad, workspace_for, xpos)
from ._lib import DilatedAttnError, LIB_PATH  # noqa: F401

__all__ = ["StageTimer", "dilated_attn", "dilated_attn_bwd", "plan", "plan_bwd", "plan_raw",
           "workspace_for", "bwd_workspace_for", "xpos", "wgrad", "layer_norm", "layer_norm_bwd",
           "qk_norm_xpos", "qk_norm_xpos_bwd", "cache_append", "paged_attn", "paged_workspace_bytes",
           "cache_scale_shape", "page_weights", "page_weights_workspace_bytes", "evict_pages",
           "DilatedAttnError", "LIB_PATH"]
