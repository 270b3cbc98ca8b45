"""libmas: batched Monotonic Alignment Search for AMD MI355X (gfx950).

The alignment, and the attention, norm and loss around it, run in hand-written
HIP kernels behind the C ABI of ``include/mas.h``; this package is the thin
Python binding with the same entry-point names.  It never computes a result in
Python.
"""
from ._native import (  # noqa: F401
    ITEM_BAD_WORKSPACE,
    ITEM_EMPTY,
    ITEM_INFEASIBLE,
    ITEM_OK,
    ITEM_OUT_OF_RANGE,
    ITEM_SYNC_TIMEOUT,
    LIB_PATH,
    STATIC_SCRATCH_BYTES,
    MasError,
    Workspace,
    lib,
    mas_align_loss,
    mas_align_loss_workspace_bytes,
    mas_attention,
    mas_attention_backward,
    mas_attention_workspace_bytes,
    mas_expand_path,
    mas_expand_text,
    mas_forward,
    mas_forward_ex,
    mas_forward_sentinel,
    mas_forward_static,
    mas_loglik,
    mas_qk_norm_rope,
    mas_qk_norm_rope_backward,
    mas_qk_norm_rope_workspace_bytes,
    mas_search,
    mas_status_string,
    mas_version,
    mas_workspace_bytes,
    mas_workspace_init,
)
