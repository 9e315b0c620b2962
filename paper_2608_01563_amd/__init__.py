"""MI355X (gfx950) attention forward and backward, attention over a 4-bit
and over a paged key/value cache, and the two derivatives of a 2-D convolution, behind a C ABI.

The compute path is libmg.so (hand-written HIP kernels, see csrc/,
include/mg_attn.h, include/mg_kv4.h, include/mg_paged.h and include/mg_conv.h);
this package is its ctypes binding.  PyTorch is used only for device memory and
streams.
"""
from ._binding import (  # noqa: F401
    ACCELERATED,
    FAST_BF16,
    CONV_HEADER_PATH,
    HEADER_PATH,
    KV4_HEADER_PATH,
    LIB_PATH,
    PAGED_HEADER_PATH,
    STRICT_F32,
    MgError,
    attention_backward,
    attention_forward,
    conv2d_backward,
    conv_shape,
    load_library,
    mg_attn_bwd,
    mg_attn_bwd_cross,
    mg_attn_bwd_cross_workspace_bytes,
    mg_attn_bwd_noalloc,
    mg_attn_bwd_workspace_bytes,
    mg_attn_fwd,
    mg_attn_fwd_cross,
    mg_conv2d_bwd,
    mg_conv2d_bwd_data,
    mg_conv2d_bwd_data_workspace_bytes,
    mg_conv2d_bwd_filter,
    mg_conv2d_bwd_filter_workspace_bytes,
    mg_conv2d_bwd_workspace_bytes,
    mg_last_error_detail,
    mg_lds_probe,
    mg_mfma_peak,
    mg_profile_collect,
    mg_profile_enable,
    mg_profile_reset,
    mg_status_string,
)
from ._kv4 import (  # noqa: F401
    attention_forward_kv4,
    kv4_cache,
    mg_attn_fwd_kv4,
    mg_attn_fwd_kv4_workspace_bytes,
    mg_kv4_append,
    mg_kv4_cache_bytes,
    mg_kv4_evict,
    mg_kv4_read,
)
from ._paged import (  # noqa: F401
    attention_forward_paged,
    mg_attn_fwd_paged,
    mg_attn_fwd_paged_sparse,
    mg_attn_fwd_paged_sparse_workspace_bytes,
    mg_attn_fwd_paged_workspace_bytes,
    mg_paged_append,
    mg_paged_resize,
    mg_paged_resize_workspace_bytes,
    mg_paged_select,
    mg_paged_select_workspace_bytes,
    paged_cache,
)
