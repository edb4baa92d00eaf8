"""MI355X-native vector-wise N:M sparse matrix multiplication (NM-SpMM,
arXiv 2503.01253): C = A * B with B pruned N:M along k in blocks of V columns
and stored compressed as (Bc, idx).

The compute lives in libnmspmm.so (hand-written gfx950 HIP kernels behind a
C ABI declared in include/nmspmm.h); this package is its ctypes binding.
"""
from .binding import (  # noqa: F401
    ACTS, EXPORTS, NMSPMM_ACT_GELU, NMSPMM_ACT_NONE, NMSPMM_ACT_RELU, NMSPMM_ERR_HIP,
    NMSPMM_ERR_INVALID_ARG, NMSPMM_ERR_SCRATCH, NMSPMM_ERR_UNSUPPORTED, NMSPMM_NOALLOC_SCRATCH_BYTES, NMSPMM_OK, NmSpmmError, lib,
    nmspmm_bc_elems, nmspmm_compress, nmspmm_compress_device, nmspmm_confusion, nmspmm_idx_bytes,
    nmspmm_kernel_name, nmspmm_kernel_name_ws, nmspmm_run, nmspmm_run_ex, nmspmm_run_noalloc, nmspmm_run_ptr, nmspmm_run_ws,
    nmspmm_status_string, nmspmm_validate_idx, nmspmm_workspace_bytes,
)
from .serve import (  # noqa: F401
    HALF_ACTS, NMSPMM_BF16, NMSPMM_F16, NMSPMM_F32, SERVE_EXPORTS, HalfWeight, KvCache,
    nmspmm_half_bytes, nmspmm_half_kernel_name, nmspmm_half_pack, nmspmm_half_run, nmspmm_half_workspace_bytes,
    nmspmm_kv_append, nmspmm_kv_append_norm, nmspmm_kv_attend, nmspmm_kv_attend_workspace_bytes, nmspmm_kv_cache,
)
from .mx4 import (  # noqa: F401
    MX4_EXPORTS, Kv4Cache, Mx4Weight, nmspmm_kv4_append, nmspmm_kv4_attend, nmspmm_kv4_attend_workspace_bytes,
    nmspmm_kv4_cache, nmspmm_kv4_page_bytes, nmspmm_kv4_read, nmspmm_mx4_bytes, nmspmm_mx4_kernel_name,
    nmspmm_mx4_pack, nmspmm_mx4_quantize, nmspmm_mx4_run, nmspmm_mx4_workspace_bytes,
)
