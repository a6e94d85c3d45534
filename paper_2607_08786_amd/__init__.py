"""MI355X-native unstructured-sparse fp16 SpMM (decode-phase Y = W X).

The C ABI lives in ``include/usp.h`` and ``libusp.so``; ``usp`` is its Python
binding. Importing this package does not load the library; the first call does,
and raises if it has not been built.
"""
from . import usp  # noqa: F401
from .usp import (  # noqa: F401
    CacheRows,
    ExpertGroup,
    KVCache,
    SparseMatrix,
    SparseMatrixQ,
    UspError,
    load_library,
    usp_attention,
    usp_cache_append,
    usp_cache_copy,
    usp_cache_read,
    usp_decode,
    usp_decode_q,
    usp_densify,
    usp_encode,
    usp_encode_q,
    usp_free,
    usp_group_create,
    usp_group_free,
    usp_info,
    usp_last_error,
    usp_norm,
    usp_quantize,
    usp_spmm,
    usp_spmm_grouped,
    usp_spmm_q,
    usp_workspace_size,
)
