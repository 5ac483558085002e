"""MI355X-native E-Sparse hot path: thin ctypes binding over libesparse.so (gfx950)."""
from .binding import (Context, PruneOpts, PruneResult, Compressed, MX, MXWeight, TokenLogprobs, EsparseError, load_library,
                      compressed_size, spmm_workspace, dense_packed_size, mx_size, mx_packed_size, mx_gemm_workspace,
                      token_logprobs_workspace, num_variants, variant_name,
                      F16, BF16, F32, MX_FP4, MX_FP8, MAX_TOP, USE_ENTROPY, USE_NORM, USE_GNS, USE_LBS, USE_ALL)

__all__ = ["Context", "PruneOpts", "PruneResult", "Compressed", "MX", "MXWeight", "TokenLogprobs", "EsparseError", "load_library",
           "compressed_size", "spmm_workspace", "dense_packed_size", "mx_size", "mx_packed_size", "mx_gemm_workspace",
           "token_logprobs_workspace", "num_variants", "variant_name",
           "F16", "BF16", "F32", "MX_FP4", "MX_FP8", "MAX_TOP", "USE_ENTROPY", "USE_NORM", "USE_GNS", "USE_LBS", "USE_ALL"]
