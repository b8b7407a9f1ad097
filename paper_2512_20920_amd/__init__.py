"""RevFFN reversible MoE block for AMD MI355X: thin Python binding over librevffn.so.

Every arithmetic step runs in the HIP kernels of the shared library; this package
only marshals arguments (torch tensors are used for device memory and streams).
Importing the package does not load the library; the first call does, and raises
if it has not been built (there is no CPU fallback).
"""
from .binding import (Config, Weights, Grads, Context, load_library, library_path,
                      revffn_forward, revffn_inverse, revffn_backward, revffn_backward_stored, revffn_inverse_backward,
                      revffn_stack_forward, revffn_stack_backward, revffn_get_routing,
                      revffn_get_branch, revffn_strerror, RevffnError, EXPORTED_SYMBOLS,
                      WEIGHT_FIELDS, revffn_op_gemm, revffn_op_attention_fwd, revffn_op_attention_bwd,
                      revffn_op_attention_bwd_noalloc, revffn_op_tile_placement,
                      Merged, MERGED_FIELDS, revffn_merge_adapters, revffn_forward_merged, revffn_inverse_merged,
                      AttnDesc, AttnMask, Rotary, revffn_op_attention_ranges, revffn_op_attention_masked_workspace,
                      revffn_op_attention_masked_fwd, revffn_op_attention_masked_bwd, revffn_op_rotary_frequencies,
                      revffn_op_rotary, revffn_op_layernorm_workspace, revffn_op_layernorm_fwd, revffn_op_layernorm_bwd,
                      Cache, revffn_op_cache_append, revffn_op_attention_cached_workspace, revffn_op_attention_cached,
                      revffn_op_quantize_rows, revffn_op_gemm_int)

__all__ = ["Config", "Weights", "Grads", "Context", "load_library", "library_path",
           "revffn_forward", "revffn_inverse", "revffn_backward", "revffn_backward_stored", "revffn_inverse_backward",
           "revffn_stack_forward",
           "revffn_stack_backward", "revffn_get_routing", "revffn_get_branch",
           "revffn_strerror", "RevffnError", "EXPORTED_SYMBOLS", "WEIGHT_FIELDS", "revffn_op_gemm",
           "revffn_op_attention_fwd", "revffn_op_attention_bwd", "revffn_op_attention_bwd_noalloc",
           "revffn_op_tile_placement", "Merged", "MERGED_FIELDS", "revffn_merge_adapters", "revffn_forward_merged",
           "revffn_inverse_merged", "AttnDesc", "AttnMask", "Rotary", "revffn_op_attention_ranges",
           "revffn_op_attention_masked_workspace", "revffn_op_attention_masked_fwd", "revffn_op_attention_masked_bwd",
           "revffn_op_rotary_frequencies", "revffn_op_rotary", "revffn_op_layernorm_workspace", "revffn_op_layernorm_fwd",
           "revffn_op_layernorm_bwd", "Cache", "revffn_op_cache_append", "revffn_op_attention_cached_workspace",
           "revffn_op_attention_cached", "revffn_op_quantize_rows", "revffn_op_gemm_int"]
