"""MI355X-native chunked MoE expert layer (MemFine's per-GPU hot path).

The compute lives in libmemfine.so (hand-written gfx950 HIP kernels behind
the C ABI of include/memfine.h); this package only builds and binds it.
"""
from ._lib import (BF16, CHUNK_EXPERTS, CHUNK_TOKENS, ERR_SCRATCH, F32, NOALLOC_SCRATCH_BYTES, PASS_BWD, PASS_FWD, TILE_128, TILE_256, TILE_256_REG,  # noqa: F401
                   SCORE_SIGMOID, SCORE_SOFTMAX, TILE_AUTO, MemfineError, TorchAllocator, lib, make_attn,
                   make_cache, make_gating,
                   make_model, make_shape,
                   memfine_activation_memory, memfine_attn_bwd,
                   memfine_attn_bwd_workspace_bytes, memfine_attn_decode,
                   memfine_attn_decode_workspace_bytes, memfine_attn_fwd, memfine_count, memfine_dispatch,
                   memfine_get_launch_options, memfine_kv_write, memfine_mact_select, memfine_mact_thresholds,
                   memfine_moe_bwd, memfine_moe_fwd, memfine_moe_fwd_noalloc, memfine_plan, memfine_pool_high_water,
                   memfine_linear_mxw, memfine_linear_mxw_workspace_bytes, memfine_moe_fwd_mxw, memfine_moe_mxw_workspace_bytes,
                   memfine_mx_values, memfine_mxw_code_bytes, memfine_mxw_pack,
                   memfine_mxw_quantize, memfine_mxw_scale_bytes, memfine_mxw_unpack,
                   memfine_norm_bwd, memfine_norm_fwd,
                   memfine_profile_begin, memfine_profile_end, memfine_rope, memfine_route_bwd, memfine_route_fwd,
                   memfine_router_bwd, memfine_router_fwd, memfine_router_logits,
                   memfine_router_logits_bwd, memfine_set_launch_options, memfine_static_memory,
                   memfine_status_str, memfine_workspace_bytes, memfine_workspace_held,
                   memfine_workspace_trim)
