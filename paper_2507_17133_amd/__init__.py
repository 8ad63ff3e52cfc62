"""BrownoutMoE layer forward for MI355X (gfx950): thin Python face of libbrownout_moe.so."""
from .binding import (MoeError, RouteOut, alloc_route_out, alloc_workspace, config_of, init, latency_p90, lib,
                      make_config, moe_build_united, moe_config, moe_distill_united, moe_forward, moe_route,
                      moe_route_static, pack_gate, probe_hbm_read, probe_mfma, profile_collect, profile_disable,
                      profile_enable, salc_update, with_packed_gate, workspace_size)

from .layer import (KvCache, NormOut, Rope, alloc_attention_workspace, alloc_kv_cache, alloc_linear_workspace, alloc_norm_out, make_rope,
                    moe_linear_e4m3, moe_paged_attention, moe_quantize_rows, moe_quantize_weight, moe_rms_norm, moe_rope_append,
                    rope_frequencies)
from .draft import (Logprobs, alloc_chunk_workspace, alloc_logprob_workspace, alloc_logprobs, moe_cache_move, moe_chunk_attention, moe_rope_append_at,
                    moe_sink_attention, moe_token_logprobs, tree_masks)

__all__ = ["MoeError", "RouteOut", "alloc_route_out", "alloc_workspace", "config_of", "init", "latency_p90", "lib",
           "make_config", "moe_build_united", "moe_config", "moe_distill_united", "moe_forward", "moe_route",
           "moe_route_static", "pack_gate", "probe_hbm_read", "probe_mfma", "profile_collect", "profile_disable",
           "profile_enable", "salc_update", "with_packed_gate", "workspace_size",
           "KvCache", "NormOut", "Rope", "alloc_attention_workspace", "alloc_kv_cache", "alloc_linear_workspace", "alloc_norm_out",
           "make_rope", "moe_linear_e4m3", "moe_paged_attention", "moe_quantize_rows", "moe_quantize_weight", "moe_rms_norm",
           "moe_rope_append", "rope_frequencies",
           "Logprobs", "alloc_chunk_workspace", "alloc_logprob_workspace", "alloc_logprobs", "moe_cache_move", "moe_chunk_attention",
           "moe_rope_append_at", "moe_sink_attention", "moe_token_logprobs", "tree_masks"]
