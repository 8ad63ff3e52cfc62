// Internal declarations of the operators of a step with several new tokens of a sequence (chunk.hip, move.hip, logprob.hip, draft_api.hip).
#pragma once
#include "../../include/brownout_draft.h"
#include "layer.h"

namespace bmoe {

// The largest of three, in one instruction (fmaxf first makes sure that what it is given is no signalling NaN, an instruction each).  NaN only if all are.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// layer_api.hip
bool off(const void* p, unsigned bytes);                           // not aligned to so many bytes
bool bad_stride(int64_t stride, int unit);
bool rows_meet(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int T, int64_t width);
moe_status check_cache(const moe_kv_cache* c);
moe_status check_table(const moe_block_table* t, int32_t rows);
moe_status check_attention(const moe_kv_cache* c, int32_t n_heads, int32_t T);
// The whole calls, for the entry points with and without sinks, and with places of their own (`apart`) or not.
moe_status attention_call(const moe_kv_cache* cache, const moe_block_table* table, const void* q, int64_t q_stride, int32_t n_heads, int32_t T,
                          const int32_t* lengths, float scale, int32_t window, int32_t sinks, void* out, int64_t out_stride, float* lse, void* workspace,
                          size_t workspace_bytes, void* stream, const char* name);
moe_status rope_call(const moe_kv_cache* cache, const moe_block_table* table, const moe_rope* rope, const void* q, int64_t q_stride, const void* k,
                     int64_t k_stride, const void* v, int64_t v_stride, int32_t n_heads, int32_t T, const int32_t* positions, const int32_t* places,
                     bool apart, void* q_out, int64_t q_out_stride, void* stream, const char* name);

hipError_t init_chunk_kernels();
size_t chunk_workspace_bytes(const moe_kv_cache& c, int T, int n_heads);
hipError_t launch_chunk(const moe_kv_cache& c, const moe_block_table& t, const moe_chunk& ch, const bf16_t* q, int64_t q_stride, int n_heads, float scale,
                        bf16_t* out, int64_t out_stride, float* lse, void* ws, hipStream_t s);

hipError_t launch_move(const moe_kv_cache& c, const moe_block_table& t, const int32_t* sources, int64_t sources_stride, int max_moves, const int32_t* start,
                       const int32_t* count, int n_seqs, hipStream_t s);

size_t logprob_workspace_bytes(int64_t T, int V, int n_given, int n_top);
hipError_t launch_logprobs(const moe_logprob_args& a, void* ws, hipStream_t s);

}  // namespace bmoe
