// C ABI of the operators of a step with several new tokens of a sequence: argument checks, then the launch.
#include "draft.h"

#include <cmath>

namespace bmoe {
namespace {

constexpr int32_t kMostSeqs = 65536, kMostWords = MOE_MAX_TREE / 32;

moe_status check_logprobs(int32_t T, int32_t V, int32_t n_given, int32_t n_top)
{
    if (T < 0 || n_given < 0 || n_top < 0) return MOE_ERR_INVALID_ARG;
    if (V < 1 || n_top > V) return MOE_ERR_SHAPE;
    if (T > MOE_MAX_ROWS || V > MOE_MAX_ENTRIES || n_given > MOE_MAX_GIVEN || n_top > MOE_MAX_TOP) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

}  // namespace
}  // namespace bmoe

using namespace bmoe;

extern "C" {

moe_status moe_sink_attention(const moe_kv_cache* cache, const moe_block_table* table, const void* q, int64_t q_stride,
                              int32_t n_heads, int32_t T, const int32_t* lengths, float scale, int32_t window, int32_t sinks, void* out,
                              int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    return attention_call(cache, table, q, q_stride, n_heads, T, lengths, scale, window, sinks, out, out_stride, lse, workspace, workspace_bytes, stream,
                          "moe_sink_attention");
}

moe_status moe_rope_append_at(const moe_kv_cache* cache, const moe_block_table* table, const moe_rope* rope, const void* q,
                              int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                              int32_t n_heads, int32_t T, const int32_t* positions, const int32_t* places, void* q_out,
                              int64_t q_out_stride, void* stream)
{
    return rope_call(cache, table, rope, q, q_stride, k, k_stride, v, v_stride, n_heads, T, positions, places, true, q_out, q_out_stride, stream,
                     "moe_rope_append_at");
}

moe_status moe_tree_masks(const int32_t* parents, int32_t n, int32_t words, uint32_t* seen, int32_t* depth)
{
    return moe_tree_window_masks(parents, n, words, 0, 0, seen, depth);
}

moe_status moe_tree_window_masks(const int32_t* parents, int32_t n, int32_t words, int32_t window, int32_t sinks, uint32_t* seen, int32_t* depth)
{
    if (n < 0 || window < 0 || sinks < 0) return MOE_ERR_INVALID_ARG;
    if (n > MOE_MAX_TREE) return MOE_ERR_UNSUPPORTED;
    if (n == 0) return MOE_OK;
    if (!parents) return MOE_ERR_INVALID_ARG;
    if (seen && words < (n + 31) / 32) return MOE_ERR_SHAPE;
    for (int32_t i = 0; i < n; ++i)
        if (parents[i] < -1 || parents[i] >= i) return MOE_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        const int32_t up = parents[i];
        if (depth) depth[i] = up < 0 ? 0 : depth[up] + 1;
        if (!seen) continue;
        uint32_t* row = seen + (int64_t)i * words;
        // the parent's, and the token itself
        for (int32_t w = 0; w < words; ++w) row[w] = up < 0 ? 0 : seen[(int64_t)up * words + w];
        row[i / 32] |= 1u << (i % 32);
        if (window == 0) continue;
        // the ancestor that the parent sees and the token does not: `window` levels up, at level `of`
        int32_t level = 0, at = i, of = 0;
        for (; at >= 0 && level < window; ++level) at = parents[at];
        if (at < 0) continue;
        for (int32_t j = parents[at]; j >= 0; j = parents[j]) ++of;
        if (of >= sinks) row[at / 32] &= ~(1u << (at % 32));
    }
    return MOE_OK;
}

moe_status moe_chunk_workspace_size(const moe_kv_cache* cache, int32_t n_seqs, int32_t T, int32_t n_heads, size_t* bytes)
{
    moe_status st = check_attention(cache, n_heads, T);
    if (st != MOE_OK) return st;
    if (n_seqs < 0 || !bytes) return MOE_ERR_INVALID_ARG;
    if (n_seqs > kMostSeqs) return MOE_ERR_UNSUPPORTED;
    *bytes = chunk_workspace_bytes(*cache, T, n_heads);
    // a caller sizes its workspace before its first launch: the per-device set-up is done then, ahead of any stream capture
    if (ensure_device_init(nullptr) != hipSuccess) (void)hipGetLastError();
    return MOE_OK;
}

moe_status moe_chunk_attention(const moe_kv_cache* cache, const moe_block_table* table, const moe_chunk* chunk, const void* q,
                               int64_t q_stride, int32_t n_heads, float scale, void* out, int64_t out_stride, float* lse,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    if (!chunk) return MOE_ERR_INVALID_ARG;
    const int32_t T = chunk->T, n_seqs = chunk->n_seqs;
    moe_status st = check_attention(cache, n_heads, T);
    if (st != MOE_OK) return st;
    if (n_seqs < 0 || chunk->window < 0 || chunk->sinks < 0 || !std::isfinite(scale)) return MOE_ERR_INVALID_ARG;
    if (n_seqs > kMostSeqs) return MOE_ERR_UNSUPPORTED;
    if (chunk->seen ? chunk->seen_words < 1 : chunk->positions || chunk->seen_words) return MOE_ERR_INVALID_ARG;
    if (chunk->seen_words > kMostWords) return MOE_ERR_UNSUPPORTED;
    if (T == 0 || n_seqs == 0) return MOE_OK;                // an empty batch's table has no rows
    if ((st = check_table(table, n_seqs)) != MOE_OK) return st;
    if (!q || !out || !chunk->first || !chunk->context) return MOE_ERR_INVALID_ARG;
    if (off(q, 16) || off(chunk->first, 4) || off(chunk->context, 4) || off(chunk->seen, 4) || off(chunk->positions, 4) || off(out, 8) || off(lse, 4) ||
        bad_stride(q_stride, 8) || bad_stride(out_stride, 4))
        return MOE_ERR_ALIGNMENT;
    if ((T > 1 && out_stride < (int64_t)n_heads * cache->head_dim) || (chunk->seen && T > 1 && chunk->seen_stride < chunk->seen_words)) return MOE_ERR_SHAPE;
    if (!workspace || workspace_bytes < chunk_workspace_bytes(*cache, T, n_heads)) return MOE_ERR_WORKSPACE;
    if (off(workspace, 256)) return MOE_ERR_ALIGNMENT;
    // blocks read a token's q where others have written its out
    if (rows_meet(q, 2 * q_stride, out, 2 * out_stride, T, (int64_t)2 * n_heads * cache->head_dim)) return MOE_ERR_INVALID_ARG;
    hipError_t e = ensure_device_init(nullptr);
    if (e != hipSuccess) return hip_fail(e, "moe_chunk_attention/init");
    e = launch_chunk(*cache, *table, *chunk, static_cast<const bf16_t*>(q), q_stride, n_heads, scale, static_cast<bf16_t*>(out), out_stride, lse, workspace,
                     static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_chunk_attention");
}

moe_status moe_cache_move(const moe_kv_cache* cache, const moe_block_table* table, const int32_t* sources, int64_t sources_stride,
                          int32_t max_moves, const int32_t* start, const int32_t* count, int32_t n_seqs, void* stream)
{
    moe_status st = check_cache(cache);
    if (st != MOE_OK) return st;
    if (n_seqs < 0 || max_moves < 0) return MOE_ERR_INVALID_ARG;
    if (cache->head_dim * (cache->type == MOE_KV_E4M3 ? 1 : 2) % 16 != 0) return MOE_ERR_SHAPE;
    if (n_seqs > kMostSeqs || max_moves > MOE_MAX_TREE || (int64_t)cache->n_kv_heads * cache->head_dim > (1 << 18)) return MOE_ERR_UNSUPPORTED;
    if (n_seqs == 0 || max_moves == 0) return MOE_OK;
    if ((st = check_table(table, n_seqs)) != MOE_OK) return st;
    if (!sources || !start || !count) return MOE_ERR_INVALID_ARG;
    if (off(sources, 4) || off(start, 4) || off(count, 4)) return MOE_ERR_ALIGNMENT;
    if (sources_stride < 0 || (n_seqs > 1 && sources_stride < max_moves)) return MOE_ERR_SHAPE;
    hipError_t e = launch_move(*cache, *table, sources, sources_stride, max_moves, start, count, n_seqs, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_cache_move");
}

moe_status moe_logprob_workspace_size(int32_t T, int32_t V, int32_t n_given, int32_t n_top, size_t* bytes)
{
    moe_status st = check_logprobs(T, V, n_given, n_top);
    if (st != MOE_OK) return st;
    if (!bytes) return MOE_ERR_INVALID_ARG;
    *bytes = T > 0 ? logprob_workspace_bytes(T, V, n_given, n_top) : 0;
    return MOE_OK;
}

moe_status moe_token_logprobs(const moe_logprob_args* a, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!a || (a->type != MOE_LOGITS_BF16 && a->type != MOE_LOGITS_FP32)) return MOE_ERR_INVALID_ARG;
    moe_status st = check_logprobs(a->T, a->V, a->n_given, a->n_top);
    if (st != MOE_OK || a->T == 0) return st;
    if (!a->logits || (a->n_given > 0 && !a->tokens)) return MOE_ERR_INVALID_ARG;
    const unsigned size = a->type == MOE_LOGITS_FP32 ? 4 : 2;
    if (off(a->logits, size) || off(a->tokens, 4) || off(a->logprob, 4) || off(a->rank, 4) || off(a->lse, 4) || off(a->entropy, 4) || off(a->top_id, 4) ||
        off(a->top_logprob, 4))
        return MOE_ERR_ALIGNMENT;
    if (a->stride < 0 || (a->T > 1 && a->stride < a->V) || (a->n_given > 0 && (a->tokens_stride < 0 || (a->T > 1 && a->tokens_stride < a->n_given)))) return MOE_ERR_SHAPE;
    if (!workspace || workspace_bytes < logprob_workspace_bytes(a->T, a->V, a->n_given, a->n_top)) return MOE_ERR_WORKSPACE;
    if (off(workspace, 256)) return MOE_ERR_ALIGNMENT;
    hipError_t e = launch_logprobs(*a, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_token_logprobs");
}

}  // extern "C"
