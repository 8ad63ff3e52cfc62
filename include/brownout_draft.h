/*
 * brownout_draft.h -- C ABI of the operators of a step with several new tokens of a sequence (drafted trees of tokens that are checked in one
 * pass, chunks of prompts), of attention with sinks, and of what a model answers (same library, libbrownout_moe.so):
 *
 *   moe_rope_append_at -> moe_chunk_attention -> ... -> moe_token_logprobs -> moe_cache_move
 *
 * A tree's tokens are appended one behind the other, whatever their depth, attend to the cached context and to their ancestors, and are judged by
 * their log probabilities; the accepted path is moved to where its tokens belong, and the next step writes over the rest.
 *
 * Conventions: those of brownout_layer.h, for the cache and its block tables too.  Unless said otherwise a block table's token_row here is the row of
 * each *sequence* of the call (NULL: sequence b has row b).
 */
#ifndef BROWNOUT_DRAFT_H
#define BROWNOUT_DRAFT_H

#include "brownout_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits (MOE_ERR_UNSUPPORTED beyond). */
#define MOE_MAX_TOP 64                        /* alternatives of a row */
#define MOE_MAX_GIVEN 64                      /* given tokens of a row */
#define MOE_MAX_ENTRIES (1 << 20)             /* logits of a row */
#define MOE_MAX_TREE 4096                     /* tokens of a tree */

/*
 * moe_paged_attention with a window and sinks: token t attends to the last `window` of its lengths[t] positions and to those below `sinks`,
 *   [0, min(sinks, lengths[t])) and [max(0, lengths[t] - window), lengths[t]);
 * window 0: to all of them.  sinks 0 is moe_paged_attention, bit for bit.  For single tokens of many sequences (token_row is each token's); everything
 * else, the workspace (moe_attention_workspace_size) too, as there.  sinks < 0: MOE_ERR_INVALID_ARG.
 */
moe_status moe_sink_attention(const moe_kv_cache *cache, const moe_block_table *table, const void *q, int64_t q_stride,
                              int32_t n_heads, int32_t T, const int32_t *lengths, float scale, int32_t window, int32_t sinks, void *out,
                              int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * moe_rope_append with the place apart from the position: q and k are turned by positions[t], and k and v go to position places[t] of the token's row
 * of the block table (token_row is each token's).  Siblings in a tree have the same position and places of their own.  A negative place stores
 * nothing, q_out is written as usual; a negative position is padding, as there.
 */
moe_status moe_rope_append_at(const moe_kv_cache *cache, const moe_block_table *table, const moe_rope *rope, const void *q,
                              int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                              int32_t n_heads, int32_t T, const int32_t *positions, const int32_t *places, void *q_out,
                              int64_t q_out_stride, void *stream);

/*
 * Host function: what a tree of n tokens is to moe_chunk_attention.  parents[i] < i is token i's parent, or -1: the last token of the context.
 * seen [n][words]: bit j % 32 of word j / 32 of row i is set if j is i or an ancestor of i; words >= ceil(n/32).  depth [n]: number of ancestors (a token's
 * position is the context's length plus its depth).  Either may be NULL.  Errors: n < 0 or a parent out of its range (MOE_ERR_INVALID_ARG), too few
 * words (MOE_ERR_SHAPE), n > MOE_MAX_TREE.
 */
moe_status moe_tree_masks(const int32_t *parents, int32_t n, int32_t words, uint32_t *seen, int32_t *depth);

/*
 * The same for a model whose layers see a window: of a token's ancestors those that it and the sinks leave it, depth[i] - depth[j] < window or depth[j] < sinks (window 0: all).
 * `sinks`: positions behind the context that are sinks yet, which is the model's number of them less the context's length if that is positive.  With these bits
 * a token of a tree sees what it would see at its position of a sequence.  window or sinks < 0: MOE_ERR_INVALID_ARG.
 */
moe_status moe_tree_window_masks(const int32_t *parents, int32_t n, int32_t words, int32_t window, int32_t sinks, uint32_t *seen, int32_t *depth);

/*
 * Attention of sequences' new tokens over the paged cache, each sequence's cache read once for all of them.  Sequence b has context[b] positions in the cache and
 * n_b = first[b+1] - first[b] new tokens, the rows first[b] .. of q; new token j's key and value are already at position context[b] + j.
 *   out[t][h] = sum_p softmax_p(scale * q[t][h] . k[p][h / group]) v[p][h / group]   over the positions p that token t sees:
 * A chunk (seen NULL): the j-th new token is at position P = context[b] + j and sees the positions p <= P with p > P - window or p < sinks
 *   (window 0: all p <= P).
 * A tree (seen not NULL): the token is at position P = positions[t] (NULL: context[b] + j) and sees of the context the positions p with p > P - window or
 *   p < sinks (window 0: all), and of the new tokens those whose bit is set in its row of `seen`: bits say what the window leaves of them, too (moe_tree_window_masks;
 *   those of moe_tree_masks let a path longer than the window see all of itself).  Bits of tokens that the sequence does not have count for nothing, nor do
 *   tokens beyond 32 * seen_words.  P < context[b] counts as context[b].
 * Positions whose page is not there (see moe_block_table) or that lie beyond max_pages * page_size are left out.  A token that sees nothing has
 * out = 0 and lse = -infinity.  What the cache holds in places that a token does not see does not matter to it, NaN included.
 *   first [n_seqs+1], context [n_seqs], positions [T] int32; seen [T][seen_words] uint32, rows seen_stride words apart; table's token_row [n_seqs]
 *   q [T][n_heads][head_dim] bf16, out, lse: as in moe_paged_attention.
 * first does not decrease and lies within [0, T] (beyond it is cut off there); tokens of no sequence (below first[0], from first[n_seqs] on) are left
 * as they are.  A negative context counts as 0.
 * Scores, softmax and sums are fp32.  For the product with v a probability is rounded to fp16 (2^-11 of it) beside an 8-bit cache.  Beside a bf16 cache it is held as two
 * bf16 (2^-15), as in moe_paged_attention, in calls with T * n_heads / n_kv_heads <= 128 * n_seqs, and rounded to one (2^-8) in those of more rows, where the second product costs a quarter of
 * the time.
 * The workspace (moe_chunk_workspace_size: for up to n_seqs sequences and T tokens, 256-byte aligned) needs no initialisation.  head_dim 128: 17 MB for up to 32 rows (tokens times
 * n_heads / n_kv_heads), 34 for up to 128, 68 beyond.
 * Tiles of rows go by the call's mean, T / n_seqs: a long chunk beside many single tokens is better a call of its own.  So is one sequence far longer than the others of a call of more than 1024: there
 * each tile has one block per key head, and is not shared out.
 * Limits: head_dim 64, 96, 128, 192 or 256; n_heads a multiple of n_kv_heads, at most MOE_MAX_HEADS; T <= 65536, n_seqs <= 65536, seen_words <= 128.
 */
typedef struct moe_chunk {
    const int32_t *first, *context;
    const uint32_t *seen; int64_t seen_stride;
    const int32_t *positions;                 /* trees only */
    int32_t seen_words, n_seqs, T, window, sinks;
} moe_chunk;
moe_status moe_chunk_workspace_size(const moe_kv_cache *cache, int32_t n_seqs, int32_t T, int32_t n_heads, size_t *bytes);
moe_status moe_chunk_attention(const moe_kv_cache *cache, const moe_block_table *table, const moe_chunk *chunk, const void *q,
                               int64_t q_stride, int32_t n_heads, float scale, void *out, int64_t out_stride, float *lse,
                               void *workspace, size_t workspace_bytes, void *stream);

/*
 * Moves keys and values of accepted tokens: for each sequence b and j < min(count[b], max_moves), what position sources[b][j] of its row of the block table
 * holds goes to position start[b] + j.  Sources increase and none lies before its target, so that no target is a later source; an entry that is
 * negative, not above all entries before it, or before its target, is not followed and its target keeps what it held.  Nor is anything moved whose source
 * or target has no page.  No two sequences move to the same place, and none moves from where another moves to.
 *   sources [n_seqs][max_moves] int32, rows sources_stride apart; start, count [n_seqs] int32; a count below 0 is 0
 * Rows of the cache are moved as they are, the scales of an 8-bit cache are per head.  Limits: n_seqs <= 65536, max_moves <= MOE_MAX_TREE,
 * n_kv_heads * head_dim <= 2^18; head_dim's bytes a multiple of 16 (MOE_ERR_SHAPE).
 */
moe_status moe_cache_move(const moe_kv_cache *cache, const moe_block_table *table, const int32_t *sources, int64_t sources_stride,
                          int32_t max_moves, const int32_t *start, const int32_t *count, int32_t n_seqs, void *stream);

/*
 * What rows of logits x say:  lse = log sum_i exp(x_i),   logprob of a token g = x_g - lse,   rank = entries before it in the order of falling x, equal
 * ones by rising number,   entropy = -sum_i p_i log p_i with p_i = exp(x_i - lse), 0 log 0 = 0;   and the first n_top entries of that order.
 *   logits [T][V] bf16 or fp32 (MOE_LOGITS_*), rows `stride` apart, aligned to their type only
 *   tokens [T][n_given] int32, rows tokens_stride apart (n_given 0: NULL); one outside [0, V) is no token: log probability 0, rank -1
 *   logprob [T][n_given] fp32, rank [T][n_given] int32; lse, entropy [T] fp32; top_id [T][n_top] int32, top_logprob [T][n_top] fp32, all dense; each
 *   may be NULL and is not written then.  They overlap neither the inputs nor each other.
 * Entries of -infinity have probability 0.  A row of nothing else has lse = -infinity, entropy 0, and -infinity for the log probability of each of its
 * entries.  A row that holds a NaN or +infinity has no distribution: all its fp32 results are NaN, its ids and ranks -1 (that of no token: 0 and -1).
 * Sums are fp32, entropy from values relative to the largest.  A row is read once, by as many blocks as the call needs to fill the GPU, and joined in a
 * fixed order; a row's results may differ in the last bits with T.
 * The workspace (moe_logprob_workspace_size: for up to T rows, V entries; 256-byte aligned) needs no initialisation.
 * Limits: V <= MOE_MAX_ENTRIES, n_top <= MOE_MAX_TOP and V, n_given <= MOE_MAX_GIVEN, T <= MOE_MAX_ROWS.
 */
#define MOE_LOGITS_BF16 0
#define MOE_LOGITS_FP32 1
typedef struct moe_logprob_args {
    const void *logits; int64_t stride;
    const int32_t *tokens; int64_t tokens_stride;
    float *logprob; int32_t *rank;
    float *lse, *entropy;
    int32_t *top_id; float *top_logprob;
    int32_t T, V, type, n_given, n_top;
} moe_logprob_args;
moe_status moe_logprob_workspace_size(int32_t T, int32_t V, int32_t n_given, int32_t n_top, size_t *bytes);
moe_status moe_token_logprobs(const moe_logprob_args *a, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BROWNOUT_DRAFT_H */
