/*
 * brownout_layer.h -- C ABI of the operators around the BrownoutMoE layer in a decoder layer (same library,
 * libbrownout_moe.so): the norm with its residual and 8-bit output, a linear layer in 8-bit floating point,
 * rotary positions with the append to a paged key-value cache, and the attention of new tokens over that cache.
 *
 *   norm -> linear (q, k, v) -> rotary + append -> attention -> quantise -> linear (o) -> norm + residual -> moe_forward
 *
 * Conventions: those of brownout_moe.h (device pointers of the caller, caller's stream and workspace, no host
 * synchronisation, arguments checked on the host before any launch, a moe_status from every call).  Besides:
 *   - bf16 is rounded to nearest even; e4m3 is the 8-bit type with 4 exponent and 3 mantissa bits, no infinities and
 *     a largest value of 448, rounded to nearest even.  Sums, softmax statistics and scales are fp32 (but for what the 8-bit matrix
 *     instructions add up within 8 products: moe_linear_e4m3).
 *   - Strides are in elements of their tensor and may exceed what the shape needs (slices of wider tensors); the last
 *     dimension is contiguous.  Pointers are 16-byte aligned, and so is every row that a stride leads to (8 bytes where
 *     it says so); pointers to int32, fp32 and fp64 arrays need the alignment of their type.
 *   - T == 0 (M == 0) is a valid call that does nothing; the block table of an empty batch may have no rows.
 *   - The calls work per row: a token's result has the same bits whatever other tokens are in the call, with two
 *     exceptions, where the way that a sum is split goes by the whole call: moe_paged_attention and moe_linear_e4m3.
 *     The same call gives the same bits every time.
 */
#ifndef BROWNOUT_LAYER_H
#define BROWNOUT_LAYER_H

#include "brownout_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits (MOE_ERR_UNSUPPORTED beyond). */
#define MOE_NORM_MAX_D 16384
#define MOE_MAX_HEADS 1024
#define MOE_MAX_ROWS (1 << 21)                /* rows (tokens) of a call */

/*
 * Root-mean-square norm of T rows of d columns with the residual's addition:
 *   h = x + residual (fp32; h = x without one)      residual_out = bf16(h)
 *   y = h / sqrt(mean(h^2) + eps) * weight          of the unrounded h
 * y may come out in bf16 (`y`), in e4m3 with scales (`y8`, `scale`: as moe_quantize_rows makes them of the unrounded
 * y), or both; a pointer left NULL is not written, at least one must be there.  residual_out is written if it is not NULL
 * (allowed without a residual: a copy of x) and may be the same tensor as x or residual; the other outputs may not
 * overlap the inputs.
 *   x, residual, residual_out, y  [T][d] bf16, row strides multiples of 8;  weight [d] bf16 or NULL (ones)
 *   y8 [T][d] e4m3 with 8-byte aligned rows;  scale [ceil(d/128)][scale_stride >= T] fp32
 * Limits: d a multiple of 8 (MOE_ERR_SHAPE), d <= MOE_NORM_MAX_D, T <= MOE_MAX_ROWS.
 */
typedef struct moe_norm_args {
    const void *x; int64_t x_stride;
    const void *residual; int64_t residual_stride;
    const void *weight;
    void *residual_out; int64_t residual_out_stride;
    void *y; int64_t y_stride;
    void *y8; int64_t y8_stride;
    float *scale; int64_t scale_stride;
    int32_t T, d;
    float eps;
} moe_norm_args;
moe_status moe_rms_norm(const moe_norm_args *a, void *stream);

/*
 * The 8-bit form alone.  Each row's groups of 128 columns (the last one may have fewer) get a scale
 *   s = max(largest |y| of the group, 2^-100) / 448,    y8 = e4m3(y / s),
 * so that y8 * s stands for y.  A group that holds a NaN or an infinity stands for NaN throughout (y8 * s).
 * Of `a`, x, y8, scale, T and d are used; the other pointers must be NULL.
 */
moe_status moe_quantize_rows(const moe_norm_args *a, void *stream);

/*
 * A weight [N][K] bf16 (dense) in e4m3 with one scale per block of 128 x 128, by the same rule: w8 [N][K] dense,
 * w_scale [ceil(N/128)][ceil(K/128)].  Done once per weight.  K a multiple of 16 (MOE_ERR_SHAPE).
 */
moe_status moe_quantize_weight(const void *w, int32_t N, int32_t K, void *w8, float *w_scale, void *stream);

/*
 * out[m][n] = bf16( sum over blocks b of 128 columns of x_scale[b][m] * w_scale[n/128][b] * sum_{k in b} x8[m][k] w8[n][k] )
 *   x8 [M][K] e4m3, rows x_stride apart (a multiple of 16); x_scale [ceil(K/128)][x_scale_stride >= M] (as moe_rms_norm
 *   and moe_quantize_rows write them); w8 [N][K] e4m3 dense; w_scale [ceil(N/128)][ceil(K/128)];
 *   out [M][N] bf16, rows out_stride apart (any; 2-byte aligned).
 * Blocks are scaled and added up in fp32.  Up to K = 512, and for every K where `exact` is not 0, products are exact and their sums fp32.  Else a
 * block goes through the 8-bit matrix instructions, which add up 8 neighbouring columns at a time: each product is cut off toward zero at 2^-13
 * of 2^e, e the largest sum of two exponents among the 8, and what the groups give is added in fp32.  So at most 7 * 2^-13 of its largest
 * product is lost of a group: around 1e-5 of sum |x||w| for values of like size, up to some 1e-4 of the largest where one column is
 * hundreds of times larger than its neighbours.  `exact` takes up to 2.2 times as long (many rows), for up to 64 rows 1.05 to 1.2.
 * K a multiple of 16 (MOE_ERR_SHAPE); M <= MOE_MAX_ROWS, N, K <= 2^20, x_stride <= 2^23 (MOE_ERR_UNSUPPORTED).  out overlaps no
 * input.  The workspace holds partial sums where the work is split along K: moe_linear_workspace_size bytes (0 for many shapes) for
 * exactly this M, N, K, 256-byte aligned.  The size is not monotone in M (large products are not split): a workspace kept for
 * batches of changing size has moe_linear_workspace_bound bytes, enough for every M up to M_max with this N and K.
 */
typedef struct moe_linear_args {
    const void *x8; int64_t x_stride;
    const float *x_scale; int64_t x_scale_stride;
    const void *w8;
    const float *w_scale;
    void *out; int64_t out_stride;
    int32_t M, N, K;
    int32_t exact;                            /* 0, or 1: exact products and fp32 sums for every K */
} moe_linear_args;
moe_status moe_linear_workspace_size(int32_t M, int32_t N, int32_t K, size_t *bytes);
moe_status moe_linear_workspace_bound(int32_t M_max, int32_t N, int32_t K, size_t *bytes);
moe_status moe_linear_e4m3(const moe_linear_args *a, void *workspace, size_t workspace_bytes, void *stream);

/*
 * A paged key-value cache: n_pages pages of page_size tokens, each with n_kv_heads vectors of head_dim.  The element
 * (page, token, head, i) of k (and of v) is at page*page_stride + token*token_stride + head*head_stride + i, so pages
 * may be stored token by token or head by head.  Strides are 16-byte multiples.
 * A sequence's block table row lists the pages of its positions 0, page_size, 2*page_size, ...
 * With type MOE_KV_E4M3 a stored value c of head h stands for c * k_scale[h] (v_scale[h]); with MOE_KV_BF16 the scales
 * are ignored.  k and v span at most 64 GiB each (MOE_ERR_UNSUPPORTED beyond).
 */
#define MOE_KV_BF16 0
#define MOE_KV_E4M3 1
typedef struct moe_kv_cache {
    void *k, *v;
    int64_t page_stride, token_stride, head_stride;
    const float *k_scale, *v_scale;           /* [n_kv_heads], MOE_KV_E4M3 only */
    int32_t type, n_pages, page_size, n_kv_heads, head_dim;
} moe_kv_cache;

/* The sequences' block tables, [n_rows][max_pages] int32, rows row_stride apart.  token_row [T]: row of each token of
 * the call; NULL: token t has row t.  An entry of a block table outside [0, n_pages), or a token's row outside
 * [0, n_rows), is not followed: see the calls. */
typedef struct moe_block_table {
    const int32_t *pages; int64_t row_stride;
    const int32_t *token_row;
    int32_t n_rows, max_pages;
} moe_block_table;

/*
 * Rotary positions.  Pair i of a head's first rotary_dim columns is turned by pos * turns[i] whole turns (fp64, so that
 * far positions keep their angle); cos and sin are multiplied by factor.  Pairs are (i, i + rotary_dim/2), or with
 * interleaved != 0 (2i, 2i+1).  Columns from rotary_dim on are passed on; rotary_dim 0: all are.
 */
typedef struct moe_rope {
    const double *turns;                      /* [rotary_dim/2], device */
    int32_t rotary_dim, interleaved;
    float factor;
} moe_rope;

/*
 * Host function: turns[i] = base^(-2i/rotary_dim) / 2pi for i < rotary_dim/2 (host array), and the factor for moe_rope,
 * scaled for contexts that are `factor` times the trained one of original_length positions:
 *   MOE_ROPE_NONE    as above                         MOE_ROPE_LINEAR  every frequency divided by factor
 *   MOE_ROPE_NTK     base * factor^(R/(R-2)) in place of base, R = rotary_dim (R = 2: base)
 *   MOE_ROPE_YARN    pairs that make more than beta_fast turns over original_length keep their frequency, those of
 *                    fewer than beta_slow have it divided, a linear ramp over the pair's index between; the factor on cos and sin is 0.1 ln(factor) + 1
 * Errors: rotary_dim < 2 or odd, base <= 1, factor < 1, original_length <= 0, betas not beta_fast > beta_slow > 0.
 */
#define MOE_ROPE_NONE 0
#define MOE_ROPE_LINEAR 1
#define MOE_ROPE_NTK 2
#define MOE_ROPE_YARN 3
typedef struct moe_rope_scaling {
    int32_t kind;
    double factor, original_length, beta_fast, beta_slow;   /* NONE uses none; LINEAR, NTK the factor; YARN all */
} moe_rope_scaling;
moe_status moe_rope_frequencies(int32_t rotary_dim, double base, const moe_rope_scaling *scaling, double *turns, float *factor);

/*
 * Rotates q and k of T new tokens and writes k and v to the cache.
 *   q [T][n_heads][head_dim], k and v [T][n_kv_heads][head_dim] bf16: heads are head_dim apart, tokens q_stride, k_stride,
 *   v_stride (multiples of 8).  q_out: the rotated q, same layout, tokens q_out_stride apart; it may be q itself.
 *   positions [T] int32.  Token t is written to position positions[t] of its row of the block table; no two tokens of a
 *   call may name the same place.  In an 8-bit cache values beyond 448 scales are held as 448 scales.
 * A token of a negative position is padding: its q_out is zero, and nothing goes to the cache.  Nor does a token whose
 * page or row is not there (see moe_block_table, or a position beyond max_pages * page_size); its q_out is written as usual.
 * Errors: head_dim not a multiple of 16, rotary_dim not a multiple of 16 or beyond head_dim (MOE_ERR_SHAPE); head_dim > 256,
 * n_heads > MOE_MAX_HEADS, T > MOE_MAX_ROWS (MOE_ERR_UNSUPPORTED).
 */
moe_status moe_rope_append(const moe_kv_cache *cache, const moe_block_table *table, const moe_rope *rope, const void *q,
                           int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                           int32_t n_heads, int32_t T, const int32_t *positions, void *q_out, int64_t q_out_stride,
                           void *stream);

/*
 * Attention of T new tokens, each over its own row of the block table:
 *   out[t][h] = sum_p softmax_p(scale * q[t][h] . k[p][h / group]) v[p][h / group],   group = n_heads / n_kv_heads,
 * over the positions p of [0, lengths[t]), with window > 0 only the last `window` of them.  Positions whose page is not
 * there (see moe_block_table) are left out; lengths beyond max_pages * page_size end there.  A token with no position left
 * has out = 0 and lse = -infinity.  What the cache holds in places that are left out does not matter, NaN included.
 *   q [T][n_heads][head_dim] bf16, tokens q_stride apart (a multiple of 8); out the same, out_stride (a multiple of 4, 8-byte aligned); no row
 *   of out shares memory with one of q (MOE_ERR_INVALID_ARG)
 *   lse [T][n_heads] fp32 or NULL: log of the sum of exp(scale * q . k), to join attention over several caches
 * The tokens of a prompt's chunk are T rows with lengths position + 1, appended first.
 * Scores and sums are fp32; for the product with v a probability is two bf16 that add up to it within 2^-15 of it.
 * The workspace (moe_attention_workspace_size: for up to T_max tokens of n_heads heads on such a cache, 256-byte aligned) needs no
 * initialisation.  Every token's cache is cut into equal shares of the call's whole work, so one long sequence among
 * short ones is shared by the whole GPU.
 * Limits: head_dim 64, 96, 128, 192 or 256; n_heads a multiple of n_kv_heads, at most MOE_MAX_HEADS; T <= 65536.
 */
moe_status moe_attention_workspace_size(const moe_kv_cache *cache, int32_t T_max, int32_t n_heads, size_t *bytes);
moe_status moe_paged_attention(const moe_kv_cache *cache, const moe_block_table *table, const void *q, int64_t q_stride,
                               int32_t n_heads, int32_t T, const int32_t *lengths, float scale, int32_t window, void *out,
                               int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BROWNOUT_LAYER_H */
