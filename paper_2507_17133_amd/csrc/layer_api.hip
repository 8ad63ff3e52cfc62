// C ABI of the operators around the MoE layer: argument checks, then the launch.
#include "layer.h"

#include <algorithm>
#include <cmath>

namespace bmoe {
namespace {

constexpr int32_t kMaxColumns = 1 << 20;                         // with MOE_MAX_ROWS: tile counts and grids stay within what launches take
constexpr int64_t kMaxRowBytes = (int64_t)1 << 23;               // a tile's offsets stay in 32 bits

bool off(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// A row stride of a tensor that is read: whole 16-byte (or `unit`-element) steps forward.
bool bad_stride(int64_t stride, int unit) { return stride < 0 || stride % unit != 0; }

// Whether a row of a shares memory with a row of b; T rows of `width` bytes each, strides in bytes, not negative.
bool rows_meet(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int T, int64_t width)
{
    const int64_t a0 = (int64_t)reinterpret_cast<uintptr_t>(a), b0 = (int64_t)reinterpret_cast<uintptr_t>(b);
    if (a0 + (T - 1) * a_stride + width <= b0 || b0 + (T - 1) * b_stride + width <= a0) return false;
    for (int i = 0, j = 0; i < T && j < T;) {
        const int64_t ai = a0 + i * a_stride, bj = b0 + j * b_stride;
        if (ai + width <= bj) ++i;
        else if (bj + width <= ai) ++j;
        else return true;
    }
    return false;
}

moe_status check_norm(const moe_norm_args* a, bool norm)
{
    if (!a || a->T < 0) return MOE_ERR_INVALID_ARG;
    if (a->d < 8 || a->d % 8 != 0) return MOE_ERR_SHAPE;
    if (a->d > MOE_NORM_MAX_D || a->T > MOE_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
    if (a->T == 0) return MOE_OK;
    if (!a->x || (a->y8 ? !a->scale : !a->y)) return MOE_ERR_INVALID_ARG;
    if (norm ? !(a->eps >= 0.0f && std::isfinite(a->eps)) : a->residual || a->weight || a->residual_out || a->y || !a->y8)
        return MOE_ERR_INVALID_ARG;
    if (off(a->x, 16) || off(a->residual, 16) || off(a->weight, 16) || off(a->residual_out, 16) || off(a->y, 16) || off(a->y8, 8) ||
        off(a->scale, 4))
        return MOE_ERR_ALIGNMENT;
    if (bad_stride(a->x_stride, 8) || (a->residual && bad_stride(a->residual_stride, 8)) ||
        (a->residual_out && bad_stride(a->residual_out_stride, 8)) || (a->y && bad_stride(a->y_stride, 8)) ||
        (a->y8 && bad_stride(a->y8_stride, 8)))
        return MOE_ERR_ALIGNMENT;
    // rows that are written do not overlap
    if (a->T > 1 && ((a->residual_out && a->residual_out_stride < a->d) || (a->y && a->y_stride < a->d) || (a->y8 && a->y8_stride < a->d)))
        return MOE_ERR_SHAPE;
    if (a->y8 && a->scale_stride < a->T) return MOE_ERR_SHAPE;
    return MOE_OK;
}

moe_status check_cache(const moe_kv_cache* c)
{
    if (!c || !c->k || !c->v || (c->type != MOE_KV_BF16 && c->type != MOE_KV_E4M3)) return MOE_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->head_dim < 1) return MOE_ERR_SHAPE;
    if (c->n_kv_heads > MOE_MAX_HEADS) return MOE_ERR_UNSUPPORTED;
    if (off(c->k, 16) || off(c->v, 16)) return MOE_ERR_ALIGNMENT;
    const int unit = c->type == MOE_KV_E4M3 ? 16 : 8;
    if (bad_stride(c->page_stride, unit) || bad_stride(c->token_stride, unit) || bad_stride(c->head_stride, unit)) return MOE_ERR_ALIGNMENT;
    if ((c->n_pages > 1 && c->page_stride < c->head_dim) || (c->page_size > 1 && c->token_stride < c->head_dim) ||
        (c->n_kv_heads > 1 && c->head_stride < c->head_dim))
        return MOE_ERR_SHAPE;
    // a position's place is held in 32 bits, in 16-byte steps
    constexpr int64_t most = 0xFFFFFFFF;
    const int64_t pages = c->n_pages - 1, positions = c->page_size - 1;
    const int64_t page_step = pages ? c->page_stride / unit : 0, token_step = positions ? c->token_stride / unit : 0;
    if (page_step > most / std::max<int64_t>(pages, 1) || token_step > most / std::max<int64_t>(positions, 1) ||
        page_step * pages + token_step * positions > most)
        return MOE_ERR_UNSUPPORTED;
    if (c->type == MOE_KV_E4M3) {
        if (!c->k_scale || !c->v_scale) return MOE_ERR_INVALID_ARG;
        if (off(c->k_scale, 4) || off(c->v_scale, 4)) return MOE_ERR_ALIGNMENT;
    }
    return MOE_OK;
}

moe_status check_table(const moe_block_table* t, int32_t T)
{
    if (!t || !t->pages) return MOE_ERR_INVALID_ARG;
    if (t->n_rows < 1 || t->max_pages < 1 || t->row_stride < 0) return MOE_ERR_SHAPE;
    if (!t->token_row && t->n_rows < T) return MOE_ERR_SHAPE;
    if (off(t->pages, 4) || off(t->token_row, 4)) return MOE_ERR_ALIGNMENT;
    return MOE_OK;
}

moe_status check_linear(int32_t M, int32_t N, int32_t K)
{
    if (M < 0) return MOE_ERR_INVALID_ARG;
    if (N < 1 || K < 16 || K % 16 != 0) return MOE_ERR_SHAPE;
    if (M > MOE_MAX_ROWS || N > kMaxColumns || K > kMaxColumns) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

bool attention_head_dim(int d) { return d == 64 || d == 96 || d == 128 || d == 192 || d == 256; }

moe_status check_attention(const moe_kv_cache* c, int32_t n_heads, int32_t T)
{
    moe_status st = check_cache(c);
    if (st != MOE_OK) return st;
    if (T < 0) return MOE_ERR_INVALID_ARG;
    if (n_heads < 1 || n_heads % c->n_kv_heads != 0) return MOE_ERR_SHAPE;
    if (n_heads > MOE_MAX_HEADS || T > 65536 || !attention_head_dim(c->head_dim)) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

}  // namespace
}  // namespace bmoe

using namespace bmoe;

extern "C" {

moe_status moe_rms_norm(const moe_norm_args* a, void* stream)
{
    moe_status st = check_norm(a, true);
    if (st != MOE_OK || a->T == 0) return st;
    hipError_t e = launch_norm(*a, true, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_rms_norm");
}

moe_status moe_quantize_rows(const moe_norm_args* a, void* stream)
{
    moe_status st = check_norm(a, false);
    if (st != MOE_OK || a->T == 0) return st;
    hipError_t e = launch_norm(*a, false, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_quantize_rows");
}

moe_status moe_quantize_weight(const void* w, int32_t N, int32_t K, void* w8, float* w_scale, void* stream)
{
    moe_status st = check_linear(0, N, K);
    if (st != MOE_OK) return st;
    if (!w || !w8 || !w_scale) return MOE_ERR_INVALID_ARG;
    if (off(w, 16) || off(w8, 16) || off(w_scale, 4)) return MOE_ERR_ALIGNMENT;
    hipError_t e = launch_quantize_weight(static_cast<const bf16_t*>(w), N, K, static_cast<uint8_t*>(w8), w_scale,
                                          static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_quantize_weight");
}

moe_status moe_linear_workspace_size(int32_t M, int32_t N, int32_t K, size_t* bytes)
{
    moe_status st = check_linear(M, N, K);
    if (st != MOE_OK) return st;
    if (!bytes) return MOE_ERR_INVALID_ARG;
    *bytes = M > 0 ? linear_workspace_bytes(linear_plan(M, N, K, false), M, N) : 0;
    // a caller sizes its workspace before its first launch: the per-device set-up is done then, ahead of any stream capture
    if (ensure_device_init(nullptr) != hipSuccess) (void)hipGetLastError();
    return MOE_OK;
}

moe_status moe_linear_workspace_bound(int32_t M_max, int32_t N, int32_t K, size_t* bytes)
{
    moe_status st = check_linear(M_max, N, K);
    if (st != MOE_OK) return st;
    if (!bytes) return MOE_ERR_INVALID_ARG;
    *bytes = linear_workspace_bound(M_max, N, K);
    if (ensure_device_init(nullptr) != hipSuccess) (void)hipGetLastError();      // as in moe_linear_workspace_size
    return MOE_OK;
}

moe_status moe_linear_e4m3(const moe_linear_args* a, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!a) return MOE_ERR_INVALID_ARG;
    moe_status st = check_linear(a->M, a->N, a->K);
    if (st != MOE_OK || a->M == 0) return st;
    if (!a->x8 || !a->x_scale || !a->w8 || !a->w_scale || !a->out) return MOE_ERR_INVALID_ARG;
    if (off(a->x8, 16) || off(a->w8, 16) || off(a->x_scale, 4) || off(a->w_scale, 4) || off(a->out, 2) || bad_stride(a->x_stride, 16))
        return MOE_ERR_ALIGNMENT;
    if (a->x_scale_stride < a->M || a->out_stride < 0 || (a->M > 1 && a->out_stride < a->N)) return MOE_ERR_SHAPE;
    if (a->x_stride > kMaxRowBytes) return MOE_ERR_UNSUPPORTED;
    const LinearPlan plan = linear_plan(a->M, a->N, a->K, a->exact != 0);
    const size_t need = linear_workspace_bytes(plan, a->M, a->N);
    if (need > 0 && (!workspace || workspace_bytes < need)) return MOE_ERR_WORKSPACE;
    if (need > 0 && off(workspace, 256)) return MOE_ERR_ALIGNMENT;
    hipError_t e = ensure_device_init(nullptr);
    if (e != hipSuccess) return hip_fail(e, "moe_linear_e4m3/init");
    e = launch_linear(*a, plan, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_linear_e4m3");
}

moe_status moe_rope_frequencies(int32_t rotary_dim, double base, const moe_rope_scaling* scaling, double* turns, float* factor)
{
    const int kind = scaling ? scaling->kind : MOE_ROPE_NONE;
    if (!turns || !factor || kind < MOE_ROPE_NONE || kind > MOE_ROPE_YARN) return MOE_ERR_INVALID_ARG;
    if (rotary_dim < 2 || rotary_dim % 2 != 0) return MOE_ERR_SHAPE;
    if (!(base > 1.0) || !std::isfinite(base)) return MOE_ERR_INVALID_ARG;
    const double f = kind == MOE_ROPE_NONE ? 1.0 : scaling->factor, R = rotary_dim, two_pi = 6.283185307179586476925;
    if (!(f >= 1.0) || !std::isfinite(f)) return MOE_ERR_INVALID_ARG;
    if (kind == MOE_ROPE_NTK && rotary_dim > 2) base *= std::pow(f, R / (R - 2.0));
    double low = 0.0, high = 0.0;
    if (kind == MOE_ROPE_YARN) {
        const double n = scaling->original_length;
        if (!(n > 0.0) || !std::isfinite(n) || !(scaling->beta_slow > 0.0) || !(scaling->beta_fast > scaling->beta_slow) ||
            !std::isfinite(scaling->beta_fast))
            return MOE_ERR_INVALID_ARG;
        // pair (not whole) whose wavelength fits that often into the original length: n base^(-2i/R) / 2pi = turns
        auto pair_of = [&](double made) { return R * std::log(n / (made * two_pi)) / (2.0 * std::log(base)); };
        low = std::fmax(std::floor(pair_of(scaling->beta_fast)), 0.0);
        high = std::fmin(std::ceil(pair_of(scaling->beta_slow)), R - 1.0);
        high = std::fmax(high - low, 1e-3);                // width of the ramp
    }
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double v = std::pow(base, -2.0 * i / R) / two_pi;
        if (kind == MOE_ROPE_LINEAR) v /= f;
        if (kind == MOE_ROPE_YARN) {
            const double ramp = std::fmin(std::fmax((i - low) / high, 0.0), 1.0);
            v = v * (1.0 - ramp) + v / f * ramp;
        }
        turns[i] = v;
    }
    *factor = kind == MOE_ROPE_YARN ? (float)(0.1 * std::log(f) + 1.0) : 1.0f;
    return MOE_OK;
}

moe_status moe_rope_append(const moe_kv_cache* cache, const moe_block_table* table, const moe_rope* rope, const void* q,
                           int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                           int32_t n_heads, int32_t T, const int32_t* positions, void* q_out, int64_t q_out_stride,
                           void* stream)
{
    moe_status st = check_cache(cache);
    if (st != MOE_OK) return st;
    if (T < 0 || !rope) return MOE_ERR_INVALID_ARG;
    const int D = cache->head_dim, R = rope->rotary_dim;
    if (D % 16 != 0 || R < 0 || R > D || R % 16 != 0 || n_heads < 1) return MOE_ERR_SHAPE;
    if (D > 256 || n_heads > MOE_MAX_HEADS || T > MOE_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
    if (R > 0 && !rope->turns) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;                            // an empty batch's table has no rows
    if ((st = check_table(table, T)) != MOE_OK) return st;
    if (!q || !k || !v || !positions || !q_out) return MOE_ERR_INVALID_ARG;
    if (off(q, 16) || off(k, 16) || off(v, 16) || off(q_out, 16) || off(positions, 4) || off(rope->turns, 8) || bad_stride(q_stride, 8) ||
        bad_stride(k_stride, 8) || bad_stride(v_stride, 8) || bad_stride(q_out_stride, 8))
        return MOE_ERR_ALIGNMENT;
    if (T > 1 && q_out_stride < (int64_t)n_heads * D) return MOE_ERR_SHAPE;
    hipError_t e = launch_rope(*cache, *table, *rope, static_cast<const bf16_t*>(q), q_stride, static_cast<const bf16_t*>(k), k_stride,
                               static_cast<const bf16_t*>(v), v_stride, n_heads, T, positions, static_cast<bf16_t*>(q_out), q_out_stride,
                               static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_rope_append");
}

moe_status moe_attention_workspace_size(const moe_kv_cache* cache, int32_t T_max, int32_t n_heads, size_t* bytes)
{
    moe_status st = check_attention(cache, n_heads, T_max);
    if (st != MOE_OK) return st;
    if (!bytes) return MOE_ERR_INVALID_ARG;
    *bytes = attention_workspace_bytes(*cache, T_max, n_heads);
    if (ensure_device_init(nullptr) != hipSuccess) (void)hipGetLastError();      // as in moe_linear_workspace_size
    return MOE_OK;
}

moe_status moe_paged_attention(const moe_kv_cache* cache, const moe_block_table* table, const void* q, int64_t q_stride,
                               int32_t n_heads, int32_t T, const int32_t* lengths, float scale, int32_t window, void* out,
                               int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    moe_status st = check_attention(cache, n_heads, T);
    if (st != MOE_OK) return st;
    if (window < 0 || !std::isfinite(scale)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if ((st = check_table(table, T)) != MOE_OK) return st;
    if (!q || !lengths || !out) return MOE_ERR_INVALID_ARG;
    if (off(q, 16) || off(lengths, 4) || off(out, 8) || off(lse, 4) || bad_stride(q_stride, 8) || bad_stride(out_stride, 4))
        return MOE_ERR_ALIGNMENT;
    if (T > 1 && out_stride < (int64_t)n_heads * cache->head_dim) return MOE_ERR_SHAPE;
    if (!workspace || workspace_bytes < attention_workspace_bytes(*cache, T, n_heads)) return MOE_ERR_WORKSPACE;
    if (off(workspace, 256)) return MOE_ERR_ALIGNMENT;
    // blocks read a token's q where others have written its out
    if (rows_meet(q, 2 * q_stride, out, 2 * out_stride, T, (int64_t)2 * n_heads * cache->head_dim)) return MOE_ERR_INVALID_ARG;
    hipError_t e = ensure_device_init(nullptr);
    if (e != hipSuccess) return hip_fail(e, "moe_paged_attention/init");
    e = launch_attention(*cache, *table, static_cast<const bf16_t*>(q), q_stride, n_heads, T, lengths, scale, window,
                         static_cast<bf16_t*>(out), out_stride, lse, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : hip_fail(e, "moe_paged_attention");
}

}  // extern "C"
