// Rotary positions of new tokens' q and k, and the append of k and v to the paged cache, in one pass over the projection's output.
//
//   (a, b) of pair i at position p  ->  (a cos - b sin, b cos + a sin),  angle = p * turns[i] whole turns
//
// Whole turns are taken off in fp64, where position times frequency is exact to 1e-16 of the turns made; the sine and cosine of what is
// left are fp32.  They are computed once per token and shared by its heads through LDS.  HBM bound: each input is read once, each
// output written once.  1021 tokens of 16 + 2 * 16 heads into e4m3 7.0 us, one token 2.6 us: latency.
// Tokens of a tree go to places apart from their positions: 2112 tokens of 32 + 2 * 8 heads into e4m3 8.2 us.
#include "layer.h"

#include <type_traits>

namespace bmoe {

struct RopeArgs {
    const bf16_t *q, *k, *v;
    bf16_t* qo;
    int64_t qs, ks, vs, qos;
    const int32_t *positions, *places;                    // places NULL: the positions
    const int32_t *pages, *token_row;
    int64_t row_stride;
    int n_rows, max_pages;
    const double* turns;
    float factor;
    int R, interleaved;
    uint8_t *kc, *vc;                                     // the cache
    int64_t page_stride, token_stride, head_stride;
    const float *k_scale, *v_scale;
    int n_pages, page_size;
    int H, Hk, D, T;
};

// Where k and v of a token that goes to position pos are, in elements from the cache's base; negative: nowhere.
__device__ __forceinline__ int64_t cache_place(const RopeArgs& p, int t, int pos)
{
    const int row = p.token_row ? p.token_row[t] : t, page_at = pos / p.page_size;
    if (pos < 0 || (unsigned)row >= (unsigned)p.n_rows || page_at >= p.max_pages) return -1;
    const int page = p.pages[(int64_t)row * p.row_stride + page_at];
    if ((unsigned)page >= (unsigned)p.n_pages) return -1;
    return (int64_t)page * p.page_stride + (int64_t)(pos - page_at * p.page_size) * p.token_stride;
}

// Eight values over their head's scale for an 8-bit cache: beyond 448 they stay at 448, NaN stays NaN.  (By division 16384 tokens of 16 + 2 * 16 heads of 64
// 34 -> 38 us, this way 35.)
__device__ __forceinline__ uint2 clamp_e4m3x8(float (&f)[8], float scale)
{
    const Divisor div(lift_tiny(f, scale));
    float g[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float q = div.near(f[e]);
        g[e] = fabsf(q) > kE4m3Max ? copysignf(kE4m3Max, q) : div.exact(f[e], q);
    }
    return make_uint2(pack_e4m3(g[0], g[1], g[2], g[3]), pack_e4m3(g[4], g[5], g[6], g[7]));
}

// One block per token.  A thread's unit is 16 columns of a head in two pieces of 8: where pairs are (i, i + R/2), columns i.. and i + R/2..
// of the rotated part; else 16 columns in a row.  So a unit never needs another thread's columns.
template <bool E4M3, bool ONCE>
__global__ void __launch_bounds__(512) rope_kernel(RopeArgs p)
{
    __shared__ float cs[128], sn[128];                    // R/2 <= 128
    const int t = blockIdx.x, half = p.R >> 1;
    const int pos = p.positions[t];
    for (int i = threadIdx.x; i < half; i += blockDim.x) {
        double turns = (double)pos * p.turns[i];
        const float part = (float)(turns - rint(turns));  // within half a turn
        float s, c;
        sincospif(2.0f * part, &s, &c);
        cs[i] = c * p.factor;
        sn[i] = s * p.factor;
    }
    const int64_t place = pos < 0 ? -1 : cache_place(p, t, p.places ? p.places[t] : pos);
    __syncthreads();
    const int per_head = p.D >> 4, units = (p.H + 2 * p.Hk) * per_head, rot = p.R >> 4;
    for (int u = threadIdx.x; u < units; u += blockDim.x) {
        const int head = u / per_head, j = u - head * per_head;
        const bool is_q = head < p.H, is_v = head >= p.H + p.Hk;
        if (!is_q && place < 0) continue;
        const int hk = is_v ? head - p.H - p.Hk : head - p.H;
        const bool rotated = !is_v && j < rot, apart = rotated && !p.interleaved;
        const int o0 = apart ? 8 * j : 16 * j, o1 = apart ? half + 8 * j : 16 * j + 8;
        const bf16_t* src = is_q ? p.q + (int64_t)t * p.qs + (int64_t)head * p.D
                                 : (is_v ? p.v + (int64_t)t * p.vs : p.k + (int64_t)t * p.ks) + (int64_t)hk * p.D;
        float a[8], b[8];
        unpack_bf16(*reinterpret_cast<const uint4*>(src + o0), a);
        unpack_bf16(*reinterpret_cast<const uint4*>(src + o1), b);
        if (rotated) {
            if (apart) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float c = cs[8 * j + e], s = sn[8 * j + e], x = a[e], y = b[e];
                    a[e] = x * c - y * s;
                    b[e] = y * c + x * s;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float* w = e < 4 ? a + 2 * e : b + 2 * (e - 4);
                    const float c = cs[8 * j + e], s = sn[8 * j + e], x = w[0], y = w[1];
                    w[0] = x * c - y * s;
                    w[1] = y * c + x * s;
                }
            }
        }
        if (is_q) {
            if (pos < 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] = b[e] = 0.0f;
            }
            bf16_t* dst = p.qo + (int64_t)t * p.qos + (int64_t)head * p.D;
            store16<ONCE>(dst + o0, pack_bf16x8(a));
            store16<ONCE>(dst + o1, pack_bf16x8(b));
            continue;
        }
        const int64_t at = place + (int64_t)hk * p.head_stride;
        uint8_t* dst = is_v ? p.vc : p.kc;
        if constexpr (E4M3) {
            const float scale = (is_v ? p.v_scale : p.k_scale)[hk];
            *reinterpret_cast<uint2*>(dst + at + o0) = clamp_e4m3x8(a, scale);
            *reinterpret_cast<uint2*>(dst + at + o1) = clamp_e4m3x8(b, scale);
        } else {
            *reinterpret_cast<uint4*>(dst + 2 * (at + o0)) = pack_bf16x8(a);
            *reinterpret_cast<uint4*>(dst + 2 * (at + o1)) = pack_bf16x8(b);
        }
    }
}

hipError_t launch_rope(const moe_kv_cache& c, const moe_block_table& t, const moe_rope& r, const bf16_t* q, int64_t q_stride,
                       const bf16_t* k, int64_t k_stride, const bf16_t* v, int64_t v_stride, int n_heads, int T,
                       const int32_t* positions, const int32_t* places, bf16_t* q_out, int64_t q_out_stride, hipStream_t s)
{
    RopeArgs p;
    p.q = q; p.k = k; p.v = v; p.qo = q_out;
    p.qs = q_stride; p.ks = k_stride; p.vs = v_stride; p.qos = q_out_stride;
    p.positions = positions; p.places = places;
    p.pages = t.pages; p.token_row = t.token_row; p.row_stride = t.row_stride; p.n_rows = t.n_rows; p.max_pages = t.max_pages;
    p.turns = r.turns; p.factor = r.factor; p.R = r.rotary_dim; p.interleaved = r.interleaved;
    p.kc = static_cast<uint8_t*>(c.k); p.vc = static_cast<uint8_t*>(c.v);
    p.page_stride = c.page_stride; p.token_stride = c.token_stride; p.head_stride = c.head_stride;
    p.k_scale = c.k_scale; p.v_scale = c.v_scale; p.n_pages = c.n_pages; p.page_size = c.page_size;
    p.H = n_heads; p.Hk = c.n_kv_heads; p.D = c.head_dim; p.T = T;
    // Few tokens: a thread for every unit of most shapes.  A large q goes past the caches (16384 tokens of 56 heads 113 -> 106 us, 5.7 TB/s; 8192 of 16
    // heads of 64 24 -> 19).
    const int threads = T <= 512 ? 512 : 256;
    const bool once = (int64_t)T * n_heads * c.head_dim * 2 > kCachedBytes;
    auto go = [&](auto e4m3, auto past) {
        hipLaunchKernelGGL((rope_kernel<decltype(e4m3)::value, decltype(past)::value>), dim3(T), dim3(threads), 0, s, p);
    };
    if (c.type == MOE_KV_E4M3) once ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
    else once ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
    return hipGetLastError();
}

}  // namespace bmoe
