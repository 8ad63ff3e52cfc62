// Attention of new tokens over a paged key-value cache.
//
//   out = sum_p softmax_p(scale q . k_p) v_p, in one pass: running maximum m, running sum l and the running weighted sum O of v, rescaled by
//   exp(m_old - m_new) when the maximum moves; parts of a sequence are joined by the same rule.
//
// The cache is read once, so HBM bounds it.  The products run on the matrix cores all the same, with the query heads that share a key head
// (up to 16) as the 16 columns: a wave multiplies 32 positions at a time,
//   S [32 positions][16 heads] = K Q^T,     O^T [D][16 heads] += V^T P^T,
// and operands come straight from memory into the lanes that the MFMA wants them in, with no LDS between:
//   K: lane (g, c) = (lane / 16, lane % 16) holds 8 columns of position c.
//   S leaves lane (g, c) with the scores of head c at positions 4 g .. 4 g + 3 of each 16; that is already the layout of P^T as the second
//   operand, with the 8 positions of a lane in the order {4 g + e, 16 + 4 g + e}.
//   V^T: lane (g, c) reads the same 8 positions' columns 8 c .. 8 c + 7 (whole rows of 16 lanes x 16 bytes) and transposes its 8 x 8 block with
//   byte permutes; product j then gives the rows d = 8 c + j.
// The maximum and the rescaling are per head = per lane; only the maximum crosses lanes (two exchanges per 32 positions).
//
// Work: the positions of every (token, key head, 16 query heads) in tiles of 128 form one line of tiles, cut into equal shares, one per block:
// one long sequence among short ones is spread over the whole GPU.  A share that begins or ends inside a sequence leaves (m, l, O) in the
// workspace, and join_kernel adds these up.
#include "layer.h"

#include <algorithm>

namespace bmoe {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kAttnWaves = 4, kAttnThreads = 64 * kAttnWaves;
constexpr int kStep = 32;                         // positions of a wave's step
constexpr int kTile = kStep * kAttnWaves;         // positions of a block's step
constexpr int kAttnBlocks = 512;                  // shares at most

struct AttnArgs {
    const uint8_t *kc, *vc;
    int64_t page_stride, token_stride, head_stride;
    const float *k_scale, *v_scale;
    const int32_t *pages, *token_row;
    int64_t row_stride;
    int n_rows, n_pages, page_size;
    unsigned page_magic;                          // position / page_size = position * page_magic >> page_shift
    int page_shift;
    int cap;                                      // positions that a row of the block table has
    const bf16_t* q;
    int64_t q_stride;
    const int32_t* lengths;
    int T, H, Hk, group, q_tiles, heads;          // heads: query heads of a work item (at most 16)
    float scale;
    int window;
    bf16_t* out;
    int64_t out_stride;
    float* lse;
    int4* cuts;                                   // per share: the item that it begins and does not end (token, item, shares, -)
    float* parts;                                 // per share two parts: [heads][D] O, [heads] m, [heads] l
};

// Positions [lo, hi) that token t attends to.
__device__ __forceinline__ int2 span_of(const AttnArgs& p, int t)
{
    const int hi = min(max(p.lengths[t], 0), p.cap);
    const int row = p.token_row ? p.token_row[t] : t;
    const bool there = (unsigned)row < (unsigned)p.n_rows;
    return make_int2(p.window > 0 ? max(hi - p.window, 0) : 0, there ? hi : 0);
}
__device__ __forceinline__ int tiles_of(const int2 s) { return s.y > s.x ? (int)(((unsigned)(s.y - s.x) + kTile - 1) / kTile) : 0; }

// The block's share of the line of tiles: its bounds, and where it begins.
struct Share {
    int64_t per, first, end;                      // tiles per share; this one's
    int token;                                    // token of tile `first`
    int64_t before;                               // tiles of the tokens before that one
};

__device__ __forceinline__ int64_t wave_sum_before(int64_t v, int lane, int64_t& total)
{
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    total = __shfl(x, 63);
    return x - v;
}

__device__ __forceinline__ Share find_share(const AttnArgs& p, int64_t* lds)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (p.T + kAttnThreads - 1) / kAttnThreads, t0 = min(p.T, tid * each), t1 = min(p.T, t0 + each);
    const int items = p.Hk * p.q_tiles;
    int64_t mine = 0;
    for (int t = t0; t < t1; ++t) mine += (int64_t)tiles_of(span_of(p, t)) * items;
    int64_t total;
    int64_t before = wave_sum_before(mine, lane, total);
    if (lane == 0) lds[wave] = total;
    __syncthreads();
    Share s;
    int64_t all = 0;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    s.per = (all + gridDim.x - 1) / gridDim.x;
    s.first = min(all, s.per * (int64_t)blockIdx.x);
    s.end = min(all, s.first + s.per);
    // the one thread whose tokens hold tile `first` looks for it
    if (s.first < s.end && before <= s.first && s.first < before + mine) {
        int t = t0;
        for (;; ++t) {
            const int64_t n = (int64_t)tiles_of(span_of(p, t)) * items;
            if (s.first < before + n) break;
            before += n;
        }
        lds[kAttnWaves] = t;
        lds[kAttnWaves + 1] = before;
    }
    __syncthreads();
    s.token = (int)lds[kAttnWaves];
    s.before = lds[kAttnWaves + 1];
    return s;
}

// Two e4m3 -> two bf16 (exact), from the low or the high half of a word.
template <bool HIGH>
__device__ __forceinline__ unsigned widen(unsigned w)
{
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}

// The 32 positions' K rows as a wave's lanes hold them: two 16-position operands of D / 32 products.  Which 8 columns a lane brings to a
// product is free as long as q does the same: bf16: 8 (4 s + g); e4m3: 16-byte pieces for two products at a time.
template <int D, bool E4M3>
struct KRows {
    static constexpr int S = D / 32, P16 = E4M3 ? D / 64 : S, P8 = E4M3 ? S & 1 : 0;
    uint4 w[2][P16 ? P16 : 1];
    uint2 tail[2][P8 ? P8 : 1];

    __device__ __forceinline__ void load(const uint8_t* base, const int64_t* off, int g)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* row = base + off[h] * (E4M3 ? 1 : 2);
#pragma unroll
            for (int i = 0; i < P16; ++i) w[h][i] = *reinterpret_cast<const uint4*>(row + 64 * i + 16 * g);
            if constexpr (P8) tail[h][0] = *reinterpret_cast<const uint2*>(row + 64 * P16 + 8 * g);
        }
    }
    static __device__ __forceinline__ int column(int s, int g)
    {
        if (!E4M3) return 32 * s + 8 * g;
        return s < 2 * P16 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 64 * P16 + 8 * g;
    }
    __device__ __forceinline__ bf16x8 operand(int h, int s) const
    {
        if constexpr (!E4M3) return __builtin_bit_cast(bf16x8, w[h][s]);
        else {
            uint2 v;
            if (s < 2 * P16) v = s & 1 ? make_uint2(w[h][s >> 1].z, w[h][s >> 1].w) : make_uint2(w[h][s >> 1].x, w[h][s >> 1].y);
            else v = tail[h][0];
            return __builtin_bit_cast(bf16x8, make_uint4(widen<false>(v.x), widen<true>(v.x), widen<false>(v.y), widen<true>(v.y)));
        }
    }
};

// The 8 positions' columns [C0 + c N, + N) of V that a lane holds, N = W / 16 (8, 4 or 2).
template <int W, bool E4M3>
struct VPart {
    static constexpr int N = W / 16, BYTES = N * (E4M3 ? 1 : 2);
    struct __attribute__((aligned(BYTES))) Raw { uint8_t b[BYTES]; };
    Raw v[8];

    __device__ __forceinline__ void load(const uint8_t* base, int c0, const int64_t* off, int c)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const Raw*>(base + (off[e] + c0 + c * N) * (E4M3 ? 1 : 2));
    }
    // word i of position e: columns 2 i and 2 i + 1 in bf16
    __device__ __forceinline__ unsigned word(int e, int i) const
    {
        if constexpr (!E4M3) {
            unsigned u[N / 2];
            __builtin_memcpy(u, v[e].b, sizeof u);
            return u[i];
        } else {
            if constexpr (N == 2) {
                unsigned short u;
                __builtin_memcpy(&u, v[e].b, 2);
                return widen<false>(u);
            } else {
                unsigned u[N / 4];
                __builtin_memcpy(u, v[e].b, sizeof u);
                return i & 1 ? widen<true>(u[i >> 1]) : widen<false>(u[i >> 1]);
            }
        }
    }
    // acc[j] += (column c N + j of the 8 positions) x p.  keep: bits of the positions that count; what the others hold may be anything.
    __device__ __forceinline__ void add(f32x4* acc, bf16x8 prob, bool all, unsigned keep) const
    {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            unsigned w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = word(e, i);
                if (!all) w[e] = keep >> e & 1 ? w[e] : 0;
            }
            uint4 lo, hi;
            lo.x = __builtin_amdgcn_perm(w[1], w[0], 0x05040100u); hi.x = __builtin_amdgcn_perm(w[1], w[0], 0x07060302u);
            lo.y = __builtin_amdgcn_perm(w[3], w[2], 0x05040100u); hi.y = __builtin_amdgcn_perm(w[3], w[2], 0x07060302u);
            lo.z = __builtin_amdgcn_perm(w[5], w[4], 0x05040100u); hi.z = __builtin_amdgcn_perm(w[5], w[4], 0x07060302u);
            lo.w = __builtin_amdgcn_perm(w[7], w[6], 0x05040100u); hi.w = __builtin_amdgcn_perm(w[7], w[6], 0x07060302u);
            acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), prob, acc[2 * i], 0, 0, 0);
            acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), prob, acc[2 * i + 1], 0, 0, 0);
        }
    }
};

// head_dim in pieces of 128, 64 and 32 columns
template <int D, bool E4M3>
struct VRows {
    static constexpr int N128 = D / 128, N64 = D % 128 / 64, N32 = D % 64 / 32;
    VPart<128, E4M3> a[N128 ? N128 : 1];
    VPart<64, E4M3> b;
    VPart<32, E4M3> c;
    __device__ __forceinline__ void load(const uint8_t* base, const int64_t* off, int col)
    {
#pragma unroll
        for (int i = 0; i < N128; ++i) a[i].load(base, 128 * i, off, col);
        if constexpr (N64) b.load(base, 128 * N128, off, col);
        if constexpr (N32) c.load(base, 128 * N128 + 64 * N64, off, col);
    }
    __device__ __forceinline__ void add(f32x4* acc, bf16x8 prob, bool all, unsigned keep) const
    {
#pragma unroll
        for (int i = 0; i < N128; ++i) a[i].add(acc + 8 * i, prob, all, keep);
        if constexpr (N64) b.add(acc + 8 * N128, prob, all, keep);
        if constexpr (N32) c.add(acc + 8 * N128 + 4 * N64, prob, all, keep);
    }
    // column of head_dim behind register r of acc[j]: a lane's are N in a row for each r
    static __device__ __forceinline__ int column(int j, int r, int g)
    {
        if (j < 8 * N128) return 128 * (j >> 3) + 8 * (4 * g + r) + (j & 7);
        j -= 8 * N128;
        if (j < 4 * N64) return 128 * N128 + 4 * (4 * g + r) + j;
        return 128 * N128 + 64 * N64 + 2 * (4 * g + r) + j - 4 * N64;
    }
};

template <int D, bool E4M3>
__global__ void __launch_bounds__(kAttnThreads, 2) attention_kernel(AttnArgs p)
{
    using K = KRows<D, E4M3>;
    using V = VRows<D, E4M3>;
    constexpr int NJ = D / 16;                            // products of V's columns
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ int64_t found[kAttnWaves + 2];
    __shared__ int64_t places[kAttnWaves][kStep];         // offset of a step's positions in the cache
    __shared__ float stat[kAttnWaves][2][16];
    float* joined = reinterpret_cast<float*>(smem);       // [waves][heads][D + 4]

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, c = lane & 15;

    // tokens with nothing to attend to
    for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
        if (tiles_of(span_of(p, t)) > 0) continue;
        for (int i = tid * 4; i < p.H * D; i += kAttnThreads * 4)
            *reinterpret_cast<uint2*>(p.out + (int64_t)t * p.out_stride + i) = make_uint2(0, 0);
        if (p.lse)
            for (int i = tid; i < p.H; i += kAttnThreads) p.lse[(int64_t)t * p.H + i] = -__builtin_inff();
    }

    const Share share = find_share(p, found);
    if (tid == 0) p.cuts[blockIdx.x] = make_int4(0, 0, 0, 0);
    if (share.first >= share.end) return;

    int t = share.token;
    int64_t before = share.before;
    int64_t at = share.first;
    while (at < share.end) {
        int2 span = span_of(p, t);
        int n = tiles_of(span);
        while (at >= before + (int64_t)n * p.Hk * p.q_tiles) {          // on to the next token that has tiles
            before += (int64_t)n * p.Hk * p.q_tiles;
            ++t;
            span = span_of(p, t);
            n = tiles_of(span);
        }
        const int item = (int)((at - before) / n);
        const int64_t item_first = before + (int64_t)item * n;
        const int i0 = (int)(at - item_first), i1 = (int)min((int64_t)n, share.end - item_first);
        at = item_first + i1;
        const int hk = item / p.q_tiles, h0 = hk * p.group + (item - hk * p.q_tiles) * 16;
        const int nh = min(16, (hk + 1) * p.group - h0);

        // q of my head, in the order of K's columns
        bf16x8 q[K::S];
#pragma unroll
        for (int s = 0; s < K::S; ++s) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if (c < nh) w = *reinterpret_cast<const uint4*>(p.q + (int64_t)t * p.q_stride + (int64_t)(h0 + c) * D + K::column(s, g));
            q[s] = __builtin_bit_cast(bf16x8, w);
        }
        const float to_log2 = p.scale * (E4M3 ? p.k_scale[hk] : 1.0f) * 1.4426950408889634f;
        const int32_t* row = p.pages + (int64_t)(p.token_row ? p.token_row[t] : t) * p.row_stride;
        const uint8_t* kbase = p.kc + (int64_t)hk * p.head_stride * (E4M3 ? 1 : 2);
        const uint8_t* vbase = p.vc + (int64_t)hk * p.head_stride * (E4M3 ? 1 : 2);

        // page of lane's position of step i (lanes 0..31), -1 beyond the end
        const unsigned first_pos = (unsigned)span.x + wave * kStep + (lane & 31);
        auto page_of = [&](int i, unsigned& at_in_page) -> int {
            const unsigned pos = first_pos + (unsigned)i * kTile;
            at_in_page = 0;
            if (pos >= (unsigned)span.y) return -1;
            const unsigned pg = (unsigned)((uint64_t)pos * p.page_magic >> p.page_shift);
            at_in_page = pos - pg * (unsigned)p.page_size;
            return row[pg];
        };
        unsigned mask = 0, next_mask = 0;
        int64_t koff[2], voff[8];
        // the places of a step's positions, by way of LDS to the lanes that load them
        auto place = [&](int page, unsigned at_in_page) -> unsigned {
            const bool there = (unsigned)page < (unsigned)p.n_pages;
            const int64_t off = there ? (int64_t)page * p.page_stride + (int64_t)at_in_page * p.token_stride : 0;
            if (lane < kStep) places[wave][lane] = off;
            wave_lds_order();
#pragma unroll
            for (int h = 0; h < 2; ++h) koff[h] = places[wave][16 * h + c];
#pragma unroll
            for (int e = 0; e < 8; ++e) voff[e] = places[wave][16 * (e >> 2) + 4 * g + (e & 3)];
            wave_lds_order();
            return (unsigned)__ballot(there);             // lanes 0..31
        };

        f32x4 acc[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -__builtin_inff(), l = 0.0f;
        K kr;
        V vr;
        // steps of this wave: all but perhaps the last tile, whose end may lie before its positions
        int last = i1;
        if ((int64_t)span.x + (int64_t)(i1 - 1) * kTile + wave * kStep >= span.y) --last;
        unsigned in_page = 0;
        int page = -1;
        if (i0 < last) {
            page = page_of(i0, in_page);
            mask = place(page, in_page);
            page = page_of(i0 + 1, in_page);
            kr.load(kbase, koff, g);
            vr.load(vbase, voff, c);
        }
        for (int i = i0; i < last; ++i) {
            f32x4 s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < K::S; ++k) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr.operand(h, k), q[k], s[h], 0, 0, 0);
            }
            const bool more = i + 1 < last;
            if (more) {
                next_mask = place(page, in_page);
                page = page_of(i + 2, in_page);
                kr.load(kbase, koff, g);
            }
            // scores in powers of two
            float top = -__builtin_inff();
            const bool all = mask == 0xFFFFFFFFu;
            const unsigned keep = (mask >> (4 * g) & 0xFu) | (mask >> (16 + 4 * g) & 0xFu) << 4;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[h][r] *= to_log2;
                    if (!all && !(keep >> (4 * h + r) & 1)) s[h][r] = -__builtin_inff();
                    top = fmaxf(top, s[h][r]);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m, top);
            const float ref = m_new == -__builtin_inff() ? 0.0f : m_new;     // nothing seen yet
            if (__any(m_new != m)) {
                const float f = __builtin_amdgcn_exp2f(m - ref);
                l *= f;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[j][r] *= f;
                m = m_new;
            }
            float e[8];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    e[4 * h + r] = __builtin_amdgcn_exp2f(s[h][r] - ref);
                    l += e[4 * h + r];
                }
            vr.add(acc, __builtin_bit_cast(bf16x8, pack_bf16x8(e)), all, keep);
            if (more) {
                vr.load(vbase, voff, c);
                mask = next_mask;
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);

        // join the waves
        if (g == 0) {
            stat[wave][0][c] = m;
            stat[wave][1][c] = l;
        }
        __syncthreads();
        float top = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) top = fmaxf(top, stat[w][0][c]);
        const float ref = top == -__builtin_inff() ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - ref);
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) sum += stat[w][1][c] * __builtin_amdgcn_exp2f(stat[w][0][c] - ref);
        if (c < nh) {
            float* dst = joined + (wave * p.heads + c) * (D + 4);
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) dst[V::column(j, r, g)] = acc[j][r] * f;
        }
        __syncthreads();                                  // also: everyone has read stat
        if (wave == 0 && g == 0) {
            stat[0][0][c] = top;
            stat[0][1][c] = sum;
        }
        __syncthreads();
        const bool begins = i0 == 0, ends = i1 == n;
        float* part = p.parts + ((int64_t)2 * blockIdx.x + (begins ? 1 : 0)) * ((int64_t)p.heads * (D + 2));
        const float vs = E4M3 ? p.v_scale[hk] : 1.0f;
        for (int i = tid * 4; i < nh * D; i += kAttnThreads * 4) {
            const int h = i / D;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kAttnWaves; ++w) {
                const float4 v = *reinterpret_cast<const float4*>(joined + (w * p.heads + h) * (D + 4) + (i - h * D));
                o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
            }
            if (begins && ends) {
                const float total = stat[0][1][h], k = total > 0.0f || total != total ? vs / total : 0.0f;
                *reinterpret_cast<uint2*>(p.out + (int64_t)t * p.out_stride + (int64_t)h0 * D + i) =
                    make_uint2(pack_bf16(o.x * k, o.y * k), pack_bf16(o.z * k, o.w * k));
            } else {
                *reinterpret_cast<float4*>(part + i) = o;
            }
        }
        if (tid < nh) {
            const float top_h = stat[0][0][tid], sum_h = stat[0][1][tid];
            if (begins && ends) {
                if (p.lse) p.lse[(int64_t)t * p.H + h0 + tid] = (top_h + __log2f(sum_h)) * 0.6931471805599453f;
            } else {
                part[p.heads * D + tid] = top_h;
                part[p.heads * D + p.heads + tid] = sum_h;
            }
        }
        if (begins && !ends && tid == 0) {
            const int64_t last_share = (item_first + n - 1) / share.per;
            p.cuts[blockIdx.x] = make_int4(t, item, (int)(last_share - blockIdx.x) + 1, 0);
        }
        __syncthreads();                                  // LDS is free for the next item
    }
}

// Joins the parts of the item that share x begins and does not end: one block per (share, head of the item).
template <int D>
__global__ void __launch_bounds__(256) join_kernel(AttnArgs p, int e4m3)
{
    const int4 cut = p.cuts[blockIdx.x];
    const int n = cut.z, hk = cut.y / p.q_tiles, h0 = hk * p.group + (cut.y - hk * p.q_tiles) * 16, h = blockIdx.y;
    if (n == 0 || h >= min(16, (hk + 1) * p.group - h0)) return;
    const int64_t size = (int64_t)p.heads * (D + 2);
    // share x left its part in its second place, the others in their first
    auto part = [&](int i) { return p.parts + (2 * ((int64_t)blockIdx.x + i) + (i == 0 ? 1 : 0)) * size; };
    const int tid = threadIdx.x;
    __shared__ float red[2][4];
    float top = -__builtin_inff();
    for (int i = tid; i < n; i += 256) top = fmaxf(top, part(i)[p.heads * D + h]);
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if ((tid & 63) == 0) red[0][tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    const float ref = top == -__builtin_inff() ? 0.0f : top;
    constexpr int LANES = D / 4, ROWS = 256 / LANES;      // threads of a row of O; rows side by side
    const int r = tid / LANES, col = (tid - r * LANES) * 4;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.0f;
    if (r < ROWS) {
#pragma unroll 4
        for (int i = r; i < n; i += ROWS) {
            const float* q = part(i);
            const float f = __builtin_amdgcn_exp2f(q[p.heads * D + h] - ref);
            const float4 v = *reinterpret_cast<const float4*>(q + h * D + col);
            o.x += f * v.x; o.y += f * v.y; o.z += f * v.z; o.w += f * v.w;
            sum += f * q[p.heads * D + p.heads + h];
        }
    }
    __shared__ float4 rows[ROWS][LANES];
    __shared__ float sums[ROWS];
    if (r < ROWS) {
        rows[r][col / 4] = o;
        if (col == 0) sums[r] = sum;
    }
    __syncthreads();
    if (r != 0) return;
#pragma unroll
    for (int i = 1; i < ROWS; ++i) {
        const float4 v = rows[i][col / 4];
        o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
        sum += sums[i];
    }
    const float k = sum > 0.0f || sum != sum ? (e4m3 ? p.v_scale[hk] : 1.0f) / sum : 0.0f;
    *reinterpret_cast<uint2*>(p.out + (int64_t)cut.x * p.out_stride + (int64_t)(h0 + h) * D + col) =
        make_uint2(pack_bf16(o.x * k, o.y * k), pack_bf16(o.z * k, o.w * k));
    if (p.lse && col == 0) p.lse[(int64_t)cut.x * p.H + h0 + h] = (top + __log2f(sum)) * 0.6931471805599453f;
}

static int item_heads(int group) { return group < 16 ? group : 16; }

size_t attention_workspace_bytes(const moe_kv_cache& c, int T, int n_heads)
{
    (void)T;                                              // the shares are as many for every T
    const int heads = item_heads(n_heads / c.n_kv_heads);
    return align_up(kAttnBlocks * sizeof(int4), 256) + align_up((size_t)2 * kAttnBlocks * heads * (c.head_dim + 2) * sizeof(float), 256);
}

// A row of O in LDS is 4 floats longer, so that the heads of a wave write to different banks.
template <int D>
static size_t attention_lds(int heads) { return (size_t)kAttnWaves * heads * (D + 4) * sizeof(float); }

template <int D>
static hipError_t attention_init()
{
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_kernel<D, true>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)attention_lds<D>(16));
    if (e != hipSuccess) return e;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_kernel<D, false>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)attention_lds<D>(16));
}

hipError_t init_attention_kernels()
{
    hipError_t e;
    if ((e = attention_init<64>()) != hipSuccess || (e = attention_init<96>()) != hipSuccess || (e = attention_init<128>()) != hipSuccess ||
        (e = attention_init<192>()) != hipSuccess)
        return e;
    return attention_init<256>();
}

template <int D>
static hipError_t attention_go(const AttnArgs& p, bool e4m3, int grid, hipStream_t s)
{
    const size_t lds = attention_lds<D>(p.heads);
    if (e4m3) hipLaunchKernelGGL((attention_kernel<D, true>), dim3(grid), dim3(kAttnThreads), lds, s, p);
    else hipLaunchKernelGGL((attention_kernel<D, false>), dim3(grid), dim3(kAttnThreads), lds, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || grid == 1) return e;           // one share: nothing is cut
    hipLaunchKernelGGL((join_kernel<D>), dim3(grid, p.heads), dim3(256), 0, s, p, e4m3 ? 1 : 0);
    return hipGetLastError();
}

hipError_t launch_attention(const moe_kv_cache& c, const moe_block_table& t, const bf16_t* q, int64_t q_stride, int n_heads, int T,
                            const int32_t* lengths, float scale, int window, bf16_t* out, int64_t out_stride, float* lse, void* ws,
                            hipStream_t s)
{
    AttnArgs p;
    p.kc = static_cast<const uint8_t*>(c.k); p.vc = static_cast<const uint8_t*>(c.v);
    p.page_stride = c.page_stride; p.token_stride = c.token_stride; p.head_stride = c.head_stride;
    p.k_scale = c.k_scale; p.v_scale = c.v_scale;
    p.pages = t.pages; p.token_row = t.token_row; p.row_stride = t.row_stride; p.n_rows = t.n_rows;
    p.n_pages = c.n_pages; p.page_size = c.page_size;
    // s = ceil(log2(page_size)), magic = ceil(2^(31+s) / page_size): exact for every position below 2^31
    int sh = 0;
    while (((int64_t)1 << sh) < c.page_size) ++sh;
    p.page_magic = (unsigned)((((uint64_t)1 << (31 + sh)) + c.page_size - 1) / c.page_size);
    p.page_shift = 31 + sh;
    p.cap = (int)std::min<int64_t>((int64_t)t.max_pages * c.page_size, 0x7FFFFFFF);
    p.q = q; p.q_stride = q_stride; p.lengths = lengths;
    p.T = T; p.H = n_heads; p.Hk = c.n_kv_heads; p.group = n_heads / c.n_kv_heads;
    p.q_tiles = ceil_div(p.group, 16); p.heads = item_heads(p.group);
    p.scale = scale; p.window = window;
    p.out = out; p.out_stride = out_stride; p.lse = lse;
    p.cuts = static_cast<int4*>(ws);
    p.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up(kAttnBlocks * sizeof(int4), 256));
    // no more shares than there can be tiles
    const int64_t longest = window > 0 ? std::min(window, p.cap) : p.cap;
    const int64_t most = (int64_t)T * p.Hk * p.q_tiles * ((longest + kTile - 1) / kTile);
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(most, kAttnBlocks));
    const bool e4m3 = c.type == MOE_KV_E4M3;
    switch (c.head_dim) {
        case 64: return attention_go<64>(p, e4m3, grid, s);
        case 96: return attention_go<96>(p, e4m3, grid, s);
        case 128: return attention_go<128>(p, e4m3, grid, s);
        case 192: return attention_go<192>(p, e4m3, grid, s);
        default: return attention_go<256>(p, e4m3, grid, s);
    }
}

}  // namespace bmoe
