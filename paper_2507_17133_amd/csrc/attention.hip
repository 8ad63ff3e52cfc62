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
// A probability goes to the second product as two bf16 that add up to it within 2^-15 (one bf16 alone: 2^-8 of it, and as errors do not cancel where
// values of v do, an error of the result beyond its own rounding).
//
// Work: the positions of every (token, key head, 16 query heads) in tiles of 128 form one line of tiles, cut into equal shares, one per block:
// one long sequence among short ones is spread over the whole GPU.  A share that begins or ends inside a sequence leaves (m, l, O) in the
// workspace, and join_kernel adds these up.  With a window and sinks, a token's positions are the sinks and then the window's, numbered through.
//
// Measured (join included): bf16, 256 tokens of 1024 to 2048 positions, 32 over 4 heads of 128, pages of 16, 146 us (769 MB, 5.3 TB/s); e4m3, three
// tokens of 65536 to 131072 positions, 64 over 8 heads of 128, 110 us (604 MB, 5.5 TB/s); one token of 1536 positions 12 us, latency;
// 256 tokens, a window of 4096 and 64 sinks of up to 8192 positions, 32 over 4 heads of 128, 361 us (2.1 GB, 5.7 TB/s).
#include "layer.h"

#include <algorithm>
#include <type_traits>

namespace bmoe {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kAttnWaves = 4, kAttnThreads = 64 * kAttnWaves;
constexpr int kStep = 32;                         // positions of a wave's step
constexpr int kAttnBlocks = 512;                  // shares at most: two blocks for each CU
// Blocks of a CU that the registers are dealt out for.  bf16 heads of 128 and more columns have 16 KB and more on their way per wave, which four waves of a
// CU keep the memory busy with; heads of 192 and 256 would spill at two.
constexpr int attention_resident(int D, bool e4m3) { return D >= 128 && !e4m3 ? 1 : 2; }
// Shares.  One block per CU for such heads: shares are longer, the parts fewer, and fewer places of memory are read at a time (256 and 512 shares, us:
// 256 tokens, 32 over 4 heads of 128, 1024 to 2048 positions 153, 160; one token of 131072 positions 100, 107; 64 of 4096 to 8192 271, 277; heads of 256, 32 over
// 2 50, 60).  Two where items are many, and so short that one's end should overlap another's work (512 tokens of up to 200, 16 heads: 99, 92).
static int most_shares(int D, bool e4m3, int64_t items)
{
    return attention_resident(D, e4m3) == 2 || (D == 128 && items >= 2 * kAttnBlocks) ? kAttnBlocks : kAttnBlocks / 2;
}

struct AttnArgs {
    const uint8_t *kc, *vc;
    int64_t head_stride;
    unsigned page_step, token_step;               // a page's and a position's stride in 16-byte steps
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
    int T, H, Hk, group, q_tiles, heads;          // heads: query heads of a key head that a wave takes (at most 16)
    int side, tile;                               // key heads side by side in a block; positions of its step
    float scale;
    int window, sinks;                            // sinks: first positions that a window leaves visible
    bf16_t* out;
    int64_t out_stride;
    float* lse;
    int4* cuts;                                   // per share: the item that it begins and does not end (token, item, shares, -)
    float* parts;                                 // per share two places of [side] parts: [heads][D] O, [heads] m, [heads] l
};

// Floats of a part: whole 16-byte pieces, so that rows of O are written and read in such.
constexpr __host__ __device__ int64_t part_floats(int heads, int D) { return (int64_t)heads * (D + 4); }

// Positions [lo, hi) that token t attends to.
__device__ __forceinline__ int2 span_of(const AttnArgs& p, int t)
{
    const int hi = min(max(p.lengths[t], 0), p.cap);
    const int row = p.token_row ? p.token_row[t] : t;
    const bool there = (unsigned)row < (unsigned)p.n_rows;
    return make_int2(p.window > 0 ? max(hi - p.window, 0) : 0, there ? hi : 0);
}
// Positions below lo that it attends to besides: the first ones.
__device__ __forceinline__ int sinks_of(const AttnArgs& p, const int2 s) { return min(p.sinks, s.x); }
__device__ __forceinline__ int tiles_of(const AttnArgs& p, const int2 s)
{
    return s.y > s.x ? (int)((unsigned)(s.y - s.x + sinks_of(p, s) - 1) / (unsigned)p.tile) + 1 : 0;
}
__device__ __forceinline__ int items_of(const AttnArgs& p) { return p.Hk / p.side * p.q_tiles; }

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
    const int items = items_of(p);
    int64_t mine = 0;
    for (int t = t0; t < t1; ++t) mine += (int64_t)tiles_of(p, span_of(p, t)) * items;
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
            const int64_t n = (int64_t)tiles_of(p, span_of(p, t)) * items;
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

// A tile of the line: its token, item (key heads side by side, and which 16 of their query heads) and number within the item.
struct Place {
    int64_t at;                                   // its number in the line
    int t, item, tile, n;                         // n: tiles of the token's items
    int lo, sinks, n_pos;                         // its positions: the first `sinks`, then those from lo on, n_pos in all
    int hk, h0, nh;                               // the wave's key head, its first query head and number of those
    const int32_t* row;                           // the token's row of the block table

    __device__ __forceinline__ void token(const AttnArgs& p)
    {
        const int2 s = span_of(p, t);
        lo = s.x;
        sinks = sinks_of(p, s);
        n_pos = s.y - s.x + sinks;
        n = tiles_of(p, s);
    }
    __device__ __forceinline__ void heads(const AttnArgs& p, int sub)
    {
        const int set = p.q_tiles == 1 ? item : item / p.q_tiles;
        hk = set * p.side + sub;
        h0 = hk * p.group + (item - set * p.q_tiles) * 16;
        nh = min(16, (hk + 1) * p.group - h0);
        row = p.pages + (int64_t)(p.token_row ? p.token_row[t] : t) * p.row_stride;
    }
    __device__ __forceinline__ void start(const AttnArgs& p, const Share& s, int sub)
    {
        at = s.first;
        t = s.token;
        token(p);
        item = (int)((at - s.before) / n);
        tile = (int)(at - s.before - (int64_t)item * n);
        heads(p, sub);
    }
    // to the next tile; false at the share's end
    __device__ __forceinline__ bool step(const AttnArgs& p, const Share& s, int sub)
    {
        if (++at >= s.end) return false;
        if (++tile < n) return true;
        tile = 0;
        if (++item == items_of(p)) {
            item = 0;
            do {
                ++t;
                token(p);
            } while (n == 0);                     // ends: the share's tiles belong to tokens that have some
        }
        heads(p, sub);
        return true;
    }
};

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

    __device__ __forceinline__ void load(const uint8_t* base, const unsigned* off, int g)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* row = base + (uint64_t)off[h] * 16;
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

// The probabilities of a lane's 8 positions as the MFMA's second operand, in two parts: cut off at bf16's bits, and what that leaves (rounded to bf16).
struct Probs {
    bf16x8 head, rest;
    template <bool FINITE>                        // v holds no infinities
    __device__ __forceinline__ void set(const float* e)
    {
        unsigned h[4];
        float r[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            // an infinite v times a rest of 0 would be NaN: a last bit keeps the rest above 0
            const unsigned a = __float_as_uint(e[i]) | (FINITE ? 0u : 1u), b = __float_as_uint(e[i + 1]) | (FINITE ? 0u : 1u);
            h[i / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            r[i] = __uint_as_float(a) - __uint_as_float(a & 0xFFFF0000u);
            r[i + 1] = __uint_as_float(b) - __uint_as_float(b & 0xFFFF0000u);
        }
        head = __builtin_bit_cast(bf16x8, make_uint4(h[0], h[1], h[2], h[3]));
        rest = __builtin_bit_cast(bf16x8, pack_bf16x8(r));
    }
};

// The 8 positions' columns [C0 + c N, + N) of V that a lane holds, N = W / 16 (8, 4 or 2).
template <int W, bool E4M3>
struct VPart {
    static constexpr int N = W / 16, BYTES = N * (E4M3 ? 1 : 2);
    struct __attribute__((aligned(BYTES))) Raw { uint8_t b[BYTES]; };
    Raw v[8];

    __device__ __forceinline__ void load(const uint8_t* base, int c0, const unsigned* off, int c)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const Raw*>(base + (c0 + c * N) * (E4M3 ? 1 : 2) + (uint64_t)off[e] * 16);
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
    __device__ __forceinline__ void add(f32x4* acc, const Probs& prob, bool all, unsigned keep) const
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
            const bf16x8 v0 = __builtin_bit_cast(bf16x8, lo), v1 = __builtin_bit_cast(bf16x8, hi);
            acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, prob.head, acc[2 * i], 0, 0, 0);
            acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, prob.head, acc[2 * i + 1], 0, 0, 0);
            acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, prob.rest, acc[2 * i], 0, 0, 0);
            acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, prob.rest, acc[2 * i + 1], 0, 0, 0);
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
    __device__ __forceinline__ void load(const uint8_t* base, const unsigned* off, int col)
    {
#pragma unroll
        for (int i = 0; i < N128; ++i) a[i].load(base, 128 * i, off, col);
        if constexpr (N64) b.load(base, 128 * N128, off, col);
        if constexpr (N32) c.load(base, 128 * N128 + 64 * N64, off, col);
    }
    __device__ __forceinline__ void add(f32x4* acc, const Probs& prob, bool all, unsigned keep) const
    {
#pragma unroll
        for (int i = 0; i < N128; ++i) a[i].add(acc + 8 * i, prob, all, keep);
        if constexpr (N64) b.add(acc + 8 * N128, prob, all, keep);
        if constexpr (N32) c.add(acc + 8 * N128 + 4 * N64, prob, all, keep);
    }
    // body(first column, how many in a row (8, 4 or 2), first of the accumulators that hold them, their register): a lane's results
    template <typename F>
    static __device__ __forceinline__ void runs(int g, F&& body)
    {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int i = 0; i < N128; ++i) body(128 * i + 8 * (4 * g + r), std::integral_constant<int, 8>{}, 8 * i, r);
            if constexpr (N64) body(128 * N128 + 4 * (4 * g + r), std::integral_constant<int, 4>{}, 8 * N128, r);
            if constexpr (N32) body(128 * N128 + 64 * N64 + 2 * (4 * g + r), std::integral_constant<int, 2>{}, 8 * N128 + 4 * N64, r);
        }
    }
};

// N floats (8, 4 or 2) in a row, in whole vectors.
template <int N>
__device__ __forceinline__ void put(float* dst, const float* v)
{
    if constexpr (N == 2) *reinterpret_cast<float2*>(dst) = make_float2(v[0], v[1]);
    else {
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(dst + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(kAttnThreads, attention_resident(D, E4M3)) attention_kernel(AttnArgs p)
{
    using K = KRows<D, E4M3>;
    using V = VRows<D, E4M3>;
    constexpr int NJ = D / 16;                            // products of V's columns
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ int64_t found[kAttnWaves + 2];
    __shared__ __attribute__((aligned(16))) unsigned places[kAttnWaves][kStep];      // where a step's positions are in the cache, in 16-byte steps
    __shared__ float stat[kAttnWaves][2][16];
    float* joined = reinterpret_cast<float*>(smem);       // [waves behind the first side][heads][D + 4]

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, c = lane & 15, sub = wave & (p.side - 1), behind = wave / p.side;       // key head, positions of the step

    // tokens with nothing to attend to
    for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
        if (tiles_of(p, span_of(p, t)) > 0) continue;
        for (int i = tid * 4; i < p.H * D; i += kAttnThreads * 4)
            *reinterpret_cast<uint2*>(p.out + (int64_t)t * p.out_stride + i) = make_uint2(0, 0);
        if (p.lse)
            for (int i = tid; i < p.H; i += kAttnThreads) p.lse[(int64_t)t * p.H + i] = -__builtin_inff();
    }

    const Share share = find_share(p, found);
    if (tid == 0) p.cuts[blockIdx.x] = make_int4(0, 0, 0, 0);
    if (share.first >= share.end) return;

    // The share's tiles follow each other without a stop: while one is worked on, the next one's K and V and the page numbers of the one after are on
    // their way, also where that is another head's or another token's.
    Place at;
    at.start(p, share, sub);
    bf16x8 q[K::S];
    K kr;
    V vr;
    unsigned koff[2], voff[8];
    // page of the lane's position (lanes 0..31) of the wave in a tile, -1 beyond the end
    auto page_of = [&](const Place& w, unsigned& in_page) -> int {
        const unsigned nth = (unsigned)w.tile * p.tile + behind * kStep + (lane & 31);
        in_page = 0;
        if (nth >= (unsigned)w.n_pos) return -1;
        const unsigned pos = nth < (unsigned)w.sinks ? nth : nth - w.sinks + w.lo;
        const unsigned pg = (unsigned)((uint64_t)pos * p.page_magic >> p.page_shift);
        in_page = pos - pg * (unsigned)p.page_size;
        return w.row[pg];
    };
    // where those positions are, by way of LDS to the lanes that load them; returns which are there
    auto place = [&](int page, unsigned in_page) -> unsigned {
        const bool there = (unsigned)page < (unsigned)p.n_pages;
        if (lane < kStep) places[wave][lane] = there ? (unsigned)page * p.page_step + in_page * p.token_step : 0;
        wave_lds_order();
#pragma unroll
        for (int h = 0; h < 2; ++h) koff[h] = places[wave][16 * h + c];
#pragma unroll
        for (int e = 0; e < 8; ++e) voff[e] = places[wave][16 * (e >> 2) + 4 * g + (e & 3)];
        wave_lds_order();
        return (unsigned)__ballot(there);                 // lanes 0..31
    };
    auto load_q = [&](const Place& w) {                   // of my head, in the order of K's columns
#pragma unroll
        for (int s = 0; s < K::S; ++s) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (c < w.nh) v = *reinterpret_cast<const uint4*>(p.q + (int64_t)w.t * p.q_stride + (int64_t)(w.h0 + c) * D + K::column(s, g));
            q[s] = __builtin_bit_cast(bf16x8, v);
        }
    };
    auto head_base = [&](const uint8_t* cache, int hk) { return cache + (int64_t)hk * p.head_stride * (E4M3 ? 1 : 2); };

    f32x4 acc[NJ];
    float m, l, to_log2 = 0.0f;
    auto begin_item = [&](const Place& w) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = -__builtin_inff();
        l = 0.0f;
        to_log2 = p.scale * (E4M3 ? p.k_scale[w.hk] : 1.0f) * 1.4426950408889634f;
    };
    // The end of an item, or of what the share has of it: the waves of a key head are joined, and the first of them writes the output or a part in
    // the workspace.  The next tile's loads stay in flight: barriers wait for LDS only.
    auto lds_sync = [&]() {
        __builtin_amdgcn_s_waitcnt(0xC07F);               // lgkmcnt(0)
        lds_barrier();
    };
    auto finish_item = [&](const Place& w, int first_tile) {
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (p.side < kAttnWaves) {
            if (g == 0) {
                stat[wave][0][c] = m;
                stat[wave][1][c] = l;
            }
            lds_sync();
            float top = -__builtin_inff();
            for (int k = sub; k < kAttnWaves; k += p.side) top = fmaxf(top, stat[k][0][c]);
            const float ref = top == -__builtin_inff() ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - ref);
            l = 0.0f;
            for (int k = sub; k < kAttnWaves; k += p.side) l += stat[k][1][c] * __builtin_amdgcn_exp2f(stat[k][0][c] - ref);
            m = top;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j][r] *= f;
            if (behind > 0 && c < w.nh) {
                float* dst = joined + ((wave - p.side) * p.heads + c) * (D + 4);
                V::runs(g, [&](int col, auto n, int j, int r) {
                    float v[n.value];
#pragma unroll
                    for (int i = 0; i < n.value; ++i) v[i] = acc[j + i][r];
                    put<n.value>(dst + col, v);
                });
            }
            lds_sync();
            if (behind == 0 && c < w.nh)
                for (int k = sub; k < kAttnWaves - p.side; k += p.side) {
                    const float* src = joined + (k * p.heads + c) * (D + 4);
                    V::runs(g, [&](int col, auto n, int j, int r) {
#pragma unroll
                        for (int i = 0; i < n.value; ++i) acc[j + i][r] += src[col + i];
                    });
                }
            lds_sync();                                   // LDS is free for the next item
        }
        if (behind > 0) return;
        const bool begins = first_tile == 0, ends = w.tile + 1 == w.n;
        if (begins && !ends && tid == 0) {
            const int64_t last_share = (w.at - w.tile + w.n - 1) / share.per;
            p.cuts[blockIdx.x] = make_int4(w.t, w.item, (int)(last_share - blockIdx.x) + 1, 0);
        }
        if (c >= w.nh) return;
        if (begins && ends) {
            const float k = l > 0.0f || l != l ? (E4M3 ? p.v_scale[w.hk] : 1.0f) / l : 0.0f;
            bf16_t* dst = p.out + (int64_t)w.t * p.out_stride + (int64_t)(w.h0 + c) * D;
            V::runs(g, [&](int col, auto n, int j, int r) {
                if constexpr (n.value == 2) *reinterpret_cast<unsigned*>(dst + col) = pack_bf16(acc[j][r] * k, acc[j + 1][r] * k);
                else {
#pragma unroll
                    for (int i = 0; i < n.value; i += 4)
                        *reinterpret_cast<uint2*>(dst + col + i) =
                            make_uint2(pack_bf16(acc[j + i][r] * k, acc[j + i + 1][r] * k), pack_bf16(acc[j + i + 2][r] * k, acc[j + i + 3][r] * k));
                }
            });
            if (p.lse && g == 0) p.lse[(int64_t)w.t * p.H + w.h0 + c] = (m + __log2f(l)) * 0.6931471805599453f;
        } else {
            float* part = p.parts + (((int64_t)2 * blockIdx.x + (begins ? 1 : 0)) * p.side + sub) * part_floats(p.heads, D);
            V::runs(g, [&](int col, auto n, int j, int r) {
                float v[n.value];
#pragma unroll
                for (int i = 0; i < n.value; ++i) v[i] = acc[j + i][r];
                put<n.value>(part + c * D + col, v);
            });
            if (g == 0) {
                part[p.heads * D + c] = m;
                part[p.heads * D + p.heads + c] = l;
            }
        }
    };
    unsigned in_page, mask, next_mask = 0;
    int page = page_of(at, in_page), first_tile = at.tile;
    mask = place(page, in_page);
    load_q(at);
    kr.load(head_base(p.kc, at.hk), koff, g);
    vr.load(head_base(p.vc, at.hk), voff, c);
    begin_item(at);
    Place next = at;
    bool more = next.step(p, share, sub);
    if (more) page = page_of(next, in_page);
    for (;;) {
        f32x4 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < K::S; ++k) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr.operand(h, k), q[k], s[h], 0, 0, 0);
        }
        const bool same = more && next.item == at.item && next.t == at.t;
        Place after = next;
        bool more_after = false;
        if (more) {
            next_mask = place(page, in_page);
            more_after = after.step(p, share, sub);
            if (more_after) page = page_of(after, in_page);
            if (!same) load_q(next);
            kr.load(head_base(p.kc, next.hk), koff, g);
        }
        if (mask) {
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
            Probs prob;
            prob.set<E4M3>(e);
            vr.add(acc, prob, all, keep);
        }
        if (more) vr.load(head_base(p.vc, next.hk), voff, c);
        if (!same) {
            finish_item(at, first_tile);
            if (!more) return;
            first_tile = next.tile;
            begin_item(next);
        }
        mask = next_mask;
        at = next;
        next = after;
        more = more_after;
    }
}

// Joins the parts of the item that share x begins and does not end.  SPREAD: a block of four waves for each head, where items are few and so cut
// into many parts; else a wave for each head: hardly any then has more than two parts to read, and the launch's time goes with its blocks.  Bound by
// its chain of dependent loads (cut, maxima, parts): 3.6 us for one token, 5.1 for 256.
template <int D, bool SPREAD>
__global__ void __launch_bounds__(256) join_kernel(AttnArgs p, int e4m3)
{
    constexpr int THREADS = SPREAD ? 256 : 64, LANES = D / 4, ROWS = THREADS / LANES;      // threads of a head, of a row of O; rows side by side
    __shared__ float4 rows[SPREAD ? 1 : 4][ROWS][LANES];
    __shared__ float sums[SPREAD ? 1 : 4][ROWS], red[4];
    const int4 cut = p.cuts[blockIdx.x];
    const int which = SPREAD ? 0 : threadIdx.x >> 6, y = SPREAD ? blockIdx.y : blockIdx.y * 4 + which, tid = threadIdx.x & (THREADS - 1);
    const int n = cut.z, set = cut.y / p.q_tiles, sub = y / p.heads, h = y - sub * p.heads;
    const int hk = set * p.side + sub, h0 = hk * p.group + (cut.y - set * p.q_tiles) * 16;
    if (n == 0 || sub >= p.side || h >= min(16, (hk + 1) * p.group - h0)) return;          // all threads of the head
    const int64_t size = part_floats(p.heads, D);
    // share x left its part in its second place, the others in their first
    auto part = [&](int i) { return p.parts + ((2 * ((int64_t)blockIdx.x + i) + (i == 0 ? 1 : 0)) * p.side + sub) * size; };
    auto sync = [&]() {
        if constexpr (SPREAD) __syncthreads();
        else wave_lds_order();
    };
    float top = -__builtin_inff();
    for (int i = tid; i < n; i += THREADS) top = fmaxf(top, part(i)[p.heads * D + h]);
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if constexpr (SPREAD) {
        if ((tid & 63) == 0) red[tid >> 6] = top;
        sync();
        top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    }
    const float ref = top == -__builtin_inff() ? 0.0f : top;
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
        rows[which][r][col / 4] = o;
        if (col == 0) sums[which][r] = sum;
    }
    sync();
    if (r != 0) return;
#pragma unroll
    for (int i = 1; i < ROWS; ++i) {
        const float4 v = rows[which][i][col / 4];
        o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
        sum += sums[which][i];
    }
    const float k = sum > 0.0f || sum != sum ? (e4m3 ? p.v_scale[hk] : 1.0f) / sum : 0.0f;
    *reinterpret_cast<uint2*>(p.out + (int64_t)cut.x * p.out_stride + (int64_t)(h0 + h) * D + col) =
        make_uint2(pack_bf16(o.x * k, o.y * k), pack_bf16(o.z * k, o.w * k));
    if (p.lse && col == 0) p.lse[(int64_t)cut.x * p.H + h0 + h] = (top + __log2f(sum)) * 0.6931471805599453f;
}

static int item_heads(int group) { return group < 16 ? group : 16; }

// Key heads that the waves of a block take side by side.  Where a token's heads lie next to each other, heads that are read at different times
// leave the memory's pages (and lines, where a row is no whole number of them) half used; side by side they share them, but every cut then
// leaves as many parts to write and join.  So: while the parts are at most 1/50 of what a share reads (1/3 where rows share lines), both
// at the table's full length.  One, two and four heads, us: 64 tokens, 32 over 8 heads of 128, 4096 to 8192 positions, page 16 303 / 289 / 285; 512 tokens,
// 16 over 16, up to 200 positions 110 / 95 / 93; e4m3, 64 tokens, 16 over 16, up to 4000 139 / 131 / 125; one token, 131072 positions 111 / 107 / 111; 256 tokens,
// 32 over 4, up to 2048 159 / 161 / 162; heads of 192, 16 tokens, 32 over 4, up to 8192 65 / 68 / 71; e4m3, heads of 96 33 / 28 / 29.  Stored head by
// head: 64 tokens of 8192 356 / 363 / 375.
static int heads_side_by_side(const moe_kv_cache& c, int heads, int64_t T, int64_t longest)
{
    if (c.n_kv_heads == 1 || c.head_stride >= c.token_stride) return 1;
    const int row = c.head_dim * (c.type == MOE_KV_E4M3 ? 1 : 2);
    const double share = (double)T * c.n_kv_heads * longest * 2 * row / kAttnBlocks, most = share * (row % 128 ? 0.33 : 0.02);
    int side = 4;
    while (side > 1 && (c.n_kv_heads % side != 0 || 16.0 * side * heads * c.head_dim > most)) side /= 2;
    return side;
}

size_t attention_workspace_bytes(const moe_kv_cache& c, int T, int n_heads)
{
    (void)T;                                              // the shares are as many for every T, and each has at most four heads' parts
    const int heads = item_heads(n_heads / c.n_kv_heads);
    const int side = c.n_kv_heads % 4 == 0 ? 4 : c.n_kv_heads % 2 == 0 ? 2 : 1;
    return align_up(kAttnBlocks * sizeof(int4), 256) + align_up((size_t)2 * kAttnBlocks * side * part_floats(heads, c.head_dim) * sizeof(float), 256);
}

// A row of O in LDS is 4 floats longer, so that the heads of a wave write to different banks.
template <int D>
static size_t attention_lds(int heads, int side) { return (size_t)(kAttnWaves - side) * heads * (D + 4) * sizeof(float); }

template <int D>
static hipError_t attention_init()
{
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_kernel<D, true>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)attention_lds<D>(16, 1));
    if (e != hipSuccess) return e;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_kernel<D, false>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)attention_lds<D>(16, 1));
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
    const size_t lds = attention_lds<D>(p.heads, p.side);
    if (e4m3) hipLaunchKernelGGL((attention_kernel<D, true>), dim3(grid), dim3(kAttnThreads), lds, s, p);
    else hipLaunchKernelGGL((attention_kernel<D, false>), dim3(grid), dim3(kAttnThreads), lds, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || grid == 1) return e;           // one share: nothing is cut
    const int64_t items = (int64_t)p.T * (p.Hk / p.side) * p.q_tiles;
    const int heads = p.heads * p.side;
    if (items * 4 >= grid) hipLaunchKernelGGL((join_kernel<D, false>), dim3(grid, ceil_div(heads, 4)), dim3(256), 0, s, p, e4m3 ? 1 : 0);
    else hipLaunchKernelGGL((join_kernel<D, true>), dim3(grid, heads), dim3(256), 0, s, p, e4m3 ? 1 : 0);
    return hipGetLastError();
}

hipError_t launch_attention(const moe_kv_cache& c, const moe_block_table& t, const bf16_t* q, int64_t q_stride, int n_heads, int T,
                            const int32_t* lengths, float scale, int window, int sinks, bf16_t* out, int64_t out_stride, float* lse, void* ws,
                            hipStream_t s)
{
    AttnArgs p;
    p.kc = static_cast<const uint8_t*>(c.k); p.vc = static_cast<const uint8_t*>(c.v);
    const int per16 = c.type == MOE_KV_E4M3 ? 16 : 8;
    p.head_stride = c.head_stride;
    p.page_step = (unsigned)(c.page_stride / per16);
    p.token_step = (unsigned)(c.token_stride / per16);
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
    p.scale = scale; p.window = window; p.sinks = sinks;
    p.out = out; p.out_stride = out_stride; p.lse = lse;
    p.cuts = static_cast<int4*>(ws);
    p.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up(kAttnBlocks * sizeof(int4), 256));
    // no more shares than there can be tiles
    const int64_t longest = window > 0 ? std::min<int64_t>((int64_t)window + sinks, p.cap) : p.cap;
    p.side = heads_side_by_side(c, p.heads, T, longest);
    p.tile = kStep * kAttnWaves / p.side;
    const int64_t most = (int64_t)T * (p.Hk / p.side) * p.q_tiles * ((longest + p.tile - 1) / p.tile);
    const bool e4m3 = c.type == MOE_KV_E4M3;
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(most, most_shares(c.head_dim, e4m3, (int64_t)T * (p.Hk / p.side) * p.q_tiles)));
    switch (c.head_dim) {
        case 64: return attention_go<64>(p, e4m3, grid, s);
        case 96: return attention_go<96>(p, e4m3, grid, s);
        case 128: return attention_go<128>(p, e4m3, grid, s);
        case 192: return attention_go<192>(p, e4m3, grid, s);
        default: return attention_go<256>(p, e4m3, grid, s);
    }
}

}  // namespace bmoe
