// What rows of logits say: log of the sum of exponentials, log probabilities and ranks of given tokens, entropy, the best alternatives.
//
//   m = max x,  S = sum e^(x - m),  U = sum e^(x - m) (x - m):      lse = m + log S,  log p_g = (x_g - m) - log S,  H = log S - U / S
//   rank of g = #{x > x_g} + #{x = x_g, lower number};      the n_top first entries of the order (falling x, rising number)
//
// Both terms of H are at least 0, so nothing cancels.  A row is read once: a wave takes a slice of it into registers, where the passes that follow
// (maximum, sums, ranks, the best) find it; join_rows puts the slices of a row together by the same formulas.
#include "draft.h"

#include <algorithm>

namespace bmoe {
namespace {

// A slice has one wave, with nobody to wait for (2112 rows of 131072 entries, four given tokens and eight alternatives: slices of one, two, four and eight
// waves 242, 247, 256 and 371 us).
constexpr int kThreads = 64;
constexpr int kJoinThreads = 256, kJoinWaves = kJoinThreads / 64;
// Slices from which longer ones are taken: six for each CU.  fp32, one given token and 20 alternatives, 50021 entries: 16 rows with 384 21.5 us, with 1536 19.9; 32 rows with 768 22.5, with 1536
// 20.9; 67 rows with 1536 24.6, with 3072 22.6, with 6144 23.7; but 16 rows of 131072 23.0 with 1536 and 27.2 with 3072.
constexpr int kEnough = 1536;
// Entries that a block sorts.  With 256 the same; with 1024, whose LDS leaves room for fewer blocks, 2112 rows of 131072 entries 266 us instead of 229.
constexpr int kCandidates = 512;
constexpr int kLongest = 32;                      // entries of a thread at most: slices of 2048
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

struct LogprobArgs {
    const char* logits;
    int64_t stride;                               // in elements
    const int32_t* tokens;
    int64_t tokens_stride;
    float* logprob;
    int32_t* rank;
    float *lse, *entropy;
    int32_t* top_id;
    float* top_logprob;
    int T, V, G, N, slices;
    float4* stats;                                // [T * slices]: m, S, U (U in powers of two)
    int* before;                                  // [T * slices][G]
    float2* best;                                 // [T * slices][N]: value, number (as bits)
};

// A value of the order (falling value, rising number).
struct Entry {
    float x;
    int id;
};
__device__ __forceinline__ bool precedes(const Entry a, const Entry b) { return a.x > b.x || (a.x == b.x && a.id < b.id); }

// Running sums about a maximum; joins as the exponentials do.
struct Stats {
    float m, s, u;
    __device__ __forceinline__ void join(const Stats o)
    {
        const float top = fmaxf(m, o.m), ref = top == -__builtin_inff() ? 0.0f : top;
        auto moved = [&](const Stats a, float& s2, float& u2) {
            // e^(x - top) = e^(x - m) f; what has no finite maximum has no terms (or a NaN among them)
            const float d = a.m == -__builtin_inff() ? 0.0f : (a.m - ref) * kLog2e, f = a.m == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(d);
            s2 = f * a.s;
            u2 = f == 0.0f ? f * a.u : f * (a.u + d * a.s);
        };
        float s1, u1, s2, u2;
        moved(*this, s1, u1);
        moved(o, s2, u2);
        m = top;
        s = s1 + s2;
        u = u1 + u2;
    }
};

// What is left to say about a row once its sums are known.
struct Row {
    float m, log_s, lse, entropy;
    bool none;                                    // no distribution
    __device__ __forceinline__ explicit Row(const Stats a) : m(a.m)
    {
        none = a.s != a.s;
        log_s = __builtin_amdgcn_logf(a.s) * kLn2;
        lse = none ? a.s : m == -__builtin_inff() ? m : m + log_s;
        entropy = none ? a.s : m == -__builtin_inff() ? 0.0f : log_s - a.u * kLn2 / a.s;
    }
    __device__ __forceinline__ float of(float x) const { return none ? lse : x == -__builtin_inff() ? x : x - m - log_s; }
};

// The value of the lane that is STEP on in a butterfly whose earlier steps have made groups of STEP lanes alike (so a mirrored order serves as well).
template <int STEP>
__device__ __forceinline__ int across_bits(int i)
{
    if constexpr (STEP == 1) return __builtin_amdgcn_update_dpp(i, i, 0xB1, 0xF, 0xF, false);          // quad_perm 1 0 3 2
    else if constexpr (STEP == 2) return __builtin_amdgcn_update_dpp(i, i, 0x4E, 0xF, 0xF, false);     // quad_perm 2 3 0 1
    else if constexpr (STEP == 4) return __builtin_amdgcn_update_dpp(i, i, 0x141, 0xF, 0xF, false);    // row_half_mirror
    else if constexpr (STEP == 8) return __builtin_amdgcn_update_dpp(i, i, 0x140, 0xF, 0xF, false);    // row_mirror
    else {
        static_assert(STEP == 16 || STEP == 32, "steps of a wave");
        const auto two = STEP == 16 ? __builtin_amdgcn_permlane16_swap((unsigned)i, (unsigned)i, false, false)
                                    : __builtin_amdgcn_permlane32_swap((unsigned)i, (unsigned)i, false, false);
        // one of the two is the lane's own
        const bool upper = (threadIdx.x & STEP) != 0;
        return (int)(upper ? two[0] : two[1]);
    }
}
template <int STEP>
__device__ __forceinline__ float across(float v) { return __int_as_float(across_bits<STEP>(__float_as_int(v))); }
template <int STEP>
__device__ __forceinline__ unsigned across(unsigned v) { return (unsigned)across_bits<STEP>((int)v); }
template <typename T, typename F>
__device__ __forceinline__ T wave_fold(T v, F&& f)
{
    v = f(v, across<1>(v));
    v = f(v, across<2>(v));
    v = f(v, across<4>(v));
    v = f(v, across<8>(v));
    v = f(v, across<16>(v));
    return f(v, across<32>(v));
}
__device__ __forceinline__ float wave_max(float v) { return wave_fold(v, [](float a, float b) { return fmaxf(a, b); }); }
template <typename T>
__device__ __forceinline__ T wave_sum(T v) { return wave_fold(v, [](T a, T b) { return a + b; }); }

// Whole numbers in the order of floats.
__device__ __forceinline__ unsigned order_of(float x)
{
    const unsigned b = __float_as_uint(x);
    return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(unsigned u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }

// A bound that at least n of the wave's 64 values reach (n <= 64): the n-th largest one, cut off to the upper 16 bits of its order.  (The least of the largest
// values of n groups costs a third, but ten times as many entries reach it: 67 x 50021, 20 alternatives 119 us instead of 21.)
__device__ __forceinline__ float reached_by(float v, int n)
{
    const unsigned key = order_of(v) >> 16;
    unsigned at = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
        const unsigned higher = at | 1u << b;
        if (__builtin_popcountll(__ballot(key >= higher)) >= n) at = higher;
    }
    return at < 0x0080u ? -__builtin_inff() : of_order(at << 16);
}

// LDS of the choice of a block's best entries.
template <int WAVES>
struct Choice {
    float bound[WAVES];
    int found;
    Entry list[kCandidates];
    Entry won[WAVES];
};

// The first n of the block's entries in order, to put(place, entry); a place that has none gets (-infinity, none).  `most`: the thread's largest value;
// each(bound, f): f(entry) for every entry of the thread that reaches bound.  Entries that reach a bound that n of them are known to reach hold the first n; where too many
// do, as where all are alike, the entries are taken out one by one.
template <int WAVES, typename Each, typename Put>
__device__ __forceinline__ void choose(Choice<WAVES>& c, int n, float most, Each&& each, Put&& put)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float mine = reached_by(most, n);
    if (lane == 0) c.bound[wave] = mine;
    if (tid == 0) c.found = 0;
    __syncthreads();
    float bound = c.bound[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) bound = fmaxf(bound, c.bound[w]);
    each(bound, [&](const Entry e) {
        const int at = atomicAdd(&c.found, 1);
        if (at < kCandidates) c.list[at] = e;
    });
    __syncthreads();
    const int found = c.found;
    if (found <= kCandidates) {
        // an entry's place: how many of the others precede it, counted by four neighbouring lanes
        for (int i0 = 0; i0 < max(found, n); i0 += (64 * WAVES) / 4) {
            const int i = i0 + tid / 4;
            const Entry e = i < found ? c.list[i] : Entry{-__builtin_inff(), 0x7FFFFFFF};
            int at = 0;
#pragma unroll 4
            for (int j = tid & 3; j < found; j += 4) at += precedes(c.list[j], e) ? 1 : 0;
            at += __shfl_xor(at, 1);
            at += __shfl_xor(at, 2);
            if ((tid & 3) == 0 && (i < found ? at : i) < n) put(i < found ? at : i, e);
        }
        return;
    }
    Entry last{__builtin_inff(), -1};
    for (int i = 0; i < n; ++i) {
        Entry top{-__builtin_inff(), 0x7FFFFFFF};
        each(-__builtin_inff(), [&](const Entry e) {
            if (precedes(last, e) && precedes(e, top)) top = e;
        });
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            const Entry e{__shfl_xor(top.x, o), __shfl_xor(top.id, o)};
            if (precedes(e, top)) top = e;
        }
        if (lane == 0) c.won[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            if (precedes(c.won[w], top)) top = c.won[w];
        __syncthreads();
        if (tid == 0) put(i, top);
        last = top;
    }
}

template <bool FP32>
__device__ __forceinline__ float logit(const char* row, int i)
{
    if constexpr (FP32) return reinterpret_cast<const float*>(row)[i];
    else return __uint_as_float((unsigned)reinterpret_cast<const uint16_t*>(row)[i] << 16);
}

template <bool FP32>
__device__ __forceinline__ Entry given_token(const LogprobArgs& p, const char* row, int t, int k)
{
    const int id = p.tokens[(int64_t)t * p.tokens_stride + k];
    const bool real = (unsigned)id < (unsigned)p.V;
    return Entry{real ? logit<FP32>(row, id) : 0.0f, real ? id : -1};
}

// One slice of a row, EACH entries a thread.  Large calls are bound by HBM as long as sums are all that is asked for (2112 rows of 131072 entries 95 us, 5.8 TB/s),
// by vector instructions with ranks (two per entry and given token: four tokens 168 us) and alternatives (eight 149 us, both 229 in a row of calls: 217 and the join's 12); small ones by their launches.
template <bool FP32, int EACH>
__global__ void __launch_bounds__(kThreads) slice_kernel(LogprobArgs p)
{
    constexpr int PER = FP32 ? 4 : 8, VECS = EACH / PER;          // entries of a 16-byte load
    __shared__ int counts[MOE_MAX_GIVEN + 1];             // given tokens come in twos
    __shared__ Entry given[MOE_MAX_GIVEN];
    __shared__ Choice<1> choice;
    const int tid = threadIdx.x;
    const int t = blockIdx.x / p.slices, slice = blockIdx.x - t * p.slices;
    const char* row = p.logits + (int64_t)t * p.stride * (FP32 ? 4 : 2);
    // slices begin on 16-byte lines, the first of them before the row where that begins inside one
    const int begin = slice * EACH * kThreads - (int)((reinterpret_cast<uintptr_t>(row) & 15) / (FP32 ? 4 : 2)), end = begin + EACH * kThreads;
    const bool inner = begin >= 0 && end <= p.V;
    float x[EACH];
    if (inner) {
        uint4 raw[VECS];
#pragma unroll
        for (int j = 0; j < VECS; ++j)
            raw[j] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
                                                   row + (int64_t)(begin + (j * kThreads + tid) * PER) * (FP32 ? 4 : 2))));
        if (tid < p.G) given[tid] = given_token<FP32>(p, row, t, tid);
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            if constexpr (FP32) {
                x[4 * j] = __uint_as_float(raw[j].x); x[4 * j + 1] = __uint_as_float(raw[j].y);
                x[4 * j + 2] = __uint_as_float(raw[j].z); x[4 * j + 3] = __uint_as_float(raw[j].w);
            } else unpack_bf16(raw[j], x + 8 * j);
        }
    } else {
        if (tid < p.G) given[tid] = given_token<FP32>(p, row, t, tid);
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            const int at = begin + (j * kThreads + tid) * PER;
            if (at >= 0 && at + PER <= p.V) {
                const uint4 raw = *reinterpret_cast<const uint4*>(row + (int64_t)at * (FP32 ? 4 : 2));
                if constexpr (FP32) {
                    x[4 * j] = __uint_as_float(raw.x); x[4 * j + 1] = __uint_as_float(raw.y);
                    x[4 * j + 2] = __uint_as_float(raw.z); x[4 * j + 3] = __uint_as_float(raw.w);
                } else unpack_bf16(raw, x + 8 * j);
            } else {
#pragma unroll
                for (int e = 0; e < PER; ++e) x[PER * j + e] = (unsigned)(at + e) < (unsigned)p.V ? logit<FP32>(row, at + e) : -__builtin_inff();
            }
        }
    }
    float most = -__builtin_inff(), best[VECS];
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        best[j] = max3(x[PER * j], x[PER * j + 1], x[PER * j + 2]);
        if constexpr (PER == 8) best[j] = max3(max3(best[j], x[8 * j + 3], x[8 * j + 4]), x[8 * j + 5], x[8 * j + 6]);
        best[j] = max3(best[j], x[PER * j + PER - 1], -__builtin_inff());       // a number, if only that one
        most = fmaxf(most, best[j]);
    }
    Stats a;
    a.m = wave_max(most);
    const float ref = a.m == -__builtin_inff() ? 0.0f : a.m;
    a.s = a.u = 0.0f;
    // x log2 e - c in one instruction, c the rounded m log2 e.  All terms are off by the same factor 2^-g then, which is known.
    const float c = ref * kLog2e, g = -__builtin_fmaf(ref, kLog2e, -c);
    const bool small = fabsf(ref) <= 1048576.0f;
    if (small) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float d = __builtin_fmaf(x[i], kLog2e, -c), e = __builtin_amdgcn_exp2f(d);
            a.s += e;
            a.u = __builtin_fmaf(e, d, a.u);
        }
        const float f = __builtin_amdgcn_exp2f(g);
        a.u = f * __builtin_fmaf(g, a.s, a.u);
        a.s *= f;
    }
    if (!small || __any(a.u != a.u)) {            // large values, or -infinities (0 times one is NaN)
        a.s = a.u = 0.0f;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float d = x[i] - ref, e = __builtin_amdgcn_exp2f(d * kLog2e);
            a.s += e;
            a.u = __builtin_fmaf(e, fmaxf(d, -1000.0f) * kLog2e, a.u);
        }
    }
    a.s = wave_sum(a.s);
    a.u = wave_sum(a.u);
    __syncthreads();                              // given tokens
    // ranks, two given tokens at a time (a lane's two counts in one number)
    const Entry held = p.G ? given[min(tid, p.G - 1)] : Entry{0.0f, -1};
    for (int k = 0; k < p.G; k += 2) {
        int n[2] = {0, 0};
        unsigned mine = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int from = min(k + h, p.G - 1);
            const Entry e{__int_as_float(__builtin_amdgcn_readlane(__float_as_int(held.x), from)), __builtin_amdgcn_readlane(held.id, from)};
            if (inner && (e.id < begin || e.id >= end) && e.x > -__builtin_inff()) {
                // a slice before its number: what is at least x_g, that is above the value below it; behind: what is above x_g
                const unsigned b = __float_as_uint(e.x + 0.0f);
                const float below = b == 0 ? -1.401298464324817e-45f : __uint_as_float((int)b < 0 ? b + 1 : b - 1), bound = e.id >= end ? below : e.x;
                unsigned m = 0;
#pragma unroll
                for (int j = 0; j < VECS; ++j)
                    if (__any(best[j] > bound)) {         // for a likely token hardly ever
#pragma unroll
                        for (int i = 0; i < PER; ++i) m += x[PER * j + i] > bound ? 1 : 0;
                    }
                mine |= m << (16 * h);
            } else {
                int b = begin;
                asm volatile("" : "+v"(b));               // numbers are made here each time, not kept for all entries
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const int id = b + (i / PER * kThreads + tid) * PER + i % PER;
                    n[h] += __builtin_popcountll(__ballot((unsigned)id < (unsigned)p.V && precedes(Entry{x[i], id}, e)));
                }
            }
        }
        mine = wave_sum(mine);
        if (tid < 2) counts[k + tid] = tid ? n[1] + (mine >> 16) : n[0] + (mine & 0xFFFFu);
    }
    auto each = [&](float bound, auto&& f) {
#pragma unroll
        for (int j = 0; j < VECS; ++j)
#pragma unroll
            for (int i = PER * j; i < PER * j + PER; ++i)
                if (x[i] >= bound) {
                    const int id = begin + (j * kThreads + tid) * PER + i % PER;
                    if ((unsigned)id < (unsigned)p.V) f(Entry{x[i], id});
                }
    };
    if (p.slices > 1) {
        if (tid == 0) p.stats[blockIdx.x] = make_float4(a.m, a.s, a.u, 0.0f);
        if (p.N) choose(choice, p.N, most, each, [&](int i, const Entry e) { p.best[(int64_t)blockIdx.x * p.N + i] = make_float2(e.x, __int_as_float(e.id)); });
        if (p.G) __syncthreads();
        if (tid < p.G) p.before[(int64_t)blockIdx.x * p.G + tid] = counts[tid];
        return;
    }
    const Row r(a);
    if (tid == 0) {
        if (p.lse) p.lse[t] = r.lse;
        if (p.entropy) p.entropy[t] = r.entropy;
    }
    if (p.N)
        choose(choice, p.N, most, each, [&](int i, const Entry e) {
            if (p.top_id) p.top_id[(int64_t)t * p.N + i] = r.none ? -1 : e.id;
            if (p.top_logprob) p.top_logprob[(int64_t)t * p.N + i] = r.of(e.x);
        });
    if (p.G) __syncthreads();
    if (tid < p.G) {
        const Entry e = given[tid];
        if (p.logprob) p.logprob[(int64_t)t * p.G + tid] = e.id < 0 ? 0.0f : r.of(e.x);
        if (p.rank) p.rank[(int64_t)t * p.G + tid] = e.id < 0 || r.none ? -1 : counts[tid];
    }
}

// A block for each row whose slices are joined, in whole numbers or a fixed order.  What does not depend on the sums is asked for first, and counts are added up by all
// threads (2112 rows of 64 slices, four given tokens and eight alternatives: 12 to 14 us; a thread for each token 28).  The slices' best entries are read a second time where they are chosen from: they are many only in rows of many slices.
template <bool FP32>
__global__ void __launch_bounds__(kJoinThreads) join_rows(LogprobArgs p)
{
    __shared__ Stats stats[kJoinWaves];
    __shared__ Choice<kJoinWaves> choice;
    __shared__ int ranks[MOE_MAX_GIVEN];
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t first = (int64_t)t * p.slices;
    const float2* best = p.best + first * p.N;
    const int n_best = p.slices * p.N, n_before = p.slices * p.G;
    // asked for ahead of what they are needed behind
    const int* before = p.before + first * p.G;
    const int ahead = tid < n_before ? before[tid] : 0, id = tid < p.G ? p.tokens[(int64_t)t * p.tokens_stride + tid] : -1;
    const bool real = (unsigned)id < (unsigned)p.V;
    const float x = real ? logit<FP32>(p.logits + (int64_t)t * p.stride * (FP32 ? 4 : 2), id) : 0.0f;
    if (tid < p.G) ranks[tid] = 0;
    float most = -__builtin_inff();
#pragma unroll 4
    for (int i = tid; i < n_best; i += kJoinThreads) most = fmaxf(most, best[i].x);
    Stats a{-__builtin_inff(), 0.0f, 0.0f};
    for (int i = tid; i < p.slices; i += kJoinThreads) {
        const float4 v = p.stats[first + i];
        a.join(Stats{v.x, v.y, v.z});
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        Stats b{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.u, o)};
        a.join(b);
    }
    if (lane == 0) stats[wave] = a;
    __syncthreads();
    a = stats[0];
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) a.join(stats[w]);
    const Row r(a);
    if (tid == 0) {
        if (p.lse) p.lse[t] = r.lse;
        if (p.entropy) p.entropy[t] = r.entropy;
    }
    if (p.G) {                                    // whole numbers: any order of addition is the same
        if (tid < n_before) atomicAdd(&ranks[(unsigned)tid % (unsigned)p.G], ahead);
        for (int i = tid + kJoinThreads; i < n_before; i += kJoinThreads) atomicAdd(&ranks[(unsigned)i % (unsigned)p.G], before[i]);
        __syncthreads();
        if (tid < p.G) {
            if (p.logprob) p.logprob[(int64_t)t * p.G + tid] = real ? r.of(x) : 0.0f;
            if (p.rank) p.rank[(int64_t)t * p.G + tid] = real && !r.none ? ranks[tid] : -1;
        }
    }
    if (p.N)
        choose(choice, p.N, most,
               [&](float bound, auto&& f) {
#pragma unroll 4
                   for (int i = tid; i < n_best; i += kJoinThreads) {
                       const float2 v = best[i];
                       if (v.x >= bound && __float_as_int(v.y) != 0x7FFFFFFF) f(Entry{v.x, __float_as_int(v.y)});
                   }
               },
               [&](int i, const Entry e) {
                   if (p.top_id) p.top_id[(int64_t)t * p.N + i] = r.none ? -1 : e.id;
                   if (p.top_logprob) p.top_logprob[(int64_t)t * p.N + i] = r.of(e.x);
               });
}

constexpr int slices_of(int V, int each, int ahead = 7) { return (V + ahead + each * kThreads - 1) / (each * kThreads); }      // up to 7 places before a row that begins inside a line

// Entries of a thread: the longest slices that still make enough blocks, or the shortest ones.
int entries_each(int64_t T, int V)
{
    int each = kLongest;
    while (each > 8 && T * slices_of(V, each) < kEnough) each /= 2;
    return each;
}

template <bool FP32>
hipError_t go(const LogprobArgs& p, int each, hipStream_t s)
{
    const dim3 grid((unsigned)(p.T * p.slices)), threads(kThreads);
    switch (each) {
        case 8: hipLaunchKernelGGL((slice_kernel<FP32, 8>), grid, threads, 0, s, p); break;
        case 16: hipLaunchKernelGGL((slice_kernel<FP32, 16>), grid, threads, 0, s, p); break;
        default: hipLaunchKernelGGL((slice_kernel<FP32, kLongest>), grid, threads, 0, s, p); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.slices == 1) return e;
    hipLaunchKernelGGL((join_rows<FP32>), dim3(p.T), dim3(kJoinThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace

size_t logprob_workspace_bytes(int64_t T, int V, int n_given, int n_top)
{
    // fewer rows may be cut into shorter slices, but then into fewer than twice kEnough of them
    const int64_t parts = std::max(T * slices_of(V, kLongest), std::min<int64_t>(T * slices_of(V, 8), 2 * kEnough));
    return align_up(parts * sizeof(float4), 256) + align_up(parts * sizeof(int) * n_given, 256) + align_up(parts * sizeof(float2) * n_top, 256);
}

hipError_t launch_logprobs(const moe_logprob_args& a, void* ws, hipStream_t s)
{
    LogprobArgs p;
    p.logits = static_cast<const char*>(a.logits); p.stride = a.stride;
    p.tokens = a.tokens; p.tokens_stride = a.tokens_stride;
    p.logprob = a.logprob; p.rank = a.rank; p.lse = a.lse; p.entropy = a.entropy;
    p.top_id = a.top_id; p.top_logprob = a.top_logprob;
    p.V = a.V;
    p.G = a.logprob || a.rank ? a.n_given : 0;
    p.N = a.top_id || a.top_logprob ? a.n_top : 0;
    const int each = entries_each(a.T, a.V), size = a.type == MOE_LOGITS_FP32 ? 4 : 2;
    const bool aligned = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && (a.T == 1 || a.stride * size % 16 == 0);
    p.slices = slices_of(a.V, each, aligned ? 0 : 16 / size - 1);
    const size_t parts = (size_t)a.T * p.slices;
    p.stats = static_cast<float4*>(ws);
    p.before = reinterpret_cast<int*>(static_cast<char*>(ws) + align_up(parts * sizeof(float4), 256));
    p.best = reinterpret_cast<float2*>(reinterpret_cast<char*>(p.before) + align_up(parts * sizeof(int) * p.G, 256));
    // a launch takes less than 2^32 threads: rows that need more go in several
    const int most = (int)(((int64_t)1 << 31) / kThreads / p.slices);
    for (int t = 0; t < a.T; t += p.T) {
        p.T = std::min(most, a.T - t);
        const hipError_t e = a.type == MOE_LOGITS_FP32 ? go<true>(p, each, s) : go<false>(p, each, s);
        if (e != hipSuccess) return e;
        auto on = [&](auto*& q, int64_t n) {
            if (q) q += n;
        };
        on(p.logits, (int64_t)p.T * a.stride * size);
        on(p.tokens, (int64_t)p.T * a.tokens_stride);
        on(p.logprob, (int64_t)p.T * a.n_given); on(p.rank, (int64_t)p.T * a.n_given);
        on(p.lse, p.T); on(p.entropy, p.T);
        on(p.top_id, (int64_t)p.T * a.n_top); on(p.top_logprob, (int64_t)p.T * a.n_top);
    }
    return hipSuccess;
}

}  // namespace bmoe
