// Attention of sequences' new tokens (a tree of drafted ones, a chunk of a prompt) over a paged key-value cache, each tile of it read once for all
// the rows that share it.
//
//   out = sum_p softmax_p(scale q . k_p) v_p in one pass: running maximum m, running sum l and the running weighted sum O of v.
//
// A sequence's rows are its (new token, query head of a key head) pairs, token by token.  An item is a tile of up to ROWS rows of one key head; a block
// goes through the item's positions STEP at a time.  K and V of a step lie in LDS as [64 columns][position], 16-byte pieces of a row exchanged so that
// neither of the two ways they are read meets a bank twice; while one step is worked on the next is on its way to registers (e4m3 is widened
// when it goes to LDS).  Each wave has 32 of the rows and, where rows are few, its part of the positions:
//   S [32 positions][32 rows] = K Q^T,     O^T [D][32 rows] += V^T P^T          (32 x 32 x 16 MFMAs)
// S leaves lane (g, c) = (lane / 32, lane % 32) with row c at positions 8 j + 4 g + 0..3: already the layout of P^T as the second operand, its 8
// positions in the order {16 t + 4 g + 0..3, 16 t + 8 + 4 g + 0..3}; V^T is read in the same order by transposing LDS reads.  Maximum, sum and rescaling
// are per row = per lane and its other half.  The maximum that exponentials refer to follows the true one at a distance of at most 2^kSlack, so O is
// hardly ever rescaled.
//
// A position counts for some rows of an item and not for others; its probability is then 0 for these, but 0 times a NaN or an infinity of V is NaN.  A
// part whose result is not finite is computed once more with the second product in fp32 lane by lane, which skips such places.
//
// A probability's rounding for the second product: beside an e4m3 V to fp16, which fp16 holds exactly (2^-11 of it: error of a result against 64 bits 0.0017 of the norm, which is
// the result's own rounding).  Beside a bf16 V, sequences of up to 128 rows have it as two bf16, cut off at bf16's bits and the rest, which add up to it within 2^-15 (0.0017);
// longer ones as one (half a step, 2^-8 of it: 0.0023), where a second product costs a quarter of the time (see pick).
//
// What bounds it: a CU's matrix and vector instructions, which hardly overlap.  (Beside a step of 32 x 32 x 16 MFMAs that takes 16.6 ns alone, fused multiply-adds
// of 10.1 ns alone make 22.4.)  So the loop has its products, LDS reads and the softmax of the neighbouring blocks in slots of a fixed order: block n is
// weighed, n + 1 has its exponentials taken, n + 2 its scores computed.  Measured, join included: 16384 tokens of four prompts, a window of
// 4096, 56 over 8 heads of 128, bf16 2050 to 2150 us on different cards, 900 to 940 TFLOP/s (matrix pipe 0.43 of the cycles, vector 0.51 of the issue); 64 trees of 33 tokens behind up
// to 8192 positions, 64 over 8 heads, e4m3 472 to 490 us, 1.8 TB/s and 650 TFLOP/s (0.34 and 0.44: 24 us are the join, and items begin and end); a tree of 26 tokens behind
// 2048 positions 26 us, latency.  Without that order, or with LDS rows that were not turned, the first took 2614.
#include "draft.h"
#include "chunk_span.h"

#include <algorithm>
#include <type_traits>

namespace bmoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kChunkShares = 512;                 // shares of the line of steps at most
constexpr int kBetween = 5;                       // what an item costs besides its steps, in steps; with 1 a prompt of 2048 tokens took 138 us, with 5 84
// By how many steps an item may exceed a share where each has a block.  8 chunks of 256 tokens behind up to 512 and up to 1792 positions: with 0 64 and 101 us, with 4 44 and 101, with 16 44 and
// 82, with 64 the same; behind up to 4500, 8000 and 12000 with 16 171, 272 and 373, with 64 169, 260 and 375.
constexpr int kUneven = 16;
constexpr int kMostShared = 1024;                 // sequences of a call whose steps are dealt out in shares: what LDS has room for
// How far (in powers of two) scores may exceed the maximum that they refer to.  0, so that O is rescaled whenever the maximum grows: 4096 tokens, 16 over 4
// heads of 256, 318 us, with 4 264; 16 x 16 drafted tokens 94 and 80.  2^4 costs the probabilities no bits: they are floating-point, and sums are fp32.
constexpr float kSlack = 4.0f;
constexpr int kMostContext = 0x7FFE0000;          // so that positions of new tokens stay in 32 bits

// Rows of a block 32 * WM, one of WM waves each; WK waves share the positions of a step, PB blocks of 32 each.
template <int D_, bool E4M3_, int WM_, int WK_, int PB_>
struct Shape {
    static constexpr int D = D_, WM = WM_, WK = WK_, PB = PB_;
    static constexpr bool E4M3 = E4M3_, TWO = false;
    static constexpr int WAVES = WM * WK, THREADS = 64 * WAVES;
    static_assert(WAVES == 2 || WAVES == 4 || WAVES == 8, "waves of a block");
    static constexpr int ROWS = 32 * WM, STEP = 32 * PB * WK;
    static constexpr int N64 = D / 64, N32 = D % 64 / 32;                     // panels of 64 columns, and one of 32
    static constexpr int TILE = STEP * D * 2;                                 // bytes of K (of V) of a step in LDS
    static constexpr int KS = D / 16, VS = D / 32;                            // products along D, blocks of 32 columns of V
    static constexpr int LEAD = 2 / PB;                                       // steps that K is ahead of V
    static constexpr int AHEAD = 2;                                           // slots that LDS reads are ahead of the products
    static constexpr int SCRATCH = WAVES * 32 * 32 * 4;                       // probabilities of the careful second product
    static constexpr int JOIN = (WK - 1) * WM * 32 * (D + 4) * 4;        // parts of waves that share rows
    static constexpr int FLAGS = std::max({4 * TILE, 2 * TILE + SCRATCH, JOIN}), LDS = FLAGS + 64;       // two steps of K, two of V, or one of each and the scratch, or the parts
    static constexpr int RESIDENT = WAVES <= 4 && LDS <= 80 * 1024 && D <= 128 ? 2 : 1;       // blocks of a CU
    static_assert(PB <= 2 && LDS <= 160 * 1024 && LDS >= kMostShared * 4 + 96, "LDS");
    // floats of a part: [ROWS][D] O, [ROWS] m, [ROWS] l
    static constexpr int64_t PART = (int64_t)ROWS * (D + 2);
};
// The same with two bf16 for a probability.
template <class S>
struct Fine : S {
    static_assert(!S::E4M3, "fp16 holds them well enough");
    static constexpr bool TWO = true;
};

struct ChunkArgs {
    const char *kc, *vc;
    int64_t head_stride;                          // bytes
    unsigned page_step, token_step;               // a page's and a position's stride in 16-byte steps
    const float *k_scale, *v_scale;
    const int32_t *pages, *row_of;
    int64_t row_stride;
    int n_rows, n_pages, page_size;
    unsigned page_magic;                          // position / page_size = position * page_magic >> page_shift
    int page_shift;
    int cap;                                      // positions that a row of the block table has
    const bf16_t* q;
    int64_t q_stride;
    const int32_t *first, *context, *positions;
    const uint32_t* seen;
    int64_t seen_stride;
    int words, n_seqs, T, H, Hk, group, window, sinks;
    float scale;
    bf16_t* out;
    int64_t out_stride;
    float* lse;
    int whole;                                    // one block for each item: 0 no, 1 yes, 2 if no item is much longer than a share
    int first_block;                              // of the items' blocks, the first of this launch
    int shares;                                   // of the line of steps, otherwise
    int4* cuts;                                   // per share: the item that it begins and does not end (sequence, tile, key head, shares)
    float* parts;                                 // per share two parts
};

// A sequence's tokens, cut to what the call has.
struct Seq {
    int t0, n, context;
    __device__ __forceinline__ Seq(const ChunkArgs& p, int b)
    {
        t0 = min(max(p.first[b], 0), p.T);
        n = min(max(p.first[b + 1], t0), p.T) - t0;
        context = min(max(p.context[b], 0), kMostContext);
    }
    __device__ __forceinline__ int row_tiles(const ChunkArgs& p, int rows) const { return (n * p.group + rows - 1) / rows; }
};

// The positions of a sequence's tile of rows; `there`: whether the block table has a row for it.
__device__ __forceinline__ Span span_of(const ChunkArgs& p, const Seq& s, int tile, int rows, bool there)
{
    const int j0 = tile * rows / p.group, j1 = min(s.n - 1, (tile * rows + rows - 1) / p.group);
    return Span(s.context, s.n, j0, j1, p.seen != nullptr, p.window, p.sinks, there ? p.cap : 0);
}
template <int STEP>
__device__ __forceinline__ int steps_in(const Span& s) { return max(1, (s.n + STEP - 1) / STEP); }       // an item with nothing to see has its rows cleared

__device__ __forceinline__ int table_row(const ChunkArgs& p, int b) { return p.row_of ? p.row_of[b] : b; }

// Tiles of rows are numbered through: sequence b's have the places from floor(first[b] * group / ROWS) + b on, which is room enough for them; some places
// in between have none.
template <class S>
__device__ __forceinline__ int place_of(const ChunkArgs& p, int b) { return (int)((int64_t)min(max(p.first[b], 0), p.T) * p.group / S::ROWS) + b; }

// Steps of a tile; 0 where there is none.
template <class S>
__device__ __forceinline__ int steps_of(const ChunkArgs& p, int b, int tile)
{
    const Seq s(p, b);
    if (tile >= s.row_tiles(p, S::ROWS)) return 0;
    return steps_in<S::STEP>(span_of(p, s, tile, S::ROWS, (unsigned)table_row(p, b) < (unsigned)p.n_rows));
}

// Length of an item of the tile in the line that shares are cut from: its steps, behind kBetween that stand for what it costs besides.
template <class S>
__device__ __forceinline__ int units_of(const ChunkArgs& p, int b, int tile)
{
    const int n = steps_of<S>(p, b, tile);
    return n > 0 ? n + kBetween : 0;
}

// Where a block begins in the line, and how much of it it has.
struct Begin {
    int b, tile, hk, unit;                        // unit: of the item
    int64_t at, end, per;
};

__device__ __forceinline__ int64_t sum_before(int64_t v, int lane, int64_t& total)
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

// The share's first step: every thread adds up the steps of its part of the places.  LDS: [n_seqs] places, then 8 numbers of 64 bits behind kMostShared of
// them and 8 of 32.  Decides whether each item is to have a block, and leaves the rest to find_item() then.
template <class S>
__device__ __forceinline__ bool find_share(const ChunkArgs& p, char* smem, Begin& o, bool& whole)
{
    int* place = reinterpret_cast<int*>(smem);
    int64_t* lds = reinterpret_cast<int64_t*>(smem + kMostShared * sizeof(int));
    int* longest = reinterpret_cast<int*>(lds + 8);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int b = tid; b < p.n_seqs; b += S::THREADS) place[b] = place_of<S>(p, b);
    __syncthreads();
    const int slots = (int)((int64_t)p.T * p.group / S::ROWS) + p.n_seqs, each = (slots + S::THREADS - 1) / S::THREADS;
    const int u0 = min(slots, tid * each), u1 = min(slots, u0 + each);
    int b0 = 0;                                   // the last sequence whose place is not beyond u0
    for (int n = p.n_seqs; n > 1;) {
        const int half = n / 2;
        if (place[b0 + half] <= u0) {
            b0 += half;
            n -= half;
        } else n = half;
    }
    // f(place in the order, sequence, tile) for the thread's places
    auto mine = [&](auto&& f) {
        int b = b0;
        for (int u = u0; u < u1; ++u) {
            while (b + 1 < p.n_seqs && place[b + 1] <= u) ++b;
            if (u >= place[b] && f(b, u - place[b])) return;
        }
    };
    int64_t sum = 0;
    int most = 0;
    mine([&](int b, int tile) {
        const int n = units_of<S>(p, b, tile);
        sum += (int64_t)n * p.Hk;
        most = max(most, n);
        return false;
    });
#pragma unroll
    for (int i = 32; i; i >>= 1) most = max(most, __shfl_xor(most, i));
    int64_t total;
    int64_t before = sum_before(sum, lane, total);
    if (lane == 0) {
        lds[wave] = total;
        longest[wave] = most;
    }
    __syncthreads();
    int64_t all = 0;
#pragma unroll
    for (int w = 0; w < S::WAVES; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
        most = max(most, longest[w]);
    }
    __syncthreads();
    o.per = (all + p.shares - 1) / p.shares;
    whole = __builtin_amdgcn_readfirstlane(p.whole == 2 && most <= o.per + kUneven ? 1 : 0) != 0;
    if (whole) return true;
    if ((int)blockIdx.x >= p.shares) return false;
    o.at = min(all, o.per * (int64_t)blockIdx.x);
    o.end = min(all, o.at + o.per);
    if (o.at >= o.end) return false;
    // the one thread whose tiles hold the first step looks for it
    if (before <= o.at && o.at < before + sum)
        mine([&](int b, int tile) {
            const int n = units_of<S>(p, b, tile);
            if (o.at >= before + (int64_t)n * p.Hk) {
                before += (int64_t)n * p.Hk;
                return false;
            }
            int hk = 0;
            for (; o.at >= before + n; ++hk) before += n;
            lds[0] = b;
            lds[1] = tile;
            lds[2] = hk;
            lds[3] = o.at - before;
            return true;
        });
    __syncthreads();
    o.b = __builtin_amdgcn_readfirstlane((int)lds[0]);
    o.tile = __builtin_amdgcn_readfirstlane((int)lds[1]);
    o.hk = __builtin_amdgcn_readfirstlane((int)lds[2]);
    o.unit = __builtin_amdgcn_readfirstlane((int)lds[3]);
    __syncthreads();
    return true;
}

// One block for each place and key head.  Late tiles of a chunk, which see the most, come first.
template <class S>
__device__ __forceinline__ bool find_item(const ChunkArgs& p, Begin& o)
{
    const int lane = threadIdx.x & 63, slots = (int)((int64_t)p.T * p.group / S::ROWS) + p.n_seqs, block = p.first_block + (int)blockIdx.x,
              u = slots - 1 - block / p.Hk;
    if (u < 0) return false;
    // the last sequence whose place is not beyond u, 64 of a stride at a time
    int lo = 0, n = p.n_seqs;
    while (n > 1) {
        const int stride = (n + 63) / 64, b = lo + lane * stride;
        const bool is = lane * stride < n && place_of<S>(p, b) <= u;
        const uint64_t m = __ballot(is);
        const int k = m ? 63 - __builtin_clzll(m) : 0;
        lo = __builtin_amdgcn_readfirstlane(lo + k * stride);
        n = __builtin_amdgcn_readfirstlane(min(stride, n - k * stride));
    }
    o.b = lo;
    const Seq s(p, lo);
    o.tile = u - place_of<S>(p, lo);
    o.hk = block % p.Hk;
    o.unit = 0;
    return o.tile >= 0 && o.tile < s.row_tiles(p, S::ROWS);
}

template <bool E4M3>
using pv8 = std::conditional_t<E4M3, f16x8, bf16x8>;

template <bool HIGH>
__device__ __forceinline__ unsigned to_bf16(unsigned w) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH)); }
template <bool HIGH>
__device__ __forceinline__ unsigned to_f16(unsigned w) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH)); }

// Where a panel's 16-byte pieces of a row are: exchanged so that 16 rows' same piece (K's operand) and 4 rows' four neighbours (V's) lie in different banks.
__device__ __forceinline__ int turn64(int row) { return (row & 2) << 1 | (row & 4) >> 1 | (row & 8) >> 3; }
__device__ __forceinline__ int turn32(int row) { return row >> 2 & 3; }

// Byte of (row, 16-byte piece of the row's columns) in a step's K or V.
template <class S>
__device__ __forceinline__ int piece_at(int row, int piece)
{
    if (S::N32 == 0 || piece < 8 * S::N64) return (piece >> 3) * S::STEP * 128 + row * 128 + (((piece & 7) ^ turn64(row)) << 4);
    return S::N64 * S::STEP * 128 + row * 64 + (((piece & 3) ^ turn32(row)) << 4);
}

template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T* at_lds(unsigned byte) { return (__attribute__((address_space(3))) T*)(uintptr_t)byte; }

// body(integral_constant 0), ... , body(integral_constant N - 1)
template <int N, int I = 0, typename F>
__device__ __forceinline__ void unrolled(F&& body)
{
    if constexpr (I < N) {
        body(std::integral_constant<int, I>{});
        unrolled<N, I + 1>(body);
    }
}

// The n lowest bits (none for n <= 0, all from 32 on).
__device__ __forceinline__ unsigned below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1; }

template <class S>
__global__ void __launch_bounds__(S::THREADS, S::RESIDENT * S::WAVES >= 8 ? 2 : 1) chunk_kernel(ChunkArgs p)
{
    constexpr int D = S::D, WM = S::WM, WK = S::WK, PB = S::PB, STEP = S::STEP, POS = STEP / 64;
    constexpr bool E4M3 = S::E4M3;
    using Half = pv8<E4M3>;
    struct Weights {                                      // a block's probabilities; what their rounding leaves, where that is kept
        Half of[2], rest[S::TWO ? 2 : 1];
    };
    // e4m3: probabilities as fp16, 2^kUp of them, so that small ones are not lost below fp16's range (2^(kUp + kSlack) is within it)
    constexpr float kUp = E4M3 ? 11.0f : 0.0f;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, g = lane >> 5, wm = wave % WM, wk = wave / WM;
    char *const kbuf = smem, *const vbuf = smem + 2 * S::TILE;

    Begin at;
    bool whole = p.whole == 1;
    if (!whole) {
        if (tid == 0 && (int)blockIdx.x < p.shares) p.cuts[blockIdx.x] = make_int4(0, 0, 0, 0);
        if (!find_share<S>(p, smem, at, whole)) return;
    }
    if (whole && !find_item<S>(p, at)) return;

    for (;;) {
        // ---------------- an item, or what the share has of it
        const Seq seq(p, at.b);
        const int row = table_row(p, at.b);
        const Span span = span_of(p, seq, at.tile, S::ROWS, (unsigned)row < (unsigned)p.n_rows);
        const int32_t* pages = p.pages + (span.n > 0 ? (int64_t)row * p.row_stride : 0);          // where there is nothing to see, any row will do
        const int steps = steps_in<STEP>(span), begin = whole ? 0 : max(at.unit - kBetween, 0);
        const int ends_at = whole ? steps + kBetween : (int)min((int64_t)steps + kBetween, at.unit + (at.end - at.at)), end = max(ends_at - kBetween, 0);
        // on by so much of the line; false at the share's end
        auto advance = [&](int units) {
            at.at += units;
            if (at.at >= at.end) return false;
            at.unit = 0;
            if (++at.hk < p.Hk) return true;
            at.hk = 0;
            ++at.tile;
            while (at.tile >= Seq(p, at.b).row_tiles(p, S::ROWS)) {
                at.tile = 0;
                if (++at.b >= p.n_seqs) return false;             // only where `first` decreases
            }
            return true;
        };
        if (begin >= end) {                               // no step of it
            if (!advance(ends_at - at.unit)) return;
            continue;
        }
        const int n_rows = seq.n * p.group;
        const char *kbase = p.kc + (int64_t)at.hk * p.head_stride, *vbase = p.vc + (int64_t)at.hk * p.head_stride;
        float to_log2 = p.scale * 1.4426950408889634f * (E4M3 ? p.k_scale[at.hk] : 1.0f);
        const unsigned flip = to_log2 < 0.0f ? 0x80008000u : 0u;              // the sign goes to q, so that the largest product is the largest score
        to_log2 = to_log2 != to_log2 ? to_log2 : fmaxf(fabsf(to_log2), 1.17549435e-38f);       // above 0: 0 times a masked -infinity would be NaN

        // rows of this lane: which they are, and what they see: the positions from `from` to `last` and the sinks
        struct Row {
            bool real;
            int token, head, nth;                         // nth: the token's number in the sequence
        };
        auto row_of = [&]() {
            const int i = at.tile * S::ROWS + wm * 32 + c, j = min(i, n_rows - 1) / p.group;
            return Row{i < n_rows, seq.t0 + j, at.hk * p.group + (i < n_rows ? i - j * p.group : 0), j};
        };
        const bool idle = at.tile * S::ROWS + wm * 32 >= n_rows;         // a wave without rows only brings K and V
        int last = 0x7FFFFFFF, from = 0;                  // of a lane without a row: nobody looks at what it sees
        bf16x8 q[S::KS];
        {
            const Row o = row_of();
            if (o.real) {
                const int pos = p.positions ? max(seq.context, p.positions[o.token]) : seq.context + o.nth;
                last = p.seen ? seq.context - 1 : pos;
                from = p.window > 0 ? max(pos - p.window + 1, 0) : 0;
            }
            const bf16_t* src = p.q + (int64_t)o.token * p.q_stride + (int64_t)o.head * D;
#pragma unroll
            for (int k = 0; k < S::KS; ++k) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (o.real) v = *reinterpret_cast<const uint4*>(src + 16 * k + 8 * g);
                v.x ^= flip; v.y ^= flip; v.z ^= flip; v.w ^= flip;
                q[k] = __builtin_bit_cast(bf16x8, v);
                if constexpr (S::RESIDENT * S::WAVES < 8) asm volatile("" : "+a"(q[k]));     // operands may stay in accumulation registers
            }
        }

        // LDS offsets of a lane: its K row's first piece of a panel, its V row's; the others are these with a few bits turned
        const int rk = wk * PB * 32 + c, sub = 4 * g + ((lane & 15) >> 2), rv = wk * PB * 32 + sub, piece = 2 * (lane >> 4 & 1) + (lane >> 1 & 1), in = 8 * (lane & 1);
        const int kat = rk * 128 + ((g ^ turn64(c)) << 4), kat32 = S::N64 * STEP * 128 + rk * 64 + ((g ^ turn32(c)) << 4);
        const int vat = rv * 128 + ((piece ^ turn64(sub)) << 4) + in, vat32 = S::N64 * STEP * 128 + rv * 64 + ((piece ^ turn32(sub)) << 4) + in;

        f32x16 acc[S::VS];
        float m, l;

        // ---------------- where a step's positions are: lane i has those of positions i, 64 + i, ...  Places behind the last position are read from that one.
        struct Look {
            int page[POS];
            unsigned in_page[POS];
            uint64_t counts[POS];
        };
        struct Where {
            unsigned off[POS];                            // in 16-byte steps
            uint64_t there[POS];
        };
        const int most = (int)min((int64_t)span.n, (int64_t)end * STEP);      // positions behind these are another share's, or nobody's
        auto look = [&](int step) {
            Look o;
#pragma unroll
            for (int k = 0; k < POS; ++k) {
                const int v = step * STEP + 64 * k + lane;
                o.counts[k] = __ballot(v < most);
                const unsigned pos = span.read(v, most);
                const unsigned pg = (unsigned)((uint64_t)pos * p.page_magic >> p.page_shift);
                o.in_page[k] = pos - pg * (unsigned)p.page_size;
                o.page[k] = pages[pg];
            }
            return o;
        };
        auto resolve = [&](const Look& o) {
            Where w;
#pragma unroll
            for (int k = 0; k < POS; ++k) {
                const bool is = (unsigned)o.page[k] < (unsigned)p.n_pages;
                w.off[k] = is ? (unsigned)o.page[k] * p.page_step + o.in_page[k] * p.token_step : 0;
                w.there[k] = __ballot(is) & o.counts[k];
            }
            return w;
        };
        // ---------------- K or V of a step, to registers and from there to LDS
        constexpr int ACROSS = E4M3 ? D / 16 : D / 8;                         // 16-byte pieces of a row in the cache
        constexpr int PIECES = (STEP * ACROSS + S::THREADS - 1) / S::THREADS;
        constexpr bool SAME = S::THREADS % ACROSS == 0;                    // a thread's pieces are of the same columns, rows apart
        auto row_and_piece = [&](int i) {
            const int id = i * S::THREADS + tid;
            return SAME ? make_int2(i * (S::THREADS / ACROSS) + tid / ACROSS, tid % ACROSS) : make_int2(id / ACROSS, id % ACROSS);
        };
        struct Raw {
            uint4 w[PIECES];
        };
        auto spread = [&](const unsigned (&off)[POS], unsigned (&o)[PIECES]) {          // to the threads that read there
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int r = row_and_piece(i).x;
                o[i] = __builtin_amdgcn_ds_bpermute(4 * r, off[0]);                      // the lane is taken modulo 64
                if constexpr (POS > 1) {
                    const unsigned o1 = __builtin_amdgcn_ds_bpermute(4 * r, off[POS - 1]);
                    o[i] = r < 64 ? o[i] : o1;
                }
            }
        };
        auto read = [&](const char* base, const unsigned (&o)[PIECES], Raw& raw) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) raw.w[i] = *reinterpret_cast<const uint4*>(base + 16 * row_and_piece(i).y + (uint64_t)o[i] * 16);
        };
        auto fetch = [&](const char* base, const unsigned (&off)[POS], Raw& raw) {
            unsigned o[PIECES];
            spread(off, o);
            read(base, o, raw);
        };
        auto store = [&](char* tile, const Raw& raw, auto is_v) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int r = row_and_piece(i).x, piece = row_and_piece(i).y;
                if (STEP * ACROSS % S::THREADS != 0 && r >= STEP) continue;
                const uint4 w = raw.w[i];
                if constexpr (!E4M3) *reinterpret_cast<uint4*>(tile + piece_at<S>(r, piece)) = w;
                else if constexpr (decltype(is_v)::value) {
                    *reinterpret_cast<uint4*>(tile + piece_at<S>(r, 2 * piece)) = make_uint4(to_f16<false>(w.x), to_f16<true>(w.x), to_f16<false>(w.y), to_f16<true>(w.y));
                    *reinterpret_cast<uint4*>(tile + piece_at<S>(r, 2 * piece + 1)) = make_uint4(to_f16<false>(w.z), to_f16<true>(w.z), to_f16<false>(w.w), to_f16<true>(w.w));
                } else {
                    *reinterpret_cast<uint4*>(tile + piece_at<S>(r, 2 * piece)) = make_uint4(to_bf16<false>(w.x), to_bf16<true>(w.x), to_bf16<false>(w.y), to_bf16<true>(w.y));
                    *reinterpret_cast<uint4*>(tile + piece_at<S>(r, 2 * piece + 1)) = make_uint4(to_bf16<false>(w.z), to_bf16<true>(w.z), to_bf16<false>(w.w), to_bf16<true>(w.w));
                }
            }
        };
        constexpr std::false_type of_k{};
        constexpr std::true_type of_v{};
        // ---------------- what each row sees of it: a bit for each of the 32 positions
        auto cover = [&](int step, int b, const uint64_t (&there)[POS], f32x16& s) {
            const int in_step = (wk * PB + b) * 32, vb = step * STEP + in_step;
            const uint64_t word = POS > 1 && in_step >= 64 ? there[POS - 1] : there[0];
            const unsigned is = (unsigned)(word >> (in_step & 63));
            // the first k of them are among the sinks, at positions vb on; the others at positions at on
            const int k = min(max(span.sinks - vb, 0), 32), at = vb - span.sinks + span.lo;
            if (__all(is == 0xFFFFFFFFu && k == 0 && at + 31 <= last && at >= from)) return;
            const unsigned sink = below(k);
            unsigned on = below(last - at + 1) & (~below(from - at) | below(p.sinks - at));
            const int nth = at - seq.context;         // of the new tokens, the one at position `at`
            if (p.seen && nth > -32) {
                const uint32_t* w = p.seen + (int64_t)row_of().token * p.seen_stride;
                const int i = nth >> 5;
                const uint64_t lo = i >= 0 && i < p.words ? w[i] : 0, hi = i + 1 < p.words ? w[i + 1] : 0;
                on |= (unsigned)((lo | hi << 32) >> (nth & 31)) & ~below(-nth);
            }
            on = ((sink & below(last - vb + 1)) | (~sink & on)) & is;
            on >>= 4 * g;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(on >> (8 * (i / 4) + i % 4) & 1)) s[i] = -__builtin_inff();
        };
        // ---------------- probabilities in place of scores, in three steps: the maximum, what it changes, the exponentials.
        auto largest = [&](const f32x16& s, float& top, int i) { top = i ? fmaxf(top, s[i]) : s[0]; };
        // f: what earlier sums are to be multiplied by.  Returns whether any of them are; no branch, so that products go on around it.
        auto refer = [&](float& top, float& f, float& ref) {
            const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1])) * to_log2;
            const bool moves = __any(top > m + kSlack);
            const float m_new = moves ? fmaxf(m, top) : m;
            f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - m_new);
            l *= f;
            m = m_new;
            ref = (m_new == -__builtin_inff() ? 0.0f : m_new) - kUp;
            return moves;
        };
        auto exponent = [&](f32x16& s, float ref, int i) {
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], to_log2, -ref));
            l += s[i];
        };
        auto exponents = [&](f32x16& s, float& f) {
            float top, ref;
#pragma unroll
            for (int i = 0; i < 16; ++i) largest(s, top, i);
            const bool moves = refer(top, f, ref);
#pragma unroll
            for (int i = 0; i < 16; ++i) exponent(s, ref, i);
            return moves;
        };
        auto rescale = [&](float f) {
#pragma unroll
            for (int j = 0; j < S::VS; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[j][i] *= f;
        };
        // probabilities e and e + 1 of a block, as they go to the second product
        auto rounded = [&](const f32x16& s, Weights& pr, int e) {
            if constexpr (S::TWO) {
                const unsigned a = __float_as_uint(s[e]), b = __float_as_uint(s[e + 1]);
                reinterpret_cast<unsigned(&)[4]>(pr.of[e / 8])[e % 8 / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                pr.rest[e / 8][e % 8] = s[e] - __uint_as_float(a & 0xFFFF0000u);
                pr.rest[e / 8][e % 8 + 1] = s[e + 1] - __uint_as_float(b & 0xFFFF0000u);
            } else {
                pr.of[e / 8][e % 8] = s[e];
                pr.of[e / 8][e % 8 + 1] = s[e + 1];
            }
        };
        // ---------------- a block's products, in slots: KS of S = K Q^T, then 2 * VS of O^T += V^T P^T; their operand from K or V
        union Operand {
            bf16x8 k;
            s16x4 h[2];
            Half v;
        };
        struct Lds {
            unsigned k, k32, v, v32;                      // of a lane in this step's K and V
        };
        auto operand = [&](auto slot, const Lds& o, int b, Operand& a) {
            constexpr int k = decltype(slot)::value, t = (k - S::KS) / S::VS, j = (k - S::KS) % S::VS;
            if constexpr (k < 4 * S::N64) a.k = *at_lds<bf16x8>((o.k ^ (k & 3) << 5) + (k >> 2) * STEP * 128 + b * 32 * 128);
            else if constexpr (k < S::KS) a.k = *at_lds<bf16x8>((o.k32 ^ (k & 1) << 5) + b * 32 * 64);
            else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {             // row r + 8 h
                    const unsigned at = j < 2 * S::N64 ? (o.v ^ ((j & 1) << 6 | h << 4)) + (j >> 1) * STEP * 128 + (32 * b + 16 * t + 8 * h) * 128
                                                       : (o.v32 ^ h << 5) + (32 * b + 16 * t + 8 * h) * 64;
                    a.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at_lds<s16x4>(at));
                }
            }
        };
        auto lds_of = [&](const char* kt, const char* vt) {
            const unsigned k = (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)kt, v = (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)vt;
            return Lds{k + kat, k + kat32, v + vat, v + vat32};
        };
        auto product = [&](auto slot, const Operand& a, f32x16& s, const Weights& pr) {
            constexpr int k = decltype(slot)::value, t = (k - S::KS) / S::VS, j = (k - S::KS) % S::VS;
            if constexpr (k < S::KS) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.k, q[k], k == 0 ? f32x16{} : s, 0, 0, 0);
            else if constexpr (E4M3) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.v, pr.of[t], acc[j], 0, 0, 0);
            else {
                acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, pr.of[t], acc[j], 0, 0, 0);
                if constexpr (S::TWO) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, pr.rest[t], acc[j], 0, 0, 0);
            }
        };
        auto scores = [&](const Lds& o, int b, f32x16& s) {
            const Weights none = {};
            unrolled<S::KS>([&](auto k) {
                Operand a;
                operand(k, o, b, a);
                product(k, a, s, none);
            });
        };
        // loads from memory stay on their way across it
        auto lds_sync = [&]() {
            __builtin_amdgcn_s_waitcnt(0xC07F);           // lgkmcnt(0)
            lds_barrier();
        };
        auto clear = [&]() {
            m = -__builtin_inff();
            l = 0.0f;
#pragma unroll
            for (int j = 0; j < S::VS; ++j) acc[j] = f32x16{};
        };

        // ---------------- the pipeline: block n of a wave is weighed while n + 1 has its exponentials taken and n + 2 its scores.  In step j V of step j and K
        // of step j + LEAD are in LDS, the next ones in registers, those after them on their way to there.
        {
            constexpr int LEAD = S::LEAD;
            Raw kraw, vraw;
            unsigned spots[LEAD][PIECES];                 // where the thread reads, of steps j + 2 .. j + LEAD + 1
            uint64_t there[LEAD + 3][POS];              // of steps j ..
            Look asked;
            f32x16 s0, s1;
            Weights p0, p1;
            float f;
            {
                constexpr int N = LEAD + 2;
                Look first[N];
                Where w[N];
                Raw kr[LEAD + 1], vr;
#pragma unroll
                for (int i = 0; i < N; ++i) first[i] = look(begin + i);
                asked = look(begin + N);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    w[i] = resolve(first[i]);
#pragma unroll
                    for (int k = 0; k < POS; ++k) there[i][k] = w[i].there[k];
                    if (i <= LEAD) fetch(kbase, w[i].off, kr[i]);
                    if (i == 0) fetch(vbase, w[0].off, vr);
                }
                fetch(kbase, w[LEAD + 1].off, kraw);
                fetch(vbase, w[1].off, vraw);
#pragma unroll
                for (int i = 0; i < 2; ++i) store(kbuf + i * S::TILE, kr[i], of_k);
                store(vbuf, vr, of_v);
                lds_sync();
                clear();
                scores(lds_of(kbuf, vbuf), 0, s0);
                scores(lds_of(LEAD == 1 ? kbuf : kbuf + S::TILE, vbuf), LEAD == 1 ? 1 : 0, s1);
                if constexpr (LEAD == 2) {
                    lds_sync();
                    store(kbuf, kr[2], of_k);
                }
                cover(begin, 0, there[0], s0);
                exponents(s0, f);
#pragma unroll
                for (int e = 0; e < 16; e += 2) rounded(s0, p0, e);
#pragma unroll
                for (int i = 0; i < LEAD; ++i) spread(w[2 + i].off, spots[i]);
            }
            for (int step = begin; step < end; ++step) {
                const int odd = (step - begin) & 1;
                lds_sync();                               // V of this step and K of step + LEAD are there, and nobody reads the other buffers any more
                unsigned vo[PIECES];
#pragma unroll
                for (int i = 0; i < PIECES; ++i) vo[i] = spots[0][i];
#pragma unroll
                for (int n = 0; n + 1 < LEAD; ++n)
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) spots[n][i] = spots[n + 1][i];
                const Lds tiles = lds_of(kbuf + ((odd + LEAD) & 1) * S::TILE, vbuf + odd * S::TILE);
                // what a step has to do besides, one thing behind each of the first slots
                auto beside = [&](auto slot) {
                    constexpr int k = decltype(slot)::value;
                    if constexpr (k == 0) store(kbuf + ((odd + LEAD + 1) & 1) * S::TILE, kraw, of_k);
                    if constexpr (k == 1) store(vbuf + (odd ^ 1) * S::TILE, vraw, of_v);
                    if constexpr (k == 2) {
                        const Where w = resolve(asked);
#pragma unroll
                        for (int i = 0; i < POS; ++i) there[LEAD + 2][i] = w.there[i];
                        spread(w.off, spots[LEAD - 1]);
                    }
                    if constexpr (k == 3) read(vbase, vo, vraw);
                    if constexpr (k == 4) read(kbase, spots[LEAD - 1], kraw);
                    if constexpr (k == 5) asked = look(step + LEAD + 3);
                };
                auto part = [&](auto b_, f32x16& cur, f32x16& next, const Weights& pr, Weights& pn) {
                    constexpr int b = decltype(b_)::value, SLOTS = S::KS + 2 * S::VS, FIRST = SLOTS / 4, AHEAD = S::AHEAD;
                    Operand a[AHEAD + 1];
                    unrolled<AHEAD>([&](auto i) { operand(i, tiles, b, a[i]); });
                    cover(step + (b + 1) / PB, (b + 1) % PB, there[(b + 1) / PB], cur);
                    float top, ref;
                    bool moves = false;
                    unrolled<SLOTS>([&](auto i) {
                        constexpr int k = decltype(i)::value;
                        if constexpr (k + AHEAD < SLOTS) operand(std::integral_constant<int, k + AHEAD>{}, tiles, b, a[(k + AHEAD) % (AHEAD + 1)]);
                        product(i, a[k % (AHEAD + 1)], next, pr);
                        if constexpr (k < FIRST) {
#pragma unroll
                            for (int e = 16 * k / FIRST; e < 16 * (k + 1) / FIRST; ++e) largest(cur, top, e);
                            if constexpr (k == FIRST - 1) moves = refer(top, f, ref);
                        } else {
                            constexpr int N = SLOTS - FIRST, e0 = 16 * (k - FIRST) / N / 2 * 2, e1 = k == SLOTS - 1 ? 16 : 16 * (k - FIRST + 1) / N / 2 * 2;
#pragma unroll
                            for (int e = e0; e < e1; ++e) {
                                exponent(cur, ref, e);
                                if (e & 1) rounded(cur, pn, e - 1);
                            }
                        }
                        if constexpr (b == 0) beside(i);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                    asm volatile("" : "+v"(pn.of[0]), "+v"(pn.of[1]), "+v"(l), "+v"(next));  // here, and not where they are needed
                    if constexpr (S::TWO) asm volatile("" : "+v"(pn.rest[0]), "+v"(pn.rest[1]));
                    if (__builtin_expect(moves, 0)) {
                        asm volatile("");                 // seldom: a branch, not a product with one
                        rescale(f);
                    }
                };
                if (idle) {
                    unrolled<6>(beside);
                } else if constexpr (PB == 2) {
                    part(std::integral_constant<int, 0>{}, s1, s0, p0, p1);
                    part(std::integral_constant<int, 1>{}, s0, s1, p1, p0);
                } else {
                    part(std::integral_constant<int, 0>{}, s1, s0, p0, p1);
                    s1 = s0;
                    p0 = p1;
                }
#pragma unroll
                for (int i = 0; i < LEAD + 2; ++i)
#pragma unroll
                    for (int k = 0; k < POS; ++k) there[i][k] = there[i + 1][k];
            }
        }

        bool bad = false;
        if (row_of().real)
#pragma unroll
            for (int j = 0; j < S::VS; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) bad = bad || !(fabsf(acc[j][i]) < __builtin_inff());
        int* flags = reinterpret_cast<int*>(smem + S::FLAGS);
        bad = __any(bad);
        if (lane == 0) flags[wave] = bad ? 1 : 0;
        lds_sync();                                       // all have read their last step
        bad = false;
#pragma unroll
        for (int w = 0; w < S::WAVES; ++w) bad = bad || flags[w] != 0;
        if (bad) {                                        // once more, with care and no haste
            float* scratch = reinterpret_cast<float*>(smem + S::TILE) + wave * 32 * 32;      // one step of K before it, of V behind
            char* vt = smem + S::TILE + S::SCRATCH;
            clear();
            for (int step = begin; step < end; ++step) {
                const Where w = resolve(look(step));
                Raw raw;
                fetch(kbase, w.off, raw);
                store(kbuf, raw, of_k);
                fetch(vbase, w.off, raw);
                store(vt, raw, of_v);
                __syncthreads();
                for (int b = 0; b < PB; ++b) {
                    f32x16 s;
                    float f;
                    scores(lds_of(kbuf, vt), b, s);
                    cover(step, b, w.there, s);
                    if (exponents(s, f)) rescale(f);
                    wave_lds_order();
#pragma unroll
                    for (int i = 0; i < 16; ++i) scratch[(8 * (i / 4) + 4 * g + i % 4) * 32 + c] = s[i];
                    wave_lds_order();
                    for (int e = 0; e < 32; ++e) {
                        const float weight = scratch[e * 32 + c];
                        if (weight == 0.0f) continue;
#pragma unroll
                        for (int j = 0; j < S::VS; ++j)
#pragma unroll
                            for (int i4 = 0; i4 < 4; ++i4) {
                                const uint2 raw2 = *reinterpret_cast<const uint2*>(vt + piece_at<S>((wk * PB + b) * 32 + e, 4 * j + i4) + 8 * g);
                                const unsigned u[2] = {raw2.x, raw2.y};
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const unsigned short h = (unsigned short)(u[i / 2] >> 16 * (i & 1));
                                    float val;
                                    if constexpr (E4M3) val = (float)__builtin_bit_cast(_Float16, h);
                                    else val = __uint_as_float((unsigned)h << 16);
                                    acc[j][4 * i4 + i] = __builtin_fmaf(weight, val, acc[j][4 * i4 + i]);
                                }
                            }
                    }
                }
                __syncthreads();
            }
        }

        // ---------------- the end of the item, or of the share's part of it
        l += __shfl_xor(l, 32);
        if constexpr (WK > 1) {
            float* joined = reinterpret_cast<float*>(smem);   // [WK - 1][WM][32][D + 4]: O, then m, l
            auto slot = [&](int k) { return joined + (((k - 1) * WM + wm) * 32 + c) * (D + 4); };
            if (wk > 0) {
                float* dst = slot(wk);
#pragma unroll
                for (int j = 0; j < S::VS; ++j)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4)
                        *reinterpret_cast<float4*>(dst + 32 * j + 8 * i4 + 4 * g) =
                            make_float4(acc[j][4 * i4], acc[j][4 * i4 + 1], acc[j][4 * i4 + 2], acc[j][4 * i4 + 3]);
                if (g == 0) {
                    dst[D] = m;
                    dst[D + 1] = l;
                }
            }
            lds_sync();
            if (wk == 0) {
                float top = m;
                for (int k = 1; k < WK; ++k) top = fmaxf(top, slot(k)[D]);
                const float ref = top == -__builtin_inff() ? 0.0f : top;
                float f = __builtin_amdgcn_exp2f(m - ref);
                l *= f;
#pragma unroll
                for (int j = 0; j < S::VS; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[j][i] *= f;
                for (int k = 1; k < WK; ++k) {
                    const float* src = slot(k);
                    f = __builtin_amdgcn_exp2f(src[D] - ref);
                    l += f * src[D + 1];
#pragma unroll
                    for (int j = 0; j < S::VS; ++j)
#pragma unroll
                        for (int i4 = 0; i4 < 4; ++i4) {
                            const float4 v = *reinterpret_cast<const float4*>(src + 32 * j + 8 * i4 + 4 * g);
                            acc[j][4 * i4] += f * v.x;
                            acc[j][4 * i4 + 1] += f * v.y;
                            acc[j][4 * i4 + 2] += f * v.z;
                            acc[j][4 * i4 + 3] += f * v.w;
                        }
                }
                m = top;
            }
            lds_sync();                                       // LDS is free for the next item
        }
        const bool begins = begin == 0, ends = end == steps;
        if (!whole && begins && !ends && tid == 0)
            p.cuts[blockIdx.x] = make_int4(at.b, at.tile, at.hk, (int)((at.at - at.unit + steps + kBetween - 1) / at.per - blockIdx.x) + 1);
        const Row o = row_of();
        if (wk == 0 && o.real) {
            if (begins && ends) {
                const float k = l > 0.0f || l != l ? (E4M3 ? p.v_scale[at.hk] : 1.0f) / l : 0.0f;
                bf16_t* dst = p.out + (int64_t)o.token * p.out_stride + (int64_t)o.head * D;
#pragma unroll
                for (int j = 0; j < S::VS; ++j)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4)
                        *reinterpret_cast<uint2*>(dst + 32 * j + 8 * i4 + 4 * g) =
                            make_uint2(pack_bf16(acc[j][4 * i4] * k, acc[j][4 * i4 + 1] * k), pack_bf16(acc[j][4 * i4 + 2] * k, acc[j][4 * i4 + 3] * k));
                if (p.lse && g == 0) p.lse[(int64_t)o.token * p.H + o.head] = (m - kUp + __log2f(l)) * 0.6931471805599453f;
            } else {
                float* part = p.parts + (2 * (int64_t)blockIdx.x + (begins ? 1 : 0)) * S::PART;
                const int i = wm * 32 + c;
#pragma unroll
                for (int j = 0; j < S::VS; ++j)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4)
                        *reinterpret_cast<float4*>(part + (int64_t)i * D + 32 * j + 8 * i4 + 4 * g) =
                            make_float4(acc[j][4 * i4], acc[j][4 * i4 + 1], acc[j][4 * i4 + 2], acc[j][4 * i4 + 3]);
                if (g == 0) {
                    part[S::ROWS * D + i] = m;
                    part[S::ROWS * D + S::ROWS + i] = l;
                }
            }
        }
        if (whole) return;
        if (!advance(ends_at - at.unit)) return;
    }
}

// Joins the parts of the item that share x begins and does not end, a wave for each of its rows.
template <int D>
__global__ void __launch_bounds__(256) chunk_join(ChunkArgs p, int rows, float up)
{
    constexpr int LANES = D / 4, SETS = 64 / LANES;       // lanes of a row of O, four columns each; sets of lanes that take turns at the parts
    const int4 cut = p.cuts[blockIdx.x];
    const int n = min(cut.w, (int)(gridDim.x - blockIdx.x)), lane = threadIdx.x & 63, i = blockIdx.y * 4 + (threadIdx.x >> 6);
    if (n == 0 || i >= rows) return;
    const Seq seq(p, cut.x);
    const int at = cut.y * rows + i;
    if (at >= seq.n * p.group) return;
    const int64_t size = (int64_t)rows * (D + 2);
    auto part = [&](int k) { return p.parts + (2 * ((int64_t)blockIdx.x + k) + (k == 0 ? 1 : 0)) * size; };
    float top = -__builtin_inff();
    for (int k = lane; k < n; k += 64) top = fmaxf(top, part(k)[rows * D + i]);
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float ref = top == -__builtin_inff() ? 0.0f : top;
    const int set = lane / LANES, col = 4 * (lane - set * LANES);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.0f;
    if (set < SETS) {
#pragma unroll 8
        for (int k = set; k < n; k += SETS) {
            const float* src = part(k);
            const float f = __builtin_amdgcn_exp2f(src[rows * D + i] - ref);
            const float4 v = *reinterpret_cast<const float4*>(src + (int64_t)i * D + col);
            o.x += f * v.x; o.y += f * v.y; o.z += f * v.z; o.w += f * v.w;
            sum += f * src[rows * D + rows + i];
        }
    }
#pragma unroll
    for (int s = 1; s < SETS; ++s) {                      // in this order in every lane of the first set
        const int from = (lane + s * LANES) & 63;
        const float4 v = make_float4(__shfl(o.x, from), __shfl(o.y, from), __shfl(o.z, from), __shfl(o.w, from));
        const float l = __shfl(sum, from);
        if (set == 0) {
            o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
            sum += l;
        }
    }
    const int j = at / p.group, head = cut.z * p.group + at - j * p.group, t = seq.t0 + j;
    const float k = sum > 0.0f || sum != sum ? (p.v_scale ? p.v_scale[cut.z] : 1.0f) / sum : 0.0f;
    if (set == 0)
        *reinterpret_cast<uint2*>(p.out + (int64_t)t * p.out_stride + (int64_t)head * D + col) = make_uint2(pack_bf16(o.x * k, o.y * k), pack_bf16(o.z * k, o.w * k));
    if (p.lse && lane == 0) p.lse[(int64_t)t * p.H + head] = (top - up + __log2f(sum)) * 0.6931471805599453f;
}

// body(Shape): the shape that a call takes, by the rows that a sequence has on average.  Both sides measured, in us, 32 query heads over 8 of 128
// columns if nothing else is said (prompts in shares of steps):
//   up to 32 rows    two waves with a half of the positions each, two blocks a CU, so that one reads while the other begins or ends an item: 64
//                    sequences of 8 tokens, up to 4096 positions in e4m3: 120; four waves 138; the shape for 128 rows 149 (bf16, of 4 tokens over 4 heads: 62, 67, 66).  Heads of 64 columns,
//                    whose steps are small, with four waves: 32 sequences of 8 tokens 50, two waves 53 (16 of 16 tokens, bf16: 55 and 60)
//   up to 64, e4m3   two waves of 32 rows in the same manner: 64 sequences of 8 tokens, 64 over 8 heads, up to 2048 positions: 81; the next shape 93
//   up to 64, bf16   where twice as much is on its way, the next shape: 16 tokens behind 32768 positions 47; two waves 50; four 56
//   up to 128        eight waves, of which two share the positions of 32 rows: 32 sequences of 33 tokens, up to 4096 positions: 127; the last shape 150 (16 of 24 tokens: 68 and 71; one of
//                    26 tokens behind 2048: 26 and 24)
//   more             eight waves with all positions: 4096 tokens, 32 over 8 heads of 64: 145; the shape for 128 rows 185
// Heads of 192 and 256 columns leave registers for four waves, with all positions: 4096 tokens, 16 over 4 heads of 256: 264; where two share the
// positions 477.  They do share them for few rows: 32 sequences of 4 tokens, 32 over 4 heads of 192 81 and 91, 16 of 4 tokens, heads of 256 74 and 79.
// Up to 128 rows a bf16 cache has two bf16 for a probability.  These calls wait for memory more than for products: a tree of 26 tokens 25.5 us with one and 26.2 with two, 64
// sequences of 4 tokens 61.1 and 61.9, 32 of 33 120.5 and 127.3, 16 of 24 63.5 and 68.2; heads of 192 columns 88.7 and 94.1, of 256, which leave too few registers, 79.5
// and 89.0.  Longer ones are bound by the products and by the making of their operands: a prompt of 2048 tokens 77.2 and 93.3, 16384 tokens 2065 and 2655.
template <int D, bool E4M3, typename F>
auto pick(double rows, F&& body)
{
    auto few = [&](auto shape) {
        using S = decltype(shape);
        if constexpr (E4M3) return body(S{});
        else return body(Fine<S>{});
    };
    if constexpr (D <= 128) {
        if (rows <= 32) return few(Shape<D, E4M3, 1, D == 64 ? 4 : 2, 1>{});
        if (E4M3 && rows <= 64) return few(Shape<D, E4M3, 2, 1, 2>{});
        if (rows <= 128) return few(Shape<D, E4M3, 4, 2, 1>{});
        return body(Shape<D, E4M3, 8, 1, 2>{});
    } else {
        if (rows <= 32) return few(Shape<D, E4M3, 2, 2, 1>{});
        if (rows <= 128) return few(Shape<D, E4M3, 4, 1, 2>{});
        return body(Shape<D, E4M3, 4, 1, 2>{});
    }
}

template <typename F>
auto pick(int D, bool e4m3, double rows, F&& body)
{
    auto of = [&](auto d) {
        return e4m3 ? pick<decltype(d)::value, true>(rows, body) : pick<decltype(d)::value, false>(rows, body);
    };
    switch (D) {
        case 64: return of(std::integral_constant<int, 64>{});
        case 96: return of(std::integral_constant<int, 96>{});
        case 128: return of(std::integral_constant<int, 128>{});
        case 192: return of(std::integral_constant<int, 192>{});
        default: return of(std::integral_constant<int, 256>{});
    }
}

// Shares of the line of steps at most: as many blocks as there is room for.
template <class S>
constexpr int64_t most_shares()
{
    static_assert(256 * S::RESIDENT <= kChunkShares, "cuts");
    return 256 * S::RESIDENT;
}

template <int D, bool E4M3>
hipError_t init_of()
{
    hipError_t e = hipSuccess;
    for (double rows : {32.0, 64.0, 128.0, 256.0}) {
        e = pick<D, E4M3>(rows, [](auto s) {
            using S = decltype(s);
            return hipFuncSetAttribute(reinterpret_cast<const void*>(&chunk_kernel<S>), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
        });
        if (e != hipSuccess) return e;
    }
    return e;
}

}  // namespace

hipError_t init_chunk_kernels()
{
    hipError_t e;
    if ((e = init_of<64, false>()) != hipSuccess || (e = init_of<64, true>()) != hipSuccess || (e = init_of<96, false>()) != hipSuccess ||
        (e = init_of<96, true>()) != hipSuccess || (e = init_of<128, false>()) != hipSuccess || (e = init_of<128, true>()) != hipSuccess ||
        (e = init_of<192, false>()) != hipSuccess || (e = init_of<192, true>()) != hipSuccess || (e = init_of<256, false>()) != hipSuccess)
        return e;
    return init_of<256, true>();
}

// For every split of up to T tokens over any number of sequences: the parts of the largest shape that it may take, which is one for at most as many rows as there are.
size_t chunk_workspace_bytes(const moe_kv_cache& c, int T, int n_heads)
{
    const double most = (double)T * (n_heads / c.n_kv_heads);
    int64_t floats = 0;
    for (double rows : {32.0, 64.0, 128.0, most})
        floats = std::max(floats, pick(c.head_dim, c.type == MOE_KV_E4M3, std::min(rows, most), [](auto s) { return 2 * most_shares<decltype(s)>() * decltype(s)::PART; }));
    return align_up(kChunkShares * sizeof(int4), 256) + align_up(floats * sizeof(float), 256);
}

hipError_t launch_chunk(const moe_kv_cache& c, const moe_block_table& t, const moe_chunk& ch, const bf16_t* q, int64_t q_stride, int n_heads, float scale,
                        bf16_t* out, int64_t out_stride, float* lse, void* ws, hipStream_t s)
{
    const bool e4m3 = c.type == MOE_KV_E4M3;
    const int size = e4m3 ? 1 : 2, per16 = 16 / size;
    ChunkArgs p;
    p.kc = static_cast<const char*>(c.k); p.vc = static_cast<const char*>(c.v);
    p.head_stride = c.head_stride * size;
    p.page_step = (unsigned)(c.page_stride / per16);
    p.token_step = (unsigned)(c.token_stride / per16);
    p.k_scale = e4m3 ? c.k_scale : nullptr; p.v_scale = e4m3 ? c.v_scale : nullptr;
    p.pages = t.pages; p.row_of = t.token_row; p.row_stride = t.row_stride; p.n_rows = t.n_rows;
    p.n_pages = c.n_pages; p.page_size = c.page_size;
    // as in attention.hip: exact for every position below 2^31
    int sh = 0;
    while (((int64_t)1 << sh) < c.page_size) ++sh;
    p.page_magic = (unsigned)((((uint64_t)1 << (31 + sh)) + c.page_size - 1) / c.page_size);
    p.page_shift = 31 + sh;
    p.cap = (int)std::min<int64_t>((int64_t)t.max_pages * c.page_size, 0x7FFFFFFF);
    p.q = q; p.q_stride = q_stride;
    p.first = ch.first; p.context = ch.context; p.positions = ch.seen ? ch.positions : nullptr;
    p.seen = ch.seen; p.seen_stride = ch.seen_stride; p.words = ch.seen_words;
    p.n_seqs = ch.n_seqs; p.T = ch.T; p.H = n_heads; p.Hk = c.n_kv_heads; p.group = n_heads / c.n_kv_heads;
    p.window = ch.window; p.sinks = ch.window > 0 ? ch.sinks : 0;
    p.scale = scale;
    p.out = out; p.out_stride = out_stride; p.lse = lse;
    p.cuts = static_cast<int4*>(ws);
    p.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up(kChunkShares * sizeof(int4), 256));

    const double rows = (double)ch.T * p.group / ch.n_seqs;       // of a sequence, on average
    return pick(c.head_dim, e4m3, rows, [&](auto shape) {
        using S = decltype(shape);
        const int64_t slots = (int64_t)ch.T * p.group / S::ROWS + ch.n_seqs, items = slots * p.Hk;
        // The tiles of a drafted tree see all of their sequence and go by shares: 256 trees of 8 tokens, up to 2048 positions, 230 us, with a block for each item
        // 248.  So do chunks of one tile each (256 x 8 tokens behind up to 4096: 400 us and 694).  Where a chunk has two tiles and more, its blocks read the
        // same positions at about the same time and write no parts: a prompt of 4096 tokens 164 us, in shares 197; four of 512, a window of 1024, 58 and
        // 67; sixteen of 128 95 and 109; 16384 tokens 2060 and 2194.  One sequence that is far longer than the others would keep few blocks busy, and only
        // the device knows the lengths: its blocks add them up (3 us) and take shares then.
        p.whole = ch.n_seqs > kMostShared ? 1 : !p.seen && rows >= 2 * S::ROWS && items - (int64_t)ch.n_seqs * p.Hk >= most_shares<S>() ? 2 : 0;
        p.first_block = 0;
        if (p.whole == 1) {
            constexpr int64_t kBlocks = ((int64_t)1 << 31) / S::THREADS;      // a launch takes less than 2^32 threads
            for (int64_t at = 0; at < items; at += kBlocks) {
                p.first_block = (int)at;
                hipLaunchKernelGGL((chunk_kernel<S>), dim3((unsigned)std::min(kBlocks, items - at)), dim3(S::THREADS), S::LDS, s, p);
                hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
            return hipSuccess;
        }
        const int64_t most = items * (((int64_t)p.cap + S::STEP - 1) / S::STEP);
        p.shares = (int)std::max<int64_t>(1, std::min<int64_t>(most, most_shares<S>()));
        hipLaunchKernelGGL((chunk_kernel<S>), dim3((unsigned)(p.whole ? std::max<int64_t>(items, p.shares) : p.shares)), dim3(S::THREADS), S::LDS, s, p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.shares == 1) return e;
        hipLaunchKernelGGL((chunk_join<S::D>), dim3(p.shares, S::ROWS / 4), dim3(256), 0, s, p, S::ROWS, S::E4M3 ? 11.0f : 0.0f);
        return hipGetLastError();
    });
}

}  // namespace bmoe
