// Linear layer in 8-bit floating point:
//
//   out[m][n] = bf16( sum_b x_scale[b][m] w_scale[n / 128][b] sum_{k in block b of 128} x8[m][k] w8[n][k] )
//
// One 16x16x128 MFMA is exactly one block of k deep, so its result is multiplied by the block's scales and added to the fp32
// accumulator: four multiply-adds per MFMA beside it, none of the precision of a scale lost.  The product is issued transposed
// (weights x rows): a lane then holds one row m of a tile, so the row's scale is one register, and four columns n in a row.
// Within a block the order of k is free as long as both operands keep to it: a lane's 32 bytes are the 16-byte chunks g and 4 + g of its
// row (g = lane / 16), so that 16 lanes read whole 64-byte pieces.
#include "layer.h"

#include <algorithm>
#include <type_traits>

namespace bmoe {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct LinearArgs {
    const uint8_t *x, *w;
    const float *xs, *ws;
    bf16_t* out;
    float* part;                                          // [ksplit][M][part_stride] where K is cut
    int64_t x_stride, xs_stride, out_stride;
    int M, N, K, nk;                                      // nk: blocks of K
    int tiles_m, tiles_n, group_m, ksplit;
    int part_stride;                                      // N in whole quads
    int vec, vec16;                                       // out rows take 8-byte, 16-byte stores
    int wide;                                             // operands widened to bf16
};

__device__ __forceinline__ f32x4 mfma_block(i32x8 w, i32x8 x)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);   // scales of 1
}
__device__ __forceinline__ i32x8 operand(uint4 a, uint4 b)
{
    return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// Columns n .. n + 3 of row m.
__device__ __forceinline__ void store4(const LinearArgs& p, int m, int n, const float* v)
{
    if (m >= p.M) return;
    bf16_t* dst = p.out + (int64_t)m * p.out_stride + n;
    if (p.vec && n + 4 <= p.N) {
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < p.N) dst[e] = (bf16_t)v[e];
}

// ------------------------------------------------------------------------------------------------
// Few rows (at most 64): a block takes 16 NT columns and 16 MT rows, its eight waves take the blocks of K by turns and are
// summed through LDS in wave order.  Operands come straight from memory into registers, DEPTH blocks of K ahead.  Bound by the weights'
// stream, and for few columns by the latency of a wave's few trips to memory: one row by 6144 x 4096 7.2 us (25 MB, 3.5 TB/s), 16 rows by
// 14336 x 4096 17 us (59 MB, 3.5 TB/s).
// WIDE (K up to kShortK or by the caller's wish, here and in the ring kernel below): operands are widened to bf16 (exact) for four 16x16x32 bf16 MFMAs
// per block of K, which add up in fp32.  The 8-bit MFMA adds up 8 neighbouring k at a time, each product cut off toward zero at 2^-13 of 2^e, e the
// largest sum of two exponents among the 8 (this model gives its results to the last bit): for values of like size up to 1e-5 of sum |x||w| over a block of
// 128 and 3.4e-5 over its last 16.  Beyond kShortK such values lose less than fp32 sums of K products may be off by (K 2^-24 of the same sum); at K =
// 288 one result in 16 million did not.  Where one column is hundreds of times larger than its neighbours they lose more at any K: hence the
// caller's choice.  Widening costs 16384 x 4096 x 512 67 -> 93 us, 1000 x 2048 x 512 6.1 -> 6.7; by wish 1 x 6144 x 4096 7.6 -> 7.9, 64 x 6144 x 4096 13.7 ->
// 16.0, 256 x 6144 x 4096 18.7 -> 26.0, 16384 x 7168 x 7168 661 -> 1476.
// ------------------------------------------------------------------------------------------------
constexpr int kRowWaves = 8;
constexpr int kShortK = 512;

__device__ __forceinline__ bf16x8 widen8(int a, int b)
{
    auto two = [](int w, auto high) {
        return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w, 1.0f, decltype(high)::value));
    };
    return __builtin_bit_cast(bf16x8, make_uint4(two(a, std::false_type{}), two(a, std::true_type{}), two(b, std::false_type{}), two(b, std::true_type{})));
}

template <bool WIDE>
__device__ __forceinline__ f32x4 block_product(const i32x8 w, const i32x8 x)
{
    if constexpr (!WIDE) return mfma_block(w, x);
    f32x4 t = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q)
        t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2 * q], w[2 * q + 1]), widen8(x[2 * q], x[2 * q + 1]), t, 0, 0, 0);
    return t;
}

template <int MT, int NT, int DEPTH, bool WIDE>
__global__ void __launch_bounds__(kRowWaves * 64) linear_rows_kernel(LinearArgs p)
{
    __shared__ f32x4 sums[kRowWaves][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * MT;
    const uint8_t *wrow[NT], *xrow[MT];
    const float* srow[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) wrow[j] = p.w + (int64_t)min(n0 + 16 * j + c, p.N - 1) * p.K;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = min(m0 + 16 * i + c, p.M - 1);
        xrow[i] = p.x + (int64_t)m * p.x_stride;
        srow[i] = p.xs + m;
    }
    const float* wscale = p.ws + (int64_t)(n0 / kScaleGroup) * p.nk;          // 16 NT columns are in one block of 128
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint4 w[DEPTH][NT][2], x[DEPTH][MT][2];
    float s[DEPTH][MT], sw[DEPTH];
    // chunks past K are the row's last one again, cleared below
    auto load = [&](int d, int b) {
        const int k0 = min(b * 128 + 16 * g, p.K - 16), k1 = min(b * 128 + 64 + 16 * g, p.K - 16);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            w[d][j][0] = *reinterpret_cast<const uint4*>(wrow[j] + k0);
            w[d][j][1] = *reinterpret_cast<const uint4*>(wrow[j] + k1);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            x[d][i][0] = *reinterpret_cast<const uint4*>(xrow[i] + k0);
            x[d][i][1] = *reinterpret_cast<const uint4*>(xrow[i] + k1);
            s[d][i] = srow[i][(int64_t)b * p.xs_stride];
        }
        sw[d] = wscale[b];
    };
    auto add = [&](int d, int b) {
        if (b * 128 + 128 > p.K) {
            const bool out0 = b * 128 + 16 * g >= p.K, out1 = b * 128 + 64 + 16 * g >= p.K;
            const uint4 z = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (out0) w[d][j][0] = z;
                if (out1) w[d][j][1] = z;
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (out0) x[d][i][0] = z;
                if (out1) x[d][i][1] = z;
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const f32x4 t = block_product<WIDE>(operand(w[d][j][0], w[d][j][1]), operand(x[d][i][0], x[d][i][1]));
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] += t[e] * (s[d][i] * sw[d]);
            }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (wave + d * kRowWaves < p.nk) load(d, wave + d * kRowWaves);
    for (int b0 = wave; b0 < p.nk; b0 += DEPTH * kRowWaves) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int b = b0 + d * kRowWaves, next = b + DEPTH * kRowWaves;
            if (b < p.nk) add(d, b);
            if (next < p.nk) load(d, next);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int u = threadIdx.x; u < MT * NT * 64; u += kRowWaves * 64) {
        const int q = u >> 6, l = u & 63;
        f32x4 v = sums[0][q][l];
#pragma unroll
        for (int k = 1; k < kRowWaves; ++k) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += sums[k][q][l][e];
        }
        const float o[4] = {v[0], v[1], v[2], v[3]};
        store4(p, m0 + 16 * (q / NT) + (l & 15), n0 + 16 * (q % NT) + 4 * (l >> 4), o);
    }
}

template <int MT, int NT, int DEPTH>
static void rows_go(const LinearArgs& p, hipStream_t s)
{
    const dim3 grid(ceil_div(p.N, 16 * NT), ceil_div(p.M, 16 * MT)), block(kRowWaves * 64);
    if (p.wide && p.nk <= kRowWaves) hipLaunchKernelGGL((linear_rows_kernel<MT, NT, 1, true>), grid, block, 0, s, p);
    else if (p.wide) hipLaunchKernelGGL((linear_rows_kernel<MT, NT, DEPTH, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((linear_rows_kernel<MT, NT, DEPTH, false>), grid, block, 0, s, p);
}

// ------------------------------------------------------------------------------------------------
// Tiles of BM x BN, WM x WN waves; blocks of K in LDS, filled by direct loads.  A tile row is 128 bytes = eight 16-byte chunks; chunk c of row r is
// stored in slot c ^ (r / 2 & 7), so the 16 lanes that the LDS serves together (16 rows, one chunk) fall on 16 different bank groups.
// ------------------------------------------------------------------------------------------------
// Direct loads to LDS, 16 or 4 bytes per lane: base (wave-uniform) + off -> lds + 16 (4) lane.  Written as instructions because the compiler puts a
// wait for every such load in flight before each LDS read (it cannot tell their targets apart).  They have no result register; the kernels
// wait for them by count before the barrier that hands their target over.  m0 is reserved (nothing is kept there), which the compiler warns of where a
// statement names it; named it must be, so that none comes between an instruction that reads m0 and what sets it.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds16(const uint8_t* base, unsigned off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "m0");
}
__device__ __forceinline__ void load_lds4(const uint8_t* base, unsigned off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds), "v"(off), "s"(base) : "m0");
}
#pragma clang diagnostic pop

// What the kernels below have in common: a block's tile, its loads, fragments, scales and results.
template <int BM, int BN, int WM, int WN>
struct TileWork {
    static constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    static constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW;  // loads of a wave and block of K: rows, columns
    static constexpr int STAGE = (BM + BN) * 128;             // a block of K in LDS
    static_assert(NW % 2 == 0 && LA >= 1 && LB >= 1 && TN <= kScaleGroup && kScaleGroup % TN == 0 && BM % 64 == 0 && FM % 2 == 0, "shape");
    const LinearArgs& p;
    int lane, wave, g, c, wm, wn, m0, n0, slice, nk;          // nk: blocks of K of this slice
    int last, whole, chunk_at, back, k_tail;                  // last: the block that K ends in, -1: none; whole: blocks without it
    unsigned oa[LA], ob[LB], os;
    const uint8_t *xbase, *wbase, *sbase;
    const float* wscale;
    float w64;

    __device__ __forceinline__ TileWork(const LinearArgs& args) : p(args) {}

    // Block -> tile: each XCD (block id mod 8) gets a contiguous range of tiles; group_m M tiles x all N tiles follow each other, M
    // fastest, so that the blocks an XCD runs at a time share rows of both operands in its L2.
    __device__ __forceinline__ bool find()
    {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        g = lane >> 4;
        c = lane & 15;
        wm = wave / WN;
        wn = wave % WN;
        const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.ksplit, chunk = (total + 7) >> 3;
        const int L0 = ((int)blockIdx.x & 7) * chunk + ((int)blockIdx.x >> 3);
        if (((int)blockIdx.x >> 3) >= chunk || L0 >= total) return false;
        slice = L0 / tiles;
        const int L = L0 - slice * tiles, per_group = p.group_m * p.tiles_n, grp = L / per_group, in = L - grp * per_group;
        const int gm = min(p.group_m, p.tiles_m - grp * p.group_m), nt = in / gm, mt = grp * p.group_m + in - nt * gm;
        m0 = mt * BM;
        n0 = nt * BN;
        const int k_per = (p.nk + p.ksplit - 1) / p.ksplit, kb0 = slice * k_per;
        nk = min(p.nk, kb0 + k_per) - kb0;
        // A load is a wave-uniform base plus a lane's offset.  Rows past the end are the last one again (never stored); chunks past K, in the last
        // block, are the row's last one again and are cleared in LDS.
        const int r8 = lane >> 3;
        chunk_at = ((lane & 7) ^ ((4 * (wave & 1) + (r8 >> 1)) & 7)) * 16;
        k_tail = p.K & 127;
        last = (k_tail != 0 && kb0 + nk == p.nk) ? nk - 1 : -1;
        whole = last < 0 ? nk : nk - 1;
        back = max(0, chunk_at - (k_tail - 16));
#pragma unroll
        for (int i = 0; i < LA; ++i) oa[i] = (unsigned)min((wave + i * NW) * 8 + r8, p.M - 1 - m0) * (unsigned)p.x_stride + chunk_at;
#pragma unroll
        for (int i = 0; i < LB; ++i) ob[i] = (unsigned)min((wave + i * NW) * 8 + r8, p.N - 1 - n0) * (unsigned)p.K + chunk_at;
        os = (unsigned)min((wave & (BM / 64 - 1)) * 64 + lane, p.M - 1 - m0) * 4;
        xbase = p.x + (int64_t)m0 * p.x_stride + (int64_t)kb0 * 128;
        wbase = p.w + (int64_t)n0 * p.K + (int64_t)kb0 * 128;
        sbase = reinterpret_cast<const uint8_t*>(p.xs + (int64_t)kb0 * p.xs_stride + m0);
        wscale = p.ws + (int64_t)(min(n0 + wn * TN, p.N - 1) / kScaleGroup) * p.nk + kb0;
        w64 = 0.0f;
        return true;
    }
    // Load i of the rows, of the columns, and that of the rows' scales (64 per wave) of block k.
    __device__ __forceinline__ void load_rows(int k, int i, unsigned stage) const
    {
        load_lds16(xbase + (int64_t)k * 128, oa[i] - (k == last ? back : 0), stage + (wave + i * NW) * 1024);
    }
    __device__ __forceinline__ void load_columns(int k, int i, unsigned stage) const
    {
        load_lds16(wbase + (int64_t)k * 128, ob[i] - (k == last ? back : 0), stage + BM * 128 + (wave + i * NW) * 1024);
    }
    __device__ __forceinline__ void load_scales(int k, unsigned to) const
    {
        load_lds4(sbase + (int64_t)k * p.xs_stride * 4, os, to + (wave & (BM / 64 - 1)) * 256);
    }
    // Clears what this wave loaded in place of columns past K.
    __device__ __forceinline__ void clear_tail(char* stage) const
    {
        if (chunk_at < k_tail) return;
#pragma unroll
        for (int i = 0; i < LA + LB; ++i) *reinterpret_cast<uint4*>(stage + (wave + i * NW) * 1024 + lane * 16) = make_uint4(0, 0, 0, 0);
    }
    // Fragments of 16 rows or columns: a lane's chunks g and 4 + g.
    __device__ __forceinline__ i32x8 fragment(const char* St, int row) const
    {
        const int swz = (c >> 1) & 7;
        const char* at = St + (row + c) * 128;
        return operand(*reinterpret_cast<const uint4*>(at + ((g ^ swz) << 4)), *reinterpret_cast<const uint4*>(at + (((4 + g) ^ swz) << 4)));
    }
    __device__ __forceinline__ i32x8 rows(const char* St, int i) const { return fragment(St, wm * TM + i * 16); }
    __device__ __forceinline__ i32x8 columns(const char* St, int j) const { return fragment(St, BM + wn * TN + j * 16); }
    __device__ __forceinline__ float row_scale(const char* scales, int i) const { return reinterpret_cast<const float*>(scales)[wm * TM + i * 16 + c]; }
    // The columns' scale of block kt (ascending): 64 blocks at a time, lane l has block l's.  (A load in every block would be waited for
    // with all those on their way to LDS: 128 x 128 tiles, 256 rows by 14336 x 4096, 47 -> 30 us.)
    __device__ __forceinline__ float column_scale(int kt)
    {
        if ((kt & 63) == 0) {
            w64 = wscale[min(kt + lane, nk - 1)];
            asm volatile("" : "+v"(w64));                     // waited for here
        }
        return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w64), kt & 63));
    }
    // The wave's results.  In the accumulators neighbouring lanes hold different rows; 16 rows at a time go through LDS (the stages, read to the end
    // by everyone: the caller's barrier) and are written as whole pieces of rows, 16 bytes per lane.  8-byte slot s of row r stands at s ^ 2 (r / 2) in
    // rows of 128 bytes, at s ^ 2 (r / 4) in rows of 64: writes and reads are free of bank conflicts.  (Straight from the accumulators,
    // 16384 x 4096 x 128 63 us.)
    __device__ __forceinline__ void store(const f32x4 (&acc)[FM][FN], char* smem) const
    {
        constexpr int PIECES = TN / 8, SHIFT = PIECES == 8 ? 1 : 2;       // 16-byte pieces of a row
        static_assert(TN == 64 || TN == 32, "rows of 128 or 64 bytes");
        char* mine = smem + wave * 16 * TN * 2;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int m16 = m0 + wm * TM + i * 16, n64 = n0 + wn * TN;
            if (p.ksplit > 1) {
                const int m = m16 + c;
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const int n = n64 + j * 16 + 4 * g;
                    if (m < p.M && n < p.N)
                        *reinterpret_cast<float4*>(p.part + ((int64_t)slice * p.M + m) * p.part_stride + n) =
                            make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
                }
                continue;
            }
#pragma unroll
            for (int j = 0; j < FN; ++j)
                *reinterpret_cast<uint2*>(mine + c * TN * 2 + (((4 * j + g) ^ ((c >> SHIFT) << 1)) & (2 * PIECES - 1)) * 8) =
                    make_uint2(pack_bf16(acc[i][j][0], acc[i][j][1]), pack_bf16(acc[i][j][2], acc[i][j][3]));
            wave_lds_order();
#pragma unroll
            for (int q = 0; q < 16 * PIECES / 64; ++q) {
                const int row = (q * 64 + lane) / PIECES, piece = lane % PIECES, m = m16 + row, n = n64 + piece * 8;
                const uint4 v = *reinterpret_cast<const uint4*>(mine + row * TN * 2 + (((2 * piece) ^ ((row >> SHIFT) << 1)) & (2 * PIECES - 1)) * 8);
                if (m >= p.M) continue;
                bf16_t* dst = p.out + (int64_t)m * p.out_stride + n;
                if (p.vec16 && n + 8 <= p.N) {
                    *reinterpret_cast<uint4*>(dst) = v;
                } else {
                    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (n + e < p.N) reinterpret_cast<uint16_t*>(dst)[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                }
            }
            wave_lds_order();
        }
    }
};

// A ring of NST stages.  A block of K is FM steps; step i multiplies 16 rows by the wave's columns.  Behind each MFMA stand the multiply-adds of the
// step before (left to itself the compiler has all MFMAs first, and the matrix pipe idles for as long as the multiply-adds take), the
// reads of the next step's rows and, in the first steps, the loads of the block NST - 1 ahead.  Bound by what a CU pulls past its L2 where
// tiles are small (16, 24 and 32 KB per block of K of 64 x 64, 64 x 128 and 128 x 128 take 0.32, 0.47 and 0.65 us: 50 GB/s each), by the LDS where they are large; times stand at the plan below.
template <int BM, int BN, int WM, int WN, int NST, bool WIDE>
__global__ void __launch_bounds__(WM * WN * 64) linear_tile_kernel(LinearArgs p)
{
    using W = TileWork<BM, BN, WM, WN>;
    constexpr int FM = W::FM, FN = W::FN, LA = W::LA, LB = W::LB, LD = LA + LB + 1, STAGE = W::STAGE + BM * 4;
    static_assert((NST - 2) * LD <= 63 && NST * STAGE <= 160 * 1024, "shape");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    W t(p);
    if (!t.find()) return;
    const int nk = t.nk;
    // half of the loads of block k into stage st
    auto issue = [&](int k, int st, int half) {
        const unsigned to = lds0 + st * STAGE;
#pragma unroll
        for (int u = 0; u < LD; ++u) {
            if (u * 2 / LD != half) continue;
            if (u < LB) t.load_columns(k, u < LB ? u : 0, to);
            else if (u < LB + LA) t.load_rows(k, u < LB ? 0 : u < LB + LA ? u - LB : 0, to);
            else t.load_scales(k, to + W::STAGE);
        }
    };
    f32x4 acc[FM][FN], prod[2][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < FN; ++j) prod[0][j] = prod[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float s[FM], s_before = 0.0f;                         // scales of the rows; of the step before
#pragma unroll
    for (int st = 0; st < NST - 1; ++st)
#pragma unroll
        for (int half = 0; half < 2; ++half) issue(min(st, nk - 1), st, half);
    int stage = 0;
    for (int kt = 0; kt < nk; ++kt) {
        const float sw = t.column_scale(kt);
        __builtin_amdgcn_s_waitcnt(vmcnt_lgkm0_imm((NST - 2) * LD));
        lds_barrier();                                    // block kt is there; everyone has read block kt - 1
        char* St = smem + stage * STAGE;
        const int free = stage == 0 ? NST - 1 : stage - 1;
        if (kt == t.last) {
            t.clear_tail(St);
            __builtin_amdgcn_s_waitcnt(0xC07F);           // lgkmcnt(0)
            lds_barrier();
        }
        const int ahead = min(kt + NST - 1, nk - 1);      // past the end: the last block again, never read
        i32x8 fb[FN], fa[2];
        fa[0] = t.rows(St, 0);
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[j] = t.columns(St, j);
#pragma unroll
        for (int i = 0; i < FM; ++i) s[i] = t.row_scale(St + W::STAGE, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                prod[i & 1][j] = block_product<WIDE>(fb[j], fa[i & 1]);
                __builtin_amdgcn_sched_barrier(0);
                if (j == 0 && i + 1 < FM) fa[(i + 1) & 1] = t.rows(St, i + 1);
                if (j == FN / 2 && i < 2) issue(ahead, free, i);
                f32x4& into = acc[i == 0 ? FM - 1 : i - 1][j];
#pragma unroll
                for (int e = 0; e < 4; ++e) into[e] += prod[(i + 1) & 1][j][e] * s_before;
                __builtin_amdgcn_sched_barrier(0);
            }
            s_before = s[i] * sw;
        }
        stage = stage == NST - 1 ? 0 : stage + 1;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_lgkm0_imm(0));       // nothing is on its way to LDS, or being read there
    lds_barrier();
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[FM - 1][j][e] += prod[1][j][e] * s_before;
    t.store(acc, smem);
}

// 256 x 256: two blocks of K are all that LDS holds, so a load that waits for a whole block to be read has less than a block's time.  The
// columns' fragments stay in registers for the block, so their LDS is free soon after the block has begun, and that of the first half of each
// wave's rows halfway.  Hence two barriers per block:
//   before the middle step  the second half of the rows of this block has landed; the columns and the first half have been read by everyone,
//                           and the block after next is loaded in their place;
//   before the last step    the columns and the first half of the next block have landed; the second half of this one has been read, and that
//                           of the block after next is loaded.  The last step's MFMAs run while the next block's first operands come in, each in place
//                           of one that has been used for the last time.
// So every load has about one and a half blocks' time.  16384 x 7168 x 7168 655 us in a row of calls (2570 TFLOP/s; launches under a profiler 671
// to 742, with the clock that the power limit leaves); the ring kernel above with two stages takes 5 % longer; without its loads 0.53 ms.  The LDS bounds it:
// 192 KB of reads and 64 KB of writes per block of 2048 MFMA cycles (0.87 of the cycles, the matrix pipe has work in 0.68), where a wave tile of 128 x 64 is
// what leaves room for accumulators that the multiply-adds reach (they cannot address the accumulation registers).
template <int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM * WN * 64) linear_wide_kernel(LinearArgs p)
{
    using W = TileWork<BM, BN, WM, WN>;
    constexpr int NW = W::NW, TM = W::TM, FM = W::FM, FN = W::FN, LA = W::LA, LB = W::LB, STAGE = W::STAGE;
    constexpr int EARLY = LA / 2 + LB + 1, LATE = LA / 2; // loads behind the middle barrier (first halves, columns, scales), behind the last one
    constexpr int SCALES = 2 * STAGE;
    static_assert(SCALES + 3 * BM * 4 <= 160 * 1024, "LDS of a CU");
    static_assert(FM >= 4 && LA % 2 == 0 && TM / 2 % (NW * 8) == 0, "a load's rows are in one half of a wave's rows");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    W t(p);
    if (!t.find()) return;
    const int most = max(t.whole - 1, 0);
    // Load u of block kt: 0 .. EARLY - 1 the first halves of the rows, the columns and the scales, then the second halves.  Blocks past the end are the
    // last one again and never read.
    auto load = [&](int kt, int st, int slot, int u) {
        const int k = min(kt, most);
        const unsigned to = lds0 + st * STAGE;
        constexpr int RUN = TM / 2 / (NW * 8);            // loads of one half of a wave's rows follow each other
        const int v = u < LATE ? u : u - EARLY;
        const int i = v / RUN * 2 * RUN + v % RUN + (u < LATE ? 0 : RUN);
        if (u < LATE || u >= EARLY) t.load_rows(k, u < LATE || u >= EARLY ? i : 0, to);
        else if (u < EARLY - 1) t.load_columns(k, u - LATE, to);
        else t.load_scales(k, lds0 + SCALES + slot * BM * 4);
    };
    // all but the youngest EARLY + LATE loads of every wave have landed, and every wave's reads are done
    auto hand_over = [&]() {
        __builtin_amdgcn_s_waitcnt(vmcnt_lgkm0_imm(EARLY + LATE));
        lds_barrier();
    };
    auto scale_of = [&](int slot, int i) { return t.row_scale(smem + SCALES + slot * BM * 4, i); };
    f32x4 acc[FM][FN], prod[2][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < FN; ++j) prod[0][j] = prod[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    i32x8 fb[FN], fa[2];
    float row_scale[2], s_before = 0.0f;
#pragma unroll
    for (int u = 0; u < EARLY + LATE; ++u) load(0, 0, 0, u);
#pragma unroll
    for (int u = 0; u < EARLY; ++u) load(1, 1, 1, u);
    hand_over();
#pragma unroll
    for (int u = EARLY; u < EARLY + LATE; ++u) load(1, 1, 1, u);
    fa[0] = t.rows(smem, 0);
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[j] = t.columns(smem, j);
    row_scale[0] = scale_of(0, 0);
    int slot = 0;                                         // scales have a third place: they are read to the end of their block
    for (int kt = 0; kt < t.whole; ++kt) {
        const float sw = t.column_scale(kt);
        const int st = kt & 1, next_slot = slot == 2 ? 0 : slot + 1, free_slot = slot == 0 ? 2 : slot - 1;
        const char *St = smem + st * STAGE, *Sn = smem + (st ^ 1) * STAGE;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            if (i == FM / 2 - 1 || i == FM - 1) hand_over();
            const float s = row_scale[i & 1] * sw;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                prod[i & 1][j] = mfma_block(fb[j], fa[i & 1]);
                __builtin_amdgcn_sched_barrier(0);
                if (j == 0) {
                    fa[(i + 1) & 1] = i + 1 < FM ? t.rows(St, i + 1) : t.rows(Sn, 0);
                    row_scale[(i + 1) & 1] = i + 1 < FM ? scale_of(slot, i + 1) : scale_of(next_slot, 0);
                }
                if (i == FM - 1) fb[j] = t.columns(Sn, j);
                // one load at a time: several in a row queue up and hold the wave, and the MFMAs behind them
                constexpr int FIRST = (FM / 2 - 1) * FN, SPAN = FM / 2 * FN, LAST = (FM - 1) * FN;
                const int at = i * FN + j;
#pragma unroll
                for (int u = 0; u < EARLY; ++u)
                    if (at == FIRST + u * SPAN / EARLY) load(kt + 2, st, free_slot, u);
#pragma unroll
                for (int u = 0; u < LATE; ++u)
                    if (at == LAST + u * FN / LATE) load(kt + 2, st, free_slot, EARLY + u);
                f32x4& into = acc[i == 0 ? FM - 1 : i - 1][j];
#pragma unroll
                for (int e = 0; e < 4; ++e) into[e] += prod[(i + 1) & 1][j][e] * s_before;
                __builtin_amdgcn_sched_barrier(0);
            }
            s_before = s;
        }
        slot = next_slot;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_lgkm0_imm(0));       // nothing is on its way to LDS, or being read there
    lds_barrier();
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[FM - 1][j][e] += prod[1][j][e] * s_before;
    if (t.last >= 0) {                                    // the block that K ends in, by itself
#pragma unroll
        for (int i = 0; i < LB; ++i) t.load_columns(t.last, i, lds0);
#pragma unroll
        for (int i = 0; i < LA; ++i) t.load_rows(t.last, i, lds0);
        t.load_scales(t.last, lds0 + SCALES);
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        t.clear_tail(smem);
        __syncthreads();
        const float sw = t.wscale[t.last];
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[j] = t.columns(smem, j);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            fa[0] = t.rows(smem, i);
            const float s = scale_of(0, i) * sw;
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const f32x4 v = mfma_block(fb[j], fa[0]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] += v[e] * s;
            }
        }
        __syncthreads();
    }
    t.store(acc, smem);
}

// Sum of the slices of K, in their order, so the result is the same every time: a thread has four columns of a row.  Latency bound.
__global__ void __launch_bounds__(256) linear_sum_kernel(LinearArgs p)
{
    const int quads = p.part_stride / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, m = i / quads;
    if (m >= p.M) return;
    const int n = (int)(i - m * quads) * 4;
    const float4* src = reinterpret_cast<const float4*>(p.part + m * p.part_stride + n);
    const int64_t plane = (int64_t)p.M * quads;
    float4 v = src[0];
    // three slices' loads at a time (16 slices of 100 rows of 512: 5.8 -> 4.0 us)
#pragma unroll 3
    for (int z = 1; z < p.ksplit; ++z) {
        const float4 u = src[z * plane];
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    const float o[4] = {v.x, v.y, v.z, v.w};
    store4(p, (int)m, n, o);
}

// ------------------------------------------------------------------------------------------------
template <int BM, int BN, int WM, int WN, int NST, bool WIDE = false>
struct RingTile {
    static constexpr int kM = BM, kN = BN, kThreads = WM * WN * 64;
    static constexpr size_t kLds = (size_t)NST * ((BM + BN) * 128 + BM * 4);
    static constexpr auto kernel = &linear_tile_kernel<BM, BN, WM, WN, NST, WIDE>;
};
struct WideTile {
    static constexpr int kM = 256, kN = 256, kThreads = 512;
    static constexpr size_t kLds = 2 * 512 * 128 + 3 * 256 * 4;
    static constexpr auto kernel = &linear_wide_kernel<256, 256, 2, 4>;
};

// The ways to cut the product into tiles; all but the first leave room for one block per CU.
enum { kRows, kTile64, kTile64x128, kTile128, kTile128x256, kTile256, kShort64, kShort128, kWays };
template <typename F>
static auto with_tile(int way, F&& f)
{
    switch (way) {
        case kTile64: return f(RingTile<64, 64, 2, 2, 5>{});
        case kTile64x128: return f(RingTile<64, 128, 2, 4, 6>{});
        case kTile128: return f(RingTile<128, 128, 2, 4, 4>{});
        case kTile128x256: return f(RingTile<128, 256, 2, 4, 3>{});
        // three stages, two of the larger one: 256 x 4096 x 512 5.8 -> 5.2 us; 16384 x 4096 x 512 93 -> 119, one block per CU then
        case kShort64: return f(RingTile<64, 64, 2, 2, 3, true>{});
        case kShort128: return f(RingTile<128, 128, 2, 4, 2, true>{});
        default: return f(WideTile{});
    }
}

// The way that should take the least time.  A CU works on one tile at a time, so a product takes rounds of tiles; a tile takes 2 us (its first loads,
// its store) and for every block of K what is listed, from products of 2048 to 16384 rows; a launch takes 2 us.  Small tiles may be cut along K
// as well, which costs a second launch and the partial sums' way to memory and back.  Foretold and measured (us), K blocks:
//   64 x 64      0.32   256 rows by 6144 x 4096 26.5, 27.4; 1024 by 4096 x 7168 81.7, 82.7
//   64 x 128     0.47   256 by 6144 x 4096 19.0, 18.9;      1024 by 4096 x 7168 58.6, 55.8
//   128 x 128    0.65   1024 by 4096 x 7168 40.4, 40.7;     4096 by 4096 x 4096 93, 97
//   128 x 256    1.06   2048 by 4096 x 4096 37.9, 40.3;     16384 by 7168 x 7168 861, 867
//   256 x 256    1.72   4096 by 4096 x 4096 59, 61;         16384 by 7168 x 7168 690, 655 (680 where the constants were fitted)
// Up to 64 rows there is the rows kernel: its time goes with the weights, and from 33 rows on with the rows' trips as well.  Its blocks take 32 columns where
// blocks of 16 would be more than the CUs (16 and 32 columns, us, K = 4096: one row by 4096 6.0, 6.9, by 5120 8.6, 7.9, by 6144 8.7, 7.6, by 10240 11.8, 13.3, by 14336
// 14.7, 14.3; 32 rows by 4096 8.6, 10.4, by 5120 15.0, 10.8, by 6144 15.3, 10.9, by 14336 28.4, 20.8; 64 rows, K = 512, by 4096 4.1, 4.2, by 6144 5.3, 4.4).
// A last round that few CUs have a tile in costs as much as a full one, so the rows of whole rounds may go ahead, and the rest be cut in tiles
// that suit it.
static constexpr struct { int m, n; double block; } kTile[] = {
    {0, 0, 0}, {64, 64, 0.32}, {64, 128, 0.47}, {128, 128, 0.65}, {128, 256, 1.06}, {256, 256, 1.72}};
constexpr int kCus = 256;

static double tile_rounds(int way, int64_t tiles, int blocks)
{
    return (double)((tiles + kCus - 1) / kCus) * (blocks * kTile[way].block + 2.0);
}

static LinearPlan one_way(int M, int N, int K, bool wide, double& least)
{
    LinearPlan best{kRows, 1, M <= 16 ? 16 : M <= 32 ? 32 : 64, 0, 0, 0, wide};
    best.columns = ceil_div(N, 16) * ceil_div(M, best.rows) > kCus ? 32 : 16;
    least = 4.0 + (M <= 16 ? 0.2e-6 : M <= 32 ? 0.28e-6 : 0.46e-6) * N * K;
    if (M <= 32 || (M <= 64 && wide)) return best;
    if (wide) {                                           // a tile is its loads and its store: large ones where they still fill the CUs
                                                          // (64 x 64 and 128 x 128, us: 16384 x 4096 x 128 59.6, 53.1; 2048 x 1024 x 256 5.5, 6.2)
        best.way = (int64_t)ceil_div(M, 128) * ceil_div(N, 128) >= kCus ? kShort128 : kShort64;
        return best;
    }
    const int nk = ceil_div(K, kScaleGroup);
    if (M > 64) least = 1e300;
    for (int way = kTile64; way <= kTile256; ++way)
        for (int ks = 1; ks <= (way == kTile64 ? 16 : 1); ks *= 2) {
            const int per = ceil_div(nk, ks);
            if (ks > 1 && (per < 4 || ceil_div(nk, per) != ks)) continue;          // no slice is empty
            const int64_t tiles = (int64_t)ceil_div(M, kTile[way].m) * ceil_div(N, kTile[way].n) * ks;
            double us = 2.0 + tile_rounds(way, tiles, per);
            if (ks > 1) us += 2.5 + 2e-6 * M * N * ks;
            if (us < least) {
                least = us;
                best = {way, ks, 0, 0, 0, 0, false};
            }
        }
    return best;
}

LinearPlan linear_plan(int M, int N, int K, bool exact)
{
    const bool wide = exact || K <= kShortK;
    double least, rest;
    LinearPlan best = one_way(M, N, K, wide, least);
    if (wide || M <= 128) return best;
    for (int way = kTile128; way <= kTile256; ++way) {
        const int cols = ceil_div(N, kTile[way].n);
        const int64_t rounds = (int64_t)ceil_div(M, kTile[way].m) * cols / kCus, rows = rounds * kCus / cols * kTile[way].m;
        if (rows <= 0 || rows >= M) continue;
        const double us = 2.0 + tile_rounds(way, rows / kTile[way].m * cols, ceil_div(K, kScaleGroup));
        if (us >= least) continue;
        LinearPlan p = one_way(M - (int)rows, N, K, false, rest);
        if (us + rest < least) {
            least = us + rest;
            best = p;
            best.first_way = way;
            best.first_rows = (int)rows;
        }
    }
    return best;
}

size_t linear_workspace_bytes(const LinearPlan& L, int M, int N)
{
    return L.ksplit > 1 ? align_up((size_t)L.ksplit * (M - L.first_rows) * align_up(N, 4) * sizeof(float), 256) : 0;
}

// Enough for every M up to M_max.  The plan sees M in tiles of 64 rows, but for the partial sums' way, which makes fewer slices the better choice as M grows:
// so the slices of the smallest M of a tile (33 of the first: fewer rows have a kernel of their own) are the most that its rows get.  Rows left
// over by whole rounds of tiles are a product of fewer rows.
size_t linear_workspace_bound(int M_max, int N, int K)
{
    if (K <= kShortK) return 0;
    size_t rows = 0;                                      // slices x rows
    double us;
    for (int first = 33; first <= M_max; first = first == 33 ? 65 : first + 64) {
        const int last = std::min(M_max, (first + 63) / 64 * 64), ks = one_way(first, N, K, false, us).ksplit;
        if (ks > 1) rows = std::max(rows, (size_t)ks * last);
    }
    return align_up(rows * align_up(N, 4) * sizeof(float), 256);
}

hipError_t init_linear_kernels()
{
    for (int way = kTile64; way < kWays; ++way) {
        hipError_t e = with_tile(way, [](auto tile) {
            return hipFuncSetAttribute(reinterpret_cast<const void*>(tile.kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)tile.kLds);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_linear(const moe_linear_args& a, const LinearPlan& L, void* ws, hipStream_t s)
{
    LinearArgs p;
    p.x = static_cast<const uint8_t*>(a.x8); p.w = static_cast<const uint8_t*>(a.w8);
    p.xs = a.x_scale; p.ws = a.w_scale;
    p.out = static_cast<bf16_t*>(a.out);
    p.part = static_cast<float*>(ws);
    p.x_stride = a.x_stride; p.xs_stride = a.x_scale_stride; p.out_stride = a.out_stride;
    p.M = a.M; p.N = a.N; p.K = a.K; p.nk = ceil_div(a.K, kScaleGroup);
    p.part_stride = (int)align_up(a.N, 4);
    p.wide = L.wide;
    p.vec = (a.out_stride & 3) == 0 && (reinterpret_cast<uintptr_t>(a.out) & 7u) == 0;
    p.vec16 = (a.out_stride & 7) == 0 && (reinterpret_cast<uintptr_t>(a.out) & 15u) == 0;
    auto tiles = [&](int way) {
        return with_tile(way, [&](auto tile) {
            p.tiles_m = ceil_div(p.M, tile.kM);
            p.tiles_n = ceil_div(p.N, tile.kN);
            p.group_m = 8;                                // fitted with 16384 x 7168 x 7168 at 694 us: 1, 4, 8, 16: 732, 694, 694, 708; 8192 x 4096 x 14336 386, 375, 373, 381
            const int total = p.tiles_m * p.tiles_n * p.ksplit;
            hipLaunchKernelGGL(tile.kernel, dim3((total + 7) / 8 * 8), dim3(tile.kThreads), tile.kLds, s, p);
            return hipGetLastError();
        });
    };
    hipError_t e;
    if (L.first_rows > 0) {
        p.M = L.first_rows;
        p.ksplit = 1;
        if ((e = tiles(L.first_way)) != hipSuccess) return e;
        p.M = a.M - L.first_rows;
        p.x += L.first_rows * p.x_stride;
        p.xs += L.first_rows;
        p.out += L.first_rows * p.out_stride;
    }
    p.ksplit = L.ksplit;
    if (L.way == kRows) {
        const bool two = L.columns == 32;
        if (L.rows == 16) two ? rows_go<1, 2, 3>(p, s) : rows_go<1, 1, 4>(p, s);
        else if (L.rows == 32) two ? rows_go<2, 2, 3>(p, s) : rows_go<2, 1, 4>(p, s);
        else two ? rows_go<4, 2, 2>(p, s) : rows_go<4, 1, 2>(p, s);
        return hipGetLastError();
    }
    e = tiles(L.way);
    if (e != hipSuccess || L.ksplit == 1) return e;
    hipLaunchKernelGGL(linear_sum_kernel, dim3((unsigned)(((int64_t)p.M * (p.part_stride / 4) + 255) / 256)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace bmoe
