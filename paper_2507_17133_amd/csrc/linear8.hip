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

namespace bmoe {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct LinearArgs {
    const uint8_t *x, *w;
    const float *xs, *ws;
    bf16_t* out;
    float* part;                                          // [ksplit][M][N] where K is cut
    int64_t x_stride, xs_stride, out_stride;
    int M, N, K, nk;                                      // nk: blocks of K
    int tiles_m, tiles_n, group_m, ksplit;
    int vec;                                              // out rows take 8-byte stores
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
// Few rows (at most 64), or short K: every block takes 16 columns and 16 MT rows, its eight waves take the blocks of K by turns and are
// summed through LDS in wave order.  Operands come straight from memory into registers and are widened to bf16 (exact) on the way to
// four 16x16x32 bf16 MFMAs per block of K, which add up in fp32.  (The 8-bit MFMA drops what lies below 2^-13 of the largest product it
// adds up at a time; over whole blocks of 128 that averages out, over a few k's it does not.)  Bound by the weights' stream.
// ------------------------------------------------------------------------------------------------
constexpr int kRowWaves = 8;
constexpr int kShortK = 256;                              // up to here every shape goes this way

__device__ __forceinline__ unsigned widen_lo(unsigned w) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)); }
__device__ __forceinline__ unsigned widen_hi(unsigned w) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)); }
__device__ __forceinline__ bf16x8 widen8(unsigned a, unsigned b)
{
    return __builtin_bit_cast(bf16x8, make_uint4(widen_lo(a), widen_hi(a), widen_lo(b), widen_hi(b)));
}

template <int MT>
__global__ void __launch_bounds__(kRowWaves * 64) linear_rows_kernel(LinearArgs p)
{
    __shared__ f32x4 sums[kRowWaves][MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
    const uint8_t* wrow = p.w + (int64_t)min(n0 + c, p.N - 1) * p.K;
    const uint8_t* xrow[MT];
    const float* srow[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = min(m0 + 16 * i + c, p.M - 1);
        xrow[i] = p.x + (int64_t)m * p.x_stride;
        srow[i] = p.xs + m;
    }
    const float* wscale = p.ws + (int64_t)(n0 / kScaleGroup) * p.nk;
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int b = wave; b < p.nk; b += kRowWaves) {
        const int k0 = b * 128 + 16 * g, k1 = k0 + 64;
        const bool in0 = k0 < p.K, in1 = k1 < p.K;
        const uint4 z = make_uint4(0, 0, 0, 0);
        auto pair = [&](const uint8_t* row, uint4& a, uint4& c2) {
            a = in0 ? *reinterpret_cast<const uint4*>(row + k0) : z;
            c2 = in1 ? *reinterpret_cast<const uint4*>(row + k1) : z;
        };
        uint4 w0, w1;
        pair(wrow, w0, w1);
        const float sw = wscale[b];
        const bf16x8 w[4] = {widen8(w0.x, w0.y), widen8(w0.z, w0.w), widen8(w1.x, w1.y), widen8(w1.z, w1.w)};
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            uint4 x0, x1;
            pair(xrow[i], x0, x1);
            const float s = sw * srow[i][(int64_t)b * p.xs_stride];
            f32x4 t = f32x4{0.f, 0.f, 0.f, 0.f};
            t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[0], widen8(x0.x, x0.y), t, 0, 0, 0);
            t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[1], widen8(x0.z, x0.w), t, 0, 0, 0);
            t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[2], widen8(x1.x, x1.y), t, 0, 0, 0);
            t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[3], widen8(x1.z, x1.w), t, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][e] += t[e] * s;
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    for (int u = threadIdx.x; u < MT * 64; u += kRowWaves * 64) {
        const int i = u >> 6, l = u & 63;
        f32x4 v = sums[0][i][l];
#pragma unroll
        for (int w = 1; w < kRowWaves; ++w) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += sums[w][i][l][e];
        }
        const float o[4] = {v[0], v[1], v[2], v[3]};
        store4(p, m0 + 16 * i + (l & 15), n0 + 4 * (l >> 4), o);
    }
}

// ------------------------------------------------------------------------------------------------
// Tiles of BM x BN, WM x WN waves, a ring of NST stages of one block of K in LDS, filled by direct loads.  A tile row is 128 bytes = eight
// 16-byte chunks; chunk c of row r is stored in slot c ^ (r / 2 & 7), so the 16 lanes that the LDS serves together (16 rows, one
// chunk) fall on 16 different bank groups.
// ------------------------------------------------------------------------------------------------
// Direct loads to LDS, 16 or 4 bytes per lane: base (wave-uniform) + off -> lds + 16 (4) lane.  Written as instructions because the compiler puts a
// wait for every such load in flight before each LDS read (it cannot tell their targets apart).  They have no result register; the kernel
// waits for them by count before the barrier that hands their stage over.  Nothing else in the kernel uses m0.
__device__ __forceinline__ void load_lds16(const uint8_t* base, unsigned off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base));
}
__device__ __forceinline__ void load_lds4(const uint8_t* base, unsigned off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base));
}

template <int BM, int BN, int WM, int WN, int NST>
__global__ void __launch_bounds__(WM * WN * 64) linear_tile_kernel(LinearArgs p)
{
    constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, LD = LA + LB + 1;       // loads of a wave and block of K
    constexpr int TILE = (BM + BN) * 128, STAGE = TILE + BM * 4;
    static_assert(NW % 2 == 0 && LA >= 1 && LB >= 1 && TN <= kScaleGroup && BM % 64 == 0 && NST * STAGE <= 160 * 1024, "shape");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;

    // Block -> tile: each XCD (block id mod 8) gets a contiguous range of tiles; group_m M tiles x all N tiles follow each other, M
    // fastest, so that the blocks an XCD runs at a time share rows of both operands in its L2.
    const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.ksplit, chunk = (total + 7) >> 3;
    const int L0 = ((int)blockIdx.x & 7) * chunk + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= chunk || L0 >= total) return;
    const int slice = L0 / tiles, L = L0 - slice * tiles;
    const int per_group = p.group_m * p.tiles_n, grp = L / per_group, in = L - grp * per_group;
    const int gm = min(p.group_m, p.tiles_m - grp * p.group_m);
    const int nt = in / gm, mt = grp * p.group_m + in - nt * gm;
    const int m0 = mt * BM, n0 = nt * BN;
    const int k_per = (p.nk + p.ksplit - 1) / p.ksplit, kb0 = min(p.nk, slice * k_per), nk = min(p.nk, kb0 + k_per) - kb0;

    // A load is a wave-uniform base plus a lane's offset.  Rows past the end are the last one again (never stored); chunks past K, in the last
    // block, are the row's last one again and are cleared in LDS.
    const int r8 = lane >> 3, chunk_at = ((lane & 7) ^ ((4 * (wave & 1) + (r8 >> 1)) & 7)) * 16;
    const int k_tail = p.K & 127, last = (k_tail != 0 && kb0 + nk == p.nk) ? nk - 1 : -1;       // the block that K ends in
    const int back = max(0, chunk_at - (k_tail - 16));
    unsigned oa[LA], ob[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) oa[i] = (unsigned)min((wave + i * NW) * 8 + r8, p.M - 1 - m0) * (unsigned)p.x_stride + chunk_at;
#pragma unroll
    for (int i = 0; i < LB; ++i) ob[i] = (unsigned)min((wave + i * NW) * 8 + r8, p.N - 1 - n0) * (unsigned)p.K + chunk_at;
    const uint8_t* xbase = p.x + (int64_t)m0 * p.x_stride + (int64_t)kb0 * 128;
    const uint8_t* wbase = p.w + (int64_t)n0 * p.K + (int64_t)kb0 * 128;
    const int piece = wave & (BM / 64 - 1);               // 64 rows' scales
    const unsigned os = (unsigned)min(piece * 64 + lane, p.M - 1 - m0) * 4;
    const uint8_t* sbase = reinterpret_cast<const uint8_t*>(p.xs + (int64_t)kb0 * p.xs_stride + m0);
    // part of FM of the loads of block kt into stage st
    auto issue = [&](int kt, int st, int part) {
        const unsigned to = lds0 + st * STAGE, less = kt == last ? back : 0;
        const uint8_t *wk = wbase + (int64_t)kt * 128, *xk = xbase + (int64_t)kt * 128;
#pragma unroll
        for (int i = 0; i < LD; ++i) {
            if (i * FM / LD != part) continue;
            if (i < LB) load_lds16(wk, ob[i < LB ? i : 0] - less, to + BM * 128 + (wave + i * NW) * 1024);
            else if (i < LB + LA) load_lds16(xk, oa[i < LB ? 0 : i < LB + LA ? i - LB : 0] - less, to + (wave + (i - LB) * NW) * 1024);
            else load_lds4(sbase + (int64_t)kt * p.xs_stride * 4, os, to + TILE + piece * 256);
        }
    };

    const int wm = wave / WN, wn = wave % WN;
    const int swz = (c >> 1) & 7, s0 = (g ^ swz) << 4, s1 = ((4 + g) ^ swz) << 4;
    const int a_off = (wm * TM + c) * 128, b_off = (BM + wn * TN + c) * 128;
    const float* wscale = p.ws + (int64_t)(min(n0 + wn * TN, p.N - 1) / kScaleGroup) * p.nk + kb0;
    f32x4 acc[FM][FN], prod[2][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < FN; ++j) prod[0][j] = prod[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float s[FM], s_last = 0.0f;                           // scales of the rows; of the last 16 rows of the block before

    // A block of K: step i multiplies 16 rows by the wave's columns.  Behind each MFMA stand the multiply-adds of the step before, and in the
    // steps the reads of the next step's rows and the loads of the block after next, one at a time.  The compiler would rather have all
    // MFMAs first, which leaves the matrix pipe idle for as long as the multiply-adds take.
    static_assert(FM % 2 == 0, "the last step's products are in the second set");
#pragma unroll
    for (int st = 0; st < NST - 1; ++st)
#pragma unroll
        for (int i = 0; i < FM; ++i) issue(min(st, nk - 1), st, i);
    int stage = 0;
    for (int kt = 0; kt < nk; ++kt) {
        const float sw = wscale[kt];
        __builtin_amdgcn_s_waitcnt(vmcnt_lgkm0_imm((NST - 2) * LD));
        lds_barrier();                                    // block kt is there; everyone has read block kt - 1
        const char* St = smem + stage * STAGE;
        const int free = stage == 0 ? NST - 1 : stage - 1;
        if (kt == last) {                                 // what was loaded in place of columns past K
            char* mine = smem + stage * STAGE + wave * 1024 + lane * 16;
            if (chunk_at >= k_tail) {
#pragma unroll
                for (int i = 0; i < LA + LB; ++i) *reinterpret_cast<uint4*>(mine + i * NW * 1024) = make_uint4(0, 0, 0, 0);
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);           // lgkmcnt(0)
            lds_barrier();
        }
        const int next = min(kt + NST - 1, nk - 1);       // past the end: the last block again, never read
        i32x8 fb[FN], fa[2];
        auto frag = [&](int at) {
            return operand(*reinterpret_cast<const uint4*>(St + at + s0), *reinterpret_cast<const uint4*>(St + at + s1));
        };
        fa[0] = frag(a_off);
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[j] = frag(b_off + j * 2048);
#pragma unroll
        for (int i = 0; i < FM; ++i) s[i] = *reinterpret_cast<const float*>(St + TILE + (wm * TM + i * 16 + c) * 4);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const float sp = i == 0 ? s_last : s[i - 1];
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                prod[i & 1][j] = mfma_block(fb[j], fa[i & 1]);
                __builtin_amdgcn_sched_barrier(0);
                if (j == 0 && i + 1 < FM) fa[(i + 1) & 1] = frag(a_off + (i + 1) * 2048);
                if (j == FN / 2) issue(next, free, i);
                f32x4& into = acc[i == 0 ? FM - 1 : i - 1][j];
#pragma unroll
                for (int e = 0; e < 4; ++e) into[e] += prod[(i + 1) & 1][j][e] * sp;
                __builtin_amdgcn_sched_barrier(0);
            }
            s[i] *= sw;
        }
        s_last = s[FM - 1];
        stage = stage == NST - 1 ? 0 : stage + 1;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));             // nothing is on its way to LDS when the block ends
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[FM - 1][j][e] += prod[1][j][e] * s_last;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int m = m0 + wm * TM + i * 16 + c;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int n = n0 + wn * TN + j * 16 + 4 * g;
            const float o[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (p.ksplit == 1) {
                store4(p, m, n, o);
            } else if (m < p.M) {
                float* dst = p.part + ((int64_t)slice * p.M + m) * p.N + n;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < p.N) dst[e] = o[e];
            }
        }
    }
}

// Sum of the slices of K, in their order.
__global__ void __launch_bounds__(256) linear_sum_kernel(LinearArgs p)
{
    const int64_t plane = (int64_t)p.M * p.N, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= plane) return;
    float v = p.part[i];
    for (int z = 1; z < p.ksplit; ++z) v += p.part[z * plane + i];
    const int64_t m = i / p.N;
    p.out[m * p.out_stride + (i - m * p.N)] = (bf16_t)v;
}

// ------------------------------------------------------------------------------------------------
struct LinearPlan { int kind, bm, bn, ksplit; };          // kind 0: rows kernel, 1: tiles

static LinearPlan linear_plan(int M, int N, int K)
{
    LinearPlan L{0, 0, 0, 1};
    if (M <= 64 || K <= kShortK) return L;
    L.kind = 1;
    L.bm = L.bn = 128;
    if ((int64_t)ceil_div(M, 256) * ceil_div(N, 256) >= 200) L.bm = L.bn = 256;
    else {
        const int tiles = ceil_div(M, 128) * ceil_div(N, 128), nk = ceil_div(K, 128);
        while (L.ksplit < 8 && tiles * L.ksplit * 2 <= 256 && nk / (L.ksplit * 2) >= 4) L.ksplit *= 2;
        L.ksplit = ceil_div(nk, ceil_div(nk, L.ksplit));  // no slice is empty
    }
    return L;
}

size_t linear_workspace_bytes(int M, int N, int K)
{
    const LinearPlan L = linear_plan(M, N, K);
    return L.ksplit > 1 ? align_up((size_t)L.ksplit * M * N * sizeof(float), 256) : 0;
}

template <int BM, int BN, int WM, int WN, int NST>
struct TileKernel {
    static constexpr size_t kLds = (size_t)NST * ((BM + BN) * 128 + BM * 4);
    static hipError_t init()
    {
        return hipFuncSetAttribute(reinterpret_cast<const void*>(&linear_tile_kernel<BM, BN, WM, WN, NST>),
                                   hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
    }
    static void go(LinearArgs& p, hipStream_t s)
    {
        p.tiles_m = ceil_div(p.M, BM);
        p.tiles_n = ceil_div(p.N, BN);
        p.group_m = 8;
        const int total = p.tiles_m * p.tiles_n * p.ksplit;
        hipLaunchKernelGGL((linear_tile_kernel<BM, BN, WM, WN, NST>), dim3((total + 7) / 8 * 8), dim3(WM * WN * 64), kLds, s, p);
    }
};
using Tile256 = TileKernel<256, 256, 2, 4, 2>;
using Tile128 = TileKernel<128, 128, 2, 2, 3>;

hipError_t init_linear_kernels()
{
    hipError_t e = Tile256::init();
    return e != hipSuccess ? e : Tile128::init();
}

hipError_t launch_linear(const moe_linear_args& a, void* ws, hipStream_t s)
{
    const LinearPlan L = linear_plan(a.M, a.N, a.K);
    LinearArgs p;
    p.x = static_cast<const uint8_t*>(a.x8); p.w = static_cast<const uint8_t*>(a.w8);
    p.xs = a.x_scale; p.ws = a.w_scale;
    p.out = static_cast<bf16_t*>(a.out);
    p.part = static_cast<float*>(ws);
    p.x_stride = a.x_stride; p.xs_stride = a.x_scale_stride; p.out_stride = a.out_stride;
    p.M = a.M; p.N = a.N; p.K = a.K; p.nk = ceil_div(a.K, 128);
    p.ksplit = L.ksplit;
    p.vec = (a.out_stride & 3) == 0 && (reinterpret_cast<uintptr_t>(a.out) & 7u) == 0;
    if (L.kind == 0) {
        const int mt = a.M <= 16 ? 1 : a.M <= 32 ? 2 : 4;
        const dim3 grid(ceil_div(a.N, 16), ceil_div(a.M, 16 * mt)), block(kRowWaves * 64);
        if (mt == 1) hipLaunchKernelGGL((linear_rows_kernel<1>), grid, block, 0, s, p);
        else if (mt == 2) hipLaunchKernelGGL((linear_rows_kernel<2>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((linear_rows_kernel<4>), grid, block, 0, s, p);
        return hipGetLastError();
    }
    if (L.bm == 256) Tile256::go(p, s);
    else Tile128::go(p, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || L.ksplit == 1) return e;
    hipLaunchKernelGGL(linear_sum_kernel, dim3((unsigned)(((int64_t)a.M * a.N + 255) / 256)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace bmoe
