// Root-mean-square norm with the residual's addition and an 8-bit output, the 8-bit output alone, and the 8-bit form of a weight.
//
//   h = x + r      y = h * rsqrt(mean(h^2) + eps) * w      per group of 128 columns: s = max(amax|y|, 2^-100) / 448, y8 = e4m3(y / s)
//
// One pass: a row's vectors stay in the registers of the threads that share it between the sum of squares and the outputs, so every
// input is read once and every output written once: HBM bound.  The norm's inputs and the residual, whose next reader is far off, pass by the caches, and so do large bf16
// rows (16384 x 7168 with residual to e4m3 149 -> 137 us, 6.0 TB/s, in a graph over sets of inputs; 256 x 4096 5.1 -> 4.2); e4m3 rows stay for the product that reads them (8-byte
// stores past the caches are slower besides: 142).  One row of 2048: 2.4 us, latency.
#include "layer.h"

#include <type_traits>

namespace bmoe {

struct NormArgs {
    const bf16_t *x, *r, *w;
    bf16_t *ro, *y;
    uint8_t* y8;
    float* scale;
    int64_t xs, rs, ros, ys, y8s, ss;
    int T, d;
    float eps;
};

// Largest |value| of a group by its bits: a NaN's are above an infinity's, an infinity's above every finite one, so a group that holds
// one says so in its scale.
__device__ __forceinline__ unsigned abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Its 448th part, rounded as the division rounds it (for every significand): a product, corrected by its remainder.
__device__ __forceinline__ float group_scale(unsigned bits)
{
    const float m = __uint_as_float(max(bits, __float_as_uint(kLeastMagnitude))), q = m * (1.0f / kE4m3Max);
    return m < __builtin_inff() ? __builtin_fmaf(-__builtin_fmaf(q, kE4m3Max, -m), 1.0f / kE4m3Max, q) : m;
}

// By a group's scale: at least 2^-64, infinite or NaN.  The hardware's reciprocal with one Newton step.
__device__ __forceinline__ Divisor by_group_scale(float s)
{
    const float finite = s < __builtin_inff() ? s : 0.0f, r = __builtin_amdgcn_rcpf(s);
    return Divisor(finite, __builtin_fmaf(__builtin_fmaf(-finite, r, 1.0f), r, r));
}

// A row's vectors of 8 columns are dealt out over `across` threads, NV each: vector v of thread i is columns 8 (v across + i) .., so 16 neighbouring lanes
// hold one group of 128 columns.  ONE_ROW: the whole block, in as many waves as leave few lanes without a vector; else a wave per row, four to a block.
template <bool ONE_ROW, int NV, bool NORM, bool ONCE>
__global__ void __launch_bounds__(ONE_ROW ? 1024 : 256) norm_kernel(NormArgs p)
{
    const int across = ONE_ROW ? (int)blockDim.x : 64, i = ONE_ROW ? (int)threadIdx.x : (int)threadIdx.x & 63;
    const int t = ONE_ROW ? (int)blockIdx.x : (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6);
    if (!ONE_ROW && t >= p.T) return;                     // whole waves, and no barrier then
    const bf16_t* xr = p.x + (int64_t)t * p.xs;
    float h[NV][8];
    float sum = 0.0f;
    uint4 xv[NV], rv[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = 8 * (v * across + i);
        xv[v] = rv[v] = make_uint4(0, 0, 0, 0);
        if (c < p.d) {
            xv[v] = load16<NORM || ONCE>(xr + c);
            if (NORM && p.r) rv[v] = load16<true>(p.r + (int64_t)t * p.rs + c);
        }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = 8 * (v * across + i);
        unpack_bf16(xv[v], h[v]);
        if constexpr (NORM) {
            float f[8];
            unpack_bf16(rv[v], f);
            if (p.r) {
#pragma unroll
                for (int e = 0; e < 8; ++e) h[v][e] += f[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += h[v][e] * h[v][e];
            if (p.ro && c < p.d) store16<true>(p.ro + (int64_t)t * p.ros + c, pack_bf16x8(h[v]));
        }
    }
    if constexpr (NORM) {
#pragma unroll
        for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m);
        if constexpr (ONE_ROW) {
            __shared__ float part[16];
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
            __syncthreads();
            sum = 0.0f;
            for (int k = 0; k < across >> 6; ++k) sum += part[k];
        }
        const float inv = 1.0f / sqrtf(sum / (float)p.d + p.eps);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = 8 * (v * across + i);
            float w[8];
            if (p.w) {
                uint4 wv = make_uint4(0, 0, 0, 0);
                if (c < p.d) wv = *reinterpret_cast<const uint4*>(p.w + c);
                unpack_bf16(wv, w);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) h[v][e] *= p.w ? inv * w[e] : inv;
            if (p.y && c < p.d) store16<ONCE>(p.y + (int64_t)t * p.ys + c, pack_bf16x8(h[v]));
        }
    }
    if (!p.y8) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = 8 * (v * across + i);
        unsigned bits = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) bits = max(bits, abs_bits(h[v][e]));
        if (c >= p.d) bits = 0;                           // 0 times an infinite 1 / rms is no member of the group
#pragma unroll
        for (int m = 8; m; m >>= 1) bits = max(bits, (unsigned)__shfl_xor((int)bits, m));
        const float s = group_scale(bits);
        if (c >= p.d) continue;
        const Divisor div = by_group_scale(lift_tiny(h[v], s));
        uint2 o;
        o.x = pack_e4m3(div(h[v][0]), div(h[v][1]), div(h[v][2]), div(h[v][3]));
        o.y = pack_e4m3(div(h[v][4]), div(h[v][5]), div(h[v][6]), div(h[v][7]));
        *reinterpret_cast<uint2*>(p.y8 + (int64_t)t * p.y8s + c) = o;
        if ((c & (kScaleGroup - 1)) == 0) p.scale[(int64_t)(c / kScaleGroup) * p.ss + t] = s;
    }
}

template <bool ONE_ROW, int NV>
static void norm_go(const NormArgs& p, bool norm, hipStream_t s)
{
    const int vectors = p.d / 8, threads = ONE_ROW ? ceil_div(vectors, NV * 64) * 64 : 256, grid = ONE_ROW ? p.T : ceil_div(p.T, 4);
    const bool once = (int64_t)p.T * p.d * 2 > kCachedBytes;
    auto go = [&](auto norms, auto past) {
        hipLaunchKernelGGL((norm_kernel<ONE_ROW, NV, decltype(norms)::value, decltype(past)::value>), dim3(grid), dim3(threads), 0, s, p);
    };
    if (norm) once ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
    else once ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
}

hipError_t launch_norm(const moe_norm_args& a, bool norm, hipStream_t s)
{
    NormArgs p{static_cast<const bf16_t*>(a.x), static_cast<const bf16_t*>(a.residual), static_cast<const bf16_t*>(a.weight),
               static_cast<bf16_t*>(a.residual_out), static_cast<bf16_t*>(a.y), static_cast<uint8_t*>(a.y8), a.scale,
               a.x_stride, a.residual_stride, a.residual_out_stride, a.y_stride, a.y8_stride, a.scale_stride, a.T, a.d, a.eps};
    if (a.d <= 512) norm_go<false, 1>(p, norm, s);
    else if (a.d <= 1024) norm_go<false, 2>(p, norm, s);
    else if (a.d <= 4096) norm_go<true, 1>(p, norm, s);
    else if (a.d <= 8192) norm_go<true, 2>(p, norm, s);
    else norm_go<true, 4>(p, norm, s);
    return hipGetLastError();
}

// One block per 128 x 128 block of the weight, whose values stay in registers between the maximum and the store (16 columns of four rows per
// thread): one pass, HBM bound.  7168 x 7168 27 us (5.6 TB/s, six weights in turn).
__global__ void __launch_bounds__(256) quantize_weight_kernel(const bf16_t* __restrict__ w, int N, int K, uint8_t* __restrict__ w8,
                                                              float* __restrict__ scale)
{
    const int k0 = blockIdx.x * kScaleGroup + (threadIdx.x & 7) * 16, n0 = blockIdx.y * kScaleGroup + (threadIdx.x >> 3);
    float v[4][16];
    unsigned bits = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 32 * j;
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        if (n < N && k0 < K) {
            const uint4* src = reinterpret_cast<const uint4*>(w + (int64_t)n * K + k0);
            a = src[0];
            b = src[1];
        }
        unpack_bf16(a, v[j]);
        unpack_bf16(b, v[j] + 8);
#pragma unroll
        for (int e = 0; e < 16; ++e) bits = max(bits, abs_bits(v[j][e]));
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) bits = max(bits, (unsigned)__shfl_xor((int)bits, m));
    __shared__ unsigned part[4];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = bits;
    __syncthreads();
    bits = max(max(part[0], part[1]), max(part[2], part[3]));
    const float s = group_scale(bits);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 32 * j;
        if (n >= N || k0 >= K) continue;
        const Divisor div = by_group_scale(lift_tiny(v[j], s));
        uint4 o;
        o.x = pack_e4m3(div(v[j][0]), div(v[j][1]), div(v[j][2]), div(v[j][3]));
        o.y = pack_e4m3(div(v[j][4]), div(v[j][5]), div(v[j][6]), div(v[j][7]));
        o.z = pack_e4m3(div(v[j][8]), div(v[j][9]), div(v[j][10]), div(v[j][11]));
        o.w = pack_e4m3(div(v[j][12]), div(v[j][13]), div(v[j][14]), div(v[j][15]));
        *reinterpret_cast<uint4*>(w8 + (int64_t)n * K + k0) = o;
    }
    if (threadIdx.x == 0) scale[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

hipError_t launch_quantize_weight(const bf16_t* w, int N, int K, uint8_t* w8, float* w_scale, hipStream_t s)
{
    const dim3 grid(ceil_div(K, kScaleGroup), ceil_div(N, kScaleGroup));
    hipLaunchKernelGGL(quantize_weight_kernel, grid, dim3(256), 0, s, w, N, K, w8, w_scale);
    return hipGetLastError();
}

}  // namespace bmoe
