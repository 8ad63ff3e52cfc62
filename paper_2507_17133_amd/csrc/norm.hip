// Root-mean-square norm with the residual's addition and an 8-bit output, the 8-bit output alone, and the 8-bit form of a weight.
//
//   h = x + r      y = h * rsqrt(mean(h^2) + eps) * w      per group of 128 columns: s = max(amax|y|, 2^-100) / 448, y8 = e4m3(y / s)
//
// One pass: a row's vectors stay in the registers of the threads that share it between the sum of squares and the outputs, so every
// input is read once and every output written once: HBM bound.
#include "layer.h"

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

__device__ __forceinline__ float group_magnitude(unsigned bits) { return __uint_as_float(max(bits, __float_as_uint(kLeastMagnitude))); }

// THREADS threads share a row, NV vectors of 8 columns each: vector v of thread i is columns 8 (v THREADS + i) .., so 16 neighbouring
// lanes hold one group of 128 columns.  256 threads: four rows' worth of waves per block where rows are short (THREADS = 64).
template <int THREADS, int NV, bool NORM>
__global__ void __launch_bounds__(256) norm_kernel(NormArgs p)
{
    constexpr int ROWS = 256 / THREADS, WAVES = THREADS / 64;
    const int lane_row = threadIdx.x / THREADS, i = threadIdx.x % THREADS;
    const int t = blockIdx.x * ROWS + lane_row;
    if (ROWS > 1 && t >= p.T) return;                     // whole waves, and no barrier then
    const bf16_t* xr = p.x + (int64_t)t * p.xs;
    float h[NV][8];
    float sum = 0.0f;
    uint4 xv[NV], rv[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = 8 * (v * THREADS + i);
        xv[v] = rv[v] = make_uint4(0, 0, 0, 0);
        if (c < p.d) {
            xv[v] = *reinterpret_cast<const uint4*>(xr + c);
            if (NORM && p.r) rv[v] = *reinterpret_cast<const uint4*>(p.r + (int64_t)t * p.rs + c);
        }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = 8 * (v * THREADS + i);
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
            if (p.ro && c < p.d) *reinterpret_cast<uint4*>(p.ro + (int64_t)t * p.ros + c) = pack_bf16x8(h[v]);
        }
    }
    if constexpr (NORM) {
#pragma unroll
        for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m);
        if constexpr (WAVES > 1) {
            __shared__ float part[WAVES];
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
            __syncthreads();
            sum = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) sum += part[k];
        }
        const float inv = 1.0f / sqrtf(sum / (float)p.d + p.eps);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = 8 * (v * THREADS + i);
            float w[8];
            if (p.w) {
                uint4 wv = make_uint4(0, 0, 0, 0);
                if (c < p.d) wv = *reinterpret_cast<const uint4*>(p.w + c);
                unpack_bf16(wv, w);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) h[v][e] *= p.w ? inv * w[e] : inv;
            if (p.y && c < p.d) *reinterpret_cast<uint4*>(p.y + (int64_t)t * p.ys + c) = pack_bf16x8(h[v]);
        }
    }
    if (!p.y8) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = 8 * (v * THREADS + i);
        unsigned bits = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) bits = max(bits, abs_bits(h[v][e]));
        if (c >= p.d) bits = 0;                           // 0 times an infinite 1 / rms is no member of the group
#pragma unroll
        for (int m = 8; m; m >>= 1) bits = max(bits, (unsigned)__shfl_xor((int)bits, m));
        const float mag = group_magnitude(bits), k = kE4m3Max / mag;
        if (c >= p.d) continue;
        uint2 o;
        o.x = pack_e4m3(h[v][0] * k, h[v][1] * k, h[v][2] * k, h[v][3] * k);
        o.y = pack_e4m3(h[v][4] * k, h[v][5] * k, h[v][6] * k, h[v][7] * k);
        *reinterpret_cast<uint2*>(p.y8 + (int64_t)t * p.y8s + c) = o;
        if ((c & (kScaleGroup - 1)) == 0) p.scale[(int64_t)(c / kScaleGroup) * p.ss + t] = mag / kE4m3Max;
    }
}

template <int THREADS, int NV>
static void norm_go(const NormArgs& p, bool norm, hipStream_t s)
{
    const int rows = 256 / THREADS, grid = ceil_div(p.T, rows);
    if (norm) hipLaunchKernelGGL((norm_kernel<THREADS, NV, true>), dim3(grid), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((norm_kernel<THREADS, NV, false>), dim3(grid), dim3(256), 0, s, p);
}

hipError_t launch_norm(const moe_norm_args& a, bool norm, hipStream_t s)
{
    NormArgs p{static_cast<const bf16_t*>(a.x), static_cast<const bf16_t*>(a.residual), static_cast<const bf16_t*>(a.weight),
               static_cast<bf16_t*>(a.residual_out), static_cast<bf16_t*>(a.y), static_cast<uint8_t*>(a.y8), a.scale,
               a.x_stride, a.residual_stride, a.residual_out_stride, a.y_stride, a.y8_stride, a.scale_stride, a.T, a.d, a.eps};
    if (a.d <= 512) norm_go<64, 1>(p, norm, s);
    else if (a.d <= 1024) norm_go<64, 2>(p, norm, s);
    else if (a.d <= 2048) norm_go<256, 1>(p, norm, s);
    else if (a.d <= 4096) norm_go<256, 2>(p, norm, s);
    else if (a.d <= 8192) norm_go<256, 4>(p, norm, s);
    else norm_go<256, 8>(p, norm, s);
    return hipGetLastError();
}

// One block per 128 x 128 block of the weight: 128 threads' worth of 16-column pieces of its rows stay in registers between the maximum
// and the store.
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
    const float mag = group_magnitude(bits), k = kE4m3Max / mag;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 32 * j;
        if (n >= N || k0 >= K) continue;
        uint4 o;
        o.x = pack_e4m3(v[j][0] * k, v[j][1] * k, v[j][2] * k, v[j][3] * k);
        o.y = pack_e4m3(v[j][4] * k, v[j][5] * k, v[j][6] * k, v[j][7] * k);
        o.z = pack_e4m3(v[j][8] * k, v[j][9] * k, v[j][10] * k, v[j][11] * k);
        o.w = pack_e4m3(v[j][12] * k, v[j][13] * k, v[j][14] * k, v[j][15] * k);
        *reinterpret_cast<uint4*>(w8 + (int64_t)n * K + k0) = o;
    }
    if (threadIdx.x == 0) scale[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = mag / kE4m3Max;
}

hipError_t launch_quantize_weight(const bf16_t* w, int N, int K, uint8_t* w8, float* w_scale, hipStream_t s)
{
    const dim3 grid(ceil_div(K, kScaleGroup), ceil_div(N, kScaleGroup));
    hipLaunchKernelGGL(quantize_weight_kernel, grid, dim3(256), 0, s, w, N, K, w8, w_scale);
    return hipGetLastError();
}

}  // namespace bmoe
