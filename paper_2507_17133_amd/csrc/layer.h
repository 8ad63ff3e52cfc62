// Internal declarations of the operators around the MoE layer (norm.hip, rope.hip, attention.hip, linear8.hip, layer_api.hip).
#pragma once
#include "../../include/brownout_layer.h"
#include "internal.h"

namespace bmoe {

moe_status hip_fail(hipError_t e, const char* where);      // api.hip: keeps the error's text for moe_last_hip_error

constexpr int kScaleGroup = 128;                  // columns (and, of a weight, rows) under one e4m3 scale
constexpr float kE4m3Max = 448.0f;
constexpr float kLeastMagnitude = 7.888609052210118e-31f;  // 2^-100: keeps 448 / magnitude finite

// Four floats -> four e4m3 in one 32-bit word, first value in the low byte.  Values within +-448 only (or NaN).
__device__ __forceinline__ unsigned pack_e4m3(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// y / s to the last bit for the price of three multiplications: the product with the rounded 1 / s, corrected by its own remainder.  (Every pair of bf16
// significands, of the value and of a group's largest, gives what the division gives; the product alone takes about one code in 1400 to its
// neighbour.  The division itself: norm of 16384 x 7168 136 -> 145 us, its rows alone 63 -> 70, weight of 7168 x 7168 28 -> 34; this way 137, 63, 28.)
// An infinite s leaves y * 0; where y / s is beyond fp32's range the result is NaN.
struct Divisor {
    float s, k;
    __device__ __forceinline__ Divisor(float finite, float reciprocal) : s(finite), k(reciprocal) {}
    __device__ __forceinline__ explicit Divisor(float by) : s(by < __builtin_inff() ? by : 0.0f), k(1.0f / by) {}
    __device__ __forceinline__ float near(float y) const { return y * k; }                       // within 2 ulp
    __device__ __forceinline__ float exact(float y, float q) const { return __builtin_fmaf(-__builtin_fmaf(q, s, -y), k, q); }     // in this order -0 stays -0
    __device__ __forceinline__ float operator()(float y) const { return exact(y, near(y)); }
};

// Takes the values of a group of tiny scale, and the scale that it returns, out of the way of subnormal remainders.
template <int N>
__device__ __forceinline__ float lift_tiny(float (&v)[N], float s)
{
    if (fabsf(s) >= 5.421010862427522e-20f || s != s) return s;           // 2^-64
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] *= 1.8446744073709552e19f;           // 2^64
    return s * 1.8446744073709552e19f;
}

// Eight bf16 of one 16-byte load as floats.
__device__ __forceinline__ void unpack_bf16(const uint4 w, float* f)
{
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack_bf16x8(const float* f)
{
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}

// 16 bytes past the caches where ONCE: what is read once, or written for a reader who comes too late to find it there.
constexpr int64_t kCachedBytes = (int64_t)8 << 20;        // a result of more is not kept: an XCD's L2 holds 4 MiB
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
template <bool ONCE>
__device__ __forceinline__ uint4 load16(const bf16_t* q)
{
    const u32x4* s = reinterpret_cast<const u32x4*>(q);
    return __builtin_bit_cast(uint4, ONCE ? __builtin_nontemporal_load(s) : *s);
}
template <bool ONCE>
__device__ __forceinline__ void store16(bf16_t* q, uint4 v)
{
    u32x4* d = reinterpret_cast<u32x4*>(q);
    if (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), d);
    else *d = __builtin_bit_cast(u32x4, v);
}

hipError_t launch_norm(const moe_norm_args& a, bool norm, hipStream_t s);
hipError_t launch_quantize_weight(const bf16_t* w, int N, int K, uint8_t* w8, float* w_scale, hipStream_t s);

hipError_t launch_rope(const moe_kv_cache& c, const moe_block_table& t, const moe_rope& r, const bf16_t* q, int64_t q_stride,
                       const bf16_t* k, int64_t k_stride, const bf16_t* v, int64_t v_stride, int n_heads, int T,
                       const int32_t* positions, const int32_t* places, bf16_t* q_out, int64_t q_out_stride, hipStream_t s);

hipError_t init_attention_kernels();
size_t attention_workspace_bytes(const moe_kv_cache& c, int T, int n_heads);
hipError_t launch_attention(const moe_kv_cache& c, const moe_block_table& t, const bf16_t* q, int64_t q_stride, int n_heads, int T,
                            const int32_t* lengths, float scale, int window, int sinks, bf16_t* out, int64_t out_stride, float* lse, void* ws,
                            hipStream_t s);

hipError_t init_linear_kernels();
// How a product is cut (linear8.hip).
struct LinearPlan {
    int way, ksplit, rows, columns;               // rows, columns: of the rows kernel's blocks
    int first_way, first_rows;                    // rows that go ahead in tiles of their own (0: none)
    bool wide;                                    // operands widened to bf16
};
LinearPlan linear_plan(int M, int N, int K, bool exact);
size_t linear_workspace_bytes(const LinearPlan& plan, int M, int N);
size_t linear_workspace_bound(int M_max, int N, int K);
hipError_t launch_linear(const moe_linear_args& a, const LinearPlan& plan, void* ws, hipStream_t s);

}  // namespace bmoe
