// What the 8-bit kernels share: e4m3 codes and their scales.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace quant {

constexpr int GROUP = 128;                     // columns that share a scale
constexpr float E4M3_MAX = 448.f;
constexpr float SCALE_MIN = 1.17549435e-38f;   // 2^-126: a group of zeros (or of subnormals) still has a normal scale

#ifdef __CUDACC__

// Magnitudes are compared by their bits: |v| of finite values, then infinity, then NaN, so that the largest of a group
// with a NaN in it is a NaN.
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
    const float s = __uint_as_float(amax_bits) / E4M3_MAX;
    return s < SCALE_MIN ? SCALE_MIN : s;      // a NaN stays one
}

// v / s for the codes of a group.  The quotient has to be the correctly rounded one: a product with 1 / s would put
// quotients that lie on a rounding border of e4m3 (common: bf16 values are ratios of small integers) on either side of
// it.  One correction of v * (1 / s) by its remainder, which an fma gives without rounding, is the correctly rounded quotient
// if 1 / s is (Markstein, 1990) as long as nothing leaves the range of fp32: the remainder is a multiple of about 2^-46 v.
// With s >= 2^-60 it can leave it only where the quotient is below 2^-40 and its code 0; scales below that, infinite
// and NaN ones take the division itself.  (512 x 12288 gated values: 11.2 us with the divisions, 7.8 with this.)
struct Divisor {
    float s, r;
    bool plain;
    __device__ __forceinline__ explicit Divisor(float scale) : s(scale), r(1.f / scale), plain(scale >= 8.6736174e-19f && scale <= 3.4028235e38f) {}
    __device__ __forceinline__ float quotient(float v) const {
        const float q = v * r;
        return fmaf(fmaf(-q, s, v), r, q);
    }
};
// Four values as codes; a quotient is at most 448 (1 + 2^-23), which rounds to 448.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
__device__ __forceinline__ uint2 codes8(const float (&f)[8], const Divisor& by) {
    float q[8];
    if (by.plain) {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = by.quotient(f[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = f[j] / by.s;
    }
    return make_uint2(codes4(q[0], q[1], q[2], q[3]), codes4(q[4], q[5], q[6], q[7]));
}

__device__ __forceinline__ void unpack_bf16x8(const uint4& v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = __uint_as_float(w[j] << 16);
        f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load_bf16x16(const __nv_bfloat16* p, float (&f)[16]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p), b = *reinterpret_cast<const uint4*>(p + 8);
    unpack_bf16x8(a, f);
    unpack_bf16x8(b, f + 8);
}
__device__ __forceinline__ uint32_t amax16(const float (&f)[16]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) m = max(m, mag_bits(f[j]));
    return m;
}
__device__ __forceinline__ uint32_t amax8(const float (&f)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, mag_bits(f[j]));
    return m;
}
// Largest of eight neighbouring lanes.
__device__ __forceinline__ uint32_t max8(uint32_t m) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}
// Largest of the sixteen neighbouring lanes that hold a group of 128 columns, 8 each.
__device__ __forceinline__ uint32_t max_of_16(uint32_t m) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

#endif  // __CUDACC__

}  // namespace quant
