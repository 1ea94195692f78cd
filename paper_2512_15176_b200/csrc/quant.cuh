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

// Four values as codes.  v / s is at most 448 (1 + 2^-23), which rounds to 448; the division is the IEEE one, because a
// multiplication by 1 / s would put quotients that lie on a rounding border (common: bf16 values are ratios of small
// integers) on either side of it.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float s) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a / s, b / s), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c / s, d / s), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
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
__device__ __forceinline__ uint4 codes16(const float (&f)[16], float s) {
    return make_uint4(codes4(f[0], f[1], f[2], f[3], s), codes4(f[4], f[5], f[6], f[7], s), codes4(f[8], f[9], f[10], f[11], s),
                      codes4(f[12], f[13], f[14], f[15], s));
}
// Largest of the eight neighbouring lanes that hold a group of 128 columns, 16 each.
__device__ __forceinline__ uint32_t max8(uint32_t m) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

#endif  // __CUDACC__

}  // namespace quant
