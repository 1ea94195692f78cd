// What the 8-bit kernels share: e4m3 codes and their scales.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "sm100.cuh"

namespace quant {

constexpr int GROUP = 128;                     // columns that share a scale
constexpr float E4M3_MAX = 448.f;
constexpr float SCALE_MIN = 1.17549435e-38f;   // 2^-126: a group of zeros (or of subnormals) still has a normal scale

#ifdef __CUDACC__

// A magnitude by its bits: |v| of finite values, then infinity, then NaN.
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ float scale_of(float amax) {
    const float s = amax / E4M3_MAX;
    return s < SCALE_MIN ? SCALE_MIN : s;      // a NaN stays one
}

// v / s for the codes of a group.  The quotient has to be the correctly rounded one: a product with 1 / s would put
// quotients that lie on a rounding border of e4m3 (common: bf16 values are ratios of small integers) on either side of
// it.  One correction of v * (1 / s) by its remainder, which an fma gives without rounding, is the correctly rounded quotient
// if 1 / s is (Markstein, 1990) as long as nothing leaves the range of fp32: the remainder is a multiple of about 2^-46 v.
// With s >= 2^-60 it can leave it only where the quotient is below 2^-40 and its code 0; scales below that, infinite
// and NaN ones take the division itself.  (With the pairs below, 2048 x 4096 normalised rows:
// 14.9 us with divisions, one value at a time, 11.6 like this.)
struct Divisor {
    float s;
    uint64_t r2, ns2;                          // 1 / s and -s, for two values at a time
    bool plain;
    __device__ __forceinline__ explicit Divisor(float scale) : s(scale), plain(scale >= 8.6736174e-19f && scale <= 3.4028235e38f) {
        const float r = 1.f / scale;
        r2 = sm100::pack_f32x2(r, r);
        ns2 = sm100::pack_f32x2(-scale, -scale);
    }
    __device__ __forceinline__ uint64_t quotients(uint64_t v) const {
        const uint64_t q = sm100::mul2(v, r2);
        return sm100::fma2(sm100::fma2(q, ns2, v), r2, q);
    }
};

// The row kernels are bound by the instructions they issue, so eight values are four pairs, two to an instruction.
struct V8 {
    uint64_t p[4];
};
__device__ __forceinline__ V8 unpack8(const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    V8 x;
#pragma unroll
    for (int j = 0; j < 4; ++j) x.p[j] = sm100::pack_f32x2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    return x;
}
__device__ __forceinline__ uint4 to_bf16(const V8& x) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a, b;
        sm100::unpack_f32x2(x.p[j], a, b);
        w[j] = pack_bf16(a, b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The largest of three magnitudes; a NaN if one of them is.
__device__ __forceinline__ float max_mag(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max_mag(const V8& x, float m = 0.f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a, b;
        sm100::unpack_f32x2(x.p[j], a, b);
        m = max_mag(m, a, b);
    }
    return m;
}
// Largest of N neighbouring lanes' magnitudes.
template <int N>
__device__ __forceinline__ float max_mag_of(float m) {
#pragma unroll
    for (int o = 1; o < N; o <<= 1) m = max_mag(m, __shfl_xor_sync(0xffffffffu, m, o), 0.f);
    return m;
}

// Four values as codes; a quotient is at most 448 (1 + 2^-23), which rounds to 448.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
__device__ __forceinline__ uint2 codes8(const V8& x, const Divisor& by) {
    float q[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (by.plain) {
            sm100::unpack_f32x2(by.quotients(x.p[j]), q[2 * j], q[2 * j + 1]);
        } else {
            float a, b;
            sm100::unpack_f32x2(x.p[j], a, b);
            q[2 * j] = a / by.s;
            q[2 * j + 1] = b / by.s;
        }
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
// Largest of eight neighbouring lanes.
__device__ __forceinline__ uint32_t max8(uint32_t m) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

#endif  // __CUDACC__

}  // namespace quant
