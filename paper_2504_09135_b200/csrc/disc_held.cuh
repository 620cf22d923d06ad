// Vectors held in 8 bits: one code per value and a power of two 2^e for the vector.
//
//   e4m3   e = floor(log2 amax) - 8, one more where amax 2^-e > 448 (the largest code)
//   i8     e = floor(log2 amax) - 6, one more where amax 2^-e rounds to more than 127
//   code = x 2^-e rounded to the nearest, ties to even;  e is at least -126
//
// With a power of two nothing but the code is rounded: x 2^-e and code 2^e are exact, and every way to compute them agrees bit for
// bit.  A vector with a value that is not finite has e = NAN_EXP, codes 0, and reads as NaN.
#pragma once

#include <cuda_fp8.h>

#include "disc_sm100.cuh"

namespace disc {

constexpr int NAN_EXP = -128;
constexpr int MIN_EXP = -126;

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }      // -126 <= e <= 127

// the exponent of a vector from the bits of the largest |x|; *inv gets 2^-e (0 with NAN_EXP)
template <int HELD>
__device__ __forceinline__ int hold_exponent(uint32_t amax_bits, float* inv) {
    if (amax_bits >= 0x7f800000u) { *inv = 0.f; return NAN_EXP; }
    const float amax = __uint_as_float(amax_bits);
    int e = max(MIN_EXP, int(amax_bits >> 23) - 127 - (HELD == HELD_E4M3 ? 8 : 6));
    const float top = amax * pow2f(-e);
    if (HELD == HELD_E4M3 ? top > 448.f : rintf(top) > 127.f) ++e;
    *inv = pow2f(-e);
    return e;
}
// four codes; x with NAN_EXP's inv = 0 may be anything
template <int HELD>
__device__ __forceinline__ uint32_t hold4(const float* x, float inv) {
    if (inv == 0.f) return 0;
    if (HELD == HELD_E4M3) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[0] * inv, x[1] * inv), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[2] * inv, x[3] * inv), __NV_SATFINITE, __NV_E4M3);
        return lo | hi << 16;
    }
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) c |= (uint32_t(__float2int_rn(x[i] * inv)) & 255u) << (8 * i);
    return c;
}

// the values of four codes, without the power of two, in fp32
template <int HELD>
__device__ __forceinline__ void codes4(uint32_t c, float* x) {
    if (HELD == HELD_E4M3) {
        const __half2 lo(__nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(c & 0xffffu), __NV_E4M3)), hi(__nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(c >> 16), __NV_E4M3));
        const float2 a = __half22float2(lo), b = __half22float2(hi);
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = float(int32_t(c << (24 - 8 * i)) >> 24);
    }
}
__device__ __forceinline__ float exponent_scale(int e) { return e == NAN_EXP ? CUDART_NAN_F : pow2f(max(e, MIN_EXP)); }

template <typename T> __device__ __forceinline__ constexpr bool is_half() { return false; }
template <> __device__ __forceinline__ constexpr bool is_half<__half>() { return true; }

// the largest finite value of a type, beyond which held values are cut off when they are given back in it (an e4m3 code can
// round the largest 4 % of a type's range up to the next power of two)
template <typename T> __device__ __forceinline__ float largest();
template <> __device__ __forceinline__ float largest<__nv_bfloat16>() { return __uint_as_float(0x7f7f0000u); }
template <> __device__ __forceinline__ float largest<__half>() { return 65504.f; }

// sixteen values of a vector in type T from their codes
template <typename T, int HELD>
__device__ __forceinline__ void values16(const uint4& c, float scale, uint32_t* out) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    const float top = largest<T>();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x[4];
        codes4<HELD>(w[i], x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] *= scale;
            x[j] = x[j] > top ? top : (x[j] < -top ? -top : x[j]);          // NaN stays NaN
        }
        out[2 * i] = pack2<T>(x[0], x[1]);
        out[2 * i + 1] = pack2<T>(x[2], x[3]);
    }
}

}  // namespace disc
