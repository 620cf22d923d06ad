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
// The bits of the largest |value| of a vector that LPV lanes hold, N words of two values each: found among the 16-bit patterns
// themselves, two at a time; without their signs they are in order, and infinities and NaN come last.
template <typename T, int LPV, int N>
__device__ __forceinline__ uint32_t largest_bits(const uint32_t* y) {
    constexpr uint32_t ABS = 0x7fff7fffu;
    uint32_t top = y[0] & ABS;
#pragma unroll
    for (int j = 1; j < N; ++j) top = __vmaxu2(top, y[j] & ABS);
#pragma unroll
    for (int o = 1; o < LPV; o <<= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float2 f = unpack2<T>(top);
    return max(__float_as_uint(f.x), __float_as_uint(f.y));
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long&>(d))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return d;
}
// Four codes of x 2^-e; what they are with NAN_EXP's inv = 0 does not matter (the caller writes zeros).  i8: added to 1.5 2^23, a value is
// rounded to a whole number, to the nearest, ties to even, and its last byte is the code.
template <int HELD>
__device__ __forceinline__ uint32_t hold4(float2 a, float2 b, float inv) {
    const float2 i2 = make_float2(inv, inv);
    if (HELD == HELD_E4M3) {
        const float2 x = mul2(a, i2), y = mul2(b, i2);
        uint32_t c;
        asm("{\n\t.reg .b16 lo, hi;\n\t"
            "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
            "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
            "mov.b32 %0, {lo, hi};\n\t}"
            : "=r"(c)
            : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
        return c;
    }
    const float2 magic = make_float2(12582912.f, 12582912.f);
    const float2 x = fma2(a, i2, magic), y = fma2(b, i2, magic);
    return __byte_perm(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x0040), __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x0040), 0x5410);
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

template <typename T> __host__ __device__ constexpr bool is_half() { return false; }
template <> __host__ __device__ constexpr bool is_half<__half>() { return true; }

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

// The same by 16-bit arithmetic, two values at a time: an e4m3 code's exponent and mantissa, moved to a bf16's or f16's places, stand
// for 2^-120 or 2^-8 of its value, denormal codes included; an i8 code is the f16 1152 + code, less 1152, or as a bf16 its lower seven bits
// on 128, less 128 or, with its top bit, 256.  Then one exact product with the power of two, while that product and its factor are
// normal values of the type; the rest goes through fp32.
template <typename T, int HELD>
struct FastScale {
    static constexpr int CODE = HELD == HELD_I8 ? 0 : is_half<T>() ? 8 : 120;             // log2 of value / pattern
    static constexpr int LOW = is_half<T>() ? -14 - CODE : MIN_EXP;
    static constexpr int HIGH = is_half<T>() ? (HELD == HELD_I8 ? 9 : 7) : HELD == HELD_I8 ? 120 : 7;
};
template <typename T>
__device__ __forceinline__ uint32_t mul16x2(uint32_t a, uint32_t b);
template <>
__device__ __forceinline__ uint32_t mul16x2<__nv_bfloat16>(uint32_t a, uint32_t b) {
    const __nv_bfloat162 c = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&c);
}
template <>
__device__ __forceinline__ uint32_t mul16x2<__half>(uint32_t a, uint32_t b) {
    const __half2 c = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&c);
}
template <typename T, int HELD>
__device__ __forceinline__ uint32_t pattern2(uint32_t c, uint32_t pick) {
    if (HELD == HELD_E4M3) {
        constexpr int SHIFT = is_half<T>() ? 1 : 4;
        const uint32_t w = __byte_perm(c, 0, pick & 0xf0f0u | 0x0404u);                   // the two codes as upper bytes
        return (w & 0x80008000u) | ((w & 0x7f007f00u) >> SHIFT);
    }
    if (is_half<T>()) {
        const uint32_t w = __byte_perm(c ^ 0x80808080u, 0x64646464u, pick >> 4 & 0x0f0fu | 0x4040u);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&w), __half2half2(__ushort_as_half(0x6480)));
        return *reinterpret_cast<const uint32_t*>(&x);
    }
    const uint32_t w = __byte_perm(c, 0x43434343u, pick >> 4 & 0x0f0fu | 0x4040u), a = w & 0xff7fff7fu, b = w & 0xff80ff80u;
    const __nv_bfloat162 x = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&x);
}
template <typename T, int HELD>
__device__ __forceinline__ bool fast_scale(int e, uint32_t* scale2) {
    using F = FastScale<T, HELD>;
    const int x = max(F::LOW, min(F::HIGH, e)) + F::CODE;
    const uint32_t one = is_half<T>() ? uint32_t(x + 15) << 10 : uint32_t(x + 127) << 7;
    *scale2 = one | one << 16;
    return e >= F::LOW && e <= F::HIGH;
}
template <typename T, int HELD>
__device__ __forceinline__ void fast_values16(const uint4& c, uint32_t scale2, uint32_t* out) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        out[2 * i] = mul16x2<T>(pattern2<T, HELD>(w[i], 0x1000u), scale2);                // codes 0 and 1 of the word
        out[2 * i + 1] = mul16x2<T>(pattern2<T, HELD>(w[i], 0x3020u), scale2);            // 2 and 3
    }
}

template <typename T, int HELD>
__device__ __forceinline__ void any_values16(const uint4& c, int e, uint32_t* out) {
    uint32_t scale2;
    if (fast_scale<T, HELD>(e, &scale2)) fast_values16<T, HELD>(c, scale2, out); else values16<T, HELD>(c, exponent_scale(e), out);
}

}  // namespace disc
