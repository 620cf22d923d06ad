// Attention of up to NT * 8 query vectors to a block of 16 tokens held in 8 bits, by one warp with mma.sync: what the kernels of
// disc_attend_held.cu and of disc_attend_group.cu's second step share.  The products and the reasons: disc_attend_held.cu.
#pragma once

#include "disc_attend.cuh"
#include "disc_held.cuh"

namespace disc {

// Probability times the values' power of two is at most 2^SLACK of its reference and goes into the products in f16, which ends above 2^15 and has
// steps of 2^-24 at its lower end.  So it gets this many powers of two more, of which the sums are rid at the end: what is lost of a small one
// is then 2^-32 of the reference, and not 2^-25, which 2^17 tokens of a warp, each of that probability beside a large one, made 0.0017 of 1.
constexpr float HEADROOM = 15.f - SLACK;

// shared memory of a block: keys [16][DP] | values [16][DP] | exponents of the keys [16] | of the values [16] | the user's, from HELD_SPARE on
constexpr int HELD_SPARE = 2 * BLK;
template <int DP>
__host__ __device__ constexpr int held_stage_bytes() { return 2 * BLK * DP + 128; }        // on 128-byte boundaries

// 16-byte chunk `ch` of token `row`: neighbouring tokens' chunks lie in different banks, so that ldmatrix reads eight of them at once
// without conflicts
template <int DP>
__device__ __forceinline__ uint32_t held_chunk_at(int row, int ch) {
    return DP == 128 ? uint32_t(row * 128 + ((ch ^ (row & 7)) << 4)) : uint32_t(row * 64 + ((ch ^ ((row >> 1) & 3)) << 4));
}

// Block `blk` of a page of which k and v are this head's parts; zeros beyond its tokens and its D values.  By a whole warp.  A block's codes
// are one run of bytes: where it is full and D is DP itself, lane l takes 16 of every 512 bytes.
template <int DP>
__device__ __forceinline__ void load_held_block(uint32_t stage, const unsigned char* k, const unsigned char* v, int blk, int tokens, int D, int page_size, int lane) {
    constexpr int CH = DP / 16;
    const int at = blk * BLK * D;
    const uint32_t to = stage + held_chunk_at<DP>(lane / CH, lane % CH);
    if (tokens == BLK && D == DP) {
        const unsigned char *ks = k + at + lane * 16, *vs = v + at + lane * 16;
#pragma unroll
        for (int j = 0; j < BLK * CH / 32; ++j) {
            const uint32_t dst = (to ^ (DP == 128 ? uint32_t(j & 1) << 6 : 0u)) + j * 512;        // four tokens on, the banks' turn is 4 further
            cp16(dst, ks + j * 512, true);
            cp16(dst + BLK * DP, vs + j * 512, true);
        }
    } else {
#pragma unroll
        for (int j = 0; j < BLK * CH / 32; ++j) {
            const int row = (j * 32 + lane) / CH, ch = lane % CH;
            const bool some = row < tokens && ch * 16 < D;
            const int src = some ? at + row * D + ch * 16 : 0;
            const uint32_t dst = (to ^ (DP == 128 ? uint32_t(j & 1) << 6 : 0u)) + j * 512;
            cp16(dst, k + src, some);
            cp16(dst + BLK * DP, v + src, some);
        }
    }
    if (lane < 2) cp16(stage + 2 * BLK * DP + lane * BLK, (lane ? v : k) + page_size * D + blk * BLK, true);
}

// Codes as f16, exactly.  e4m3: the conversion instruction takes two neighbouring codes, 49 of them a clock and SM (with shifts and masks
// it is seven operations for four codes).  i8: a code, its top bit turned over, is the last byte of the f16
// 1024 + 128 + code; that gives codes 0 and 2, and 1 and 3.
__device__ __forceinline__ uint32_t e4m3_f16(uint32_t two) {
    uint32_t x;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(x) : "r"(two));
    return x;
}
__device__ __forceinline__ uint32_t e4m3_f16_upper(uint32_t two) {
    uint32_t x;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(x) : "r"(two));
    return x;
}
__device__ __forceinline__ void i8_f16(uint32_t c, uint32_t& even, uint32_t& odd) {
    const __half2 bias = __half2half2(__ushort_as_half(0x6480));               // 1152
    const uint32_t a = (c & 0x00ff00ffu) ^ 0x64806480u, b = ((c >> 8) & 0x00ff00ffu) ^ 0x64806480u;
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), bias), y = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
    even = *reinterpret_cast<const uint32_t*>(&x);
    odd = *reinterpret_cast<const uint32_t*>(&y);
}
// Keys: four values of a token, in the order in which the queries lie too (held_dim).
template <int HELD>
__device__ __forceinline__ void key_codes(uint32_t c, uint32_t& first, uint32_t& second) {
    if (HELD == HELD_E4M3) {
        first = e4m3_f16(c);
        second = e4m3_f16_upper(c);
    } else {
        i8_f16(c, first, second);
    }
}
template <int HELD>
__device__ __forceinline__ constexpr int held_dim(int i) { return HELD == HELD_E4M3 || i == 0 || i == 3 ? i : 3 - i; }       // 0 1 2 3, or 0 2 1 3
// Values: two neighbouring dims of two tokens -> both tokens' first dim, both tokens' second.
template <int HELD>
__device__ __forceinline__ void value_codes(uint32_t c, uint32_t& first, uint32_t& second) {
    if (HELD == HELD_E4M3) {
        const uint32_t a = e4m3_f16(c), b = e4m3_f16_upper(c);
        first = __byte_perm(a, b, 0x5410);
        second = __byte_perm(a, b, 0x7632);
    } else {
        i8_f16(c, first, second);
    }
}

template <int DP, int NT>
struct HeldQueries {
    uint32_t f[NT][DP / 16][2];        // vector lane / 4; values 16 kk + 4 (lane % 4) + held_dim(0, 1) and (2, 3)
    float c2[NT][2];                   // what a score of this thread's vectors, 2 (lane % 4) and the next, is multiplied with: units of log2
};
// q: this lane's vector (lane / 4 of the eight), `some`: there is one
template <typename T, int DP, int HELD, int NT>
__device__ __forceinline__ void load_held_queries(HeldQueries<DP, NT>& qs, int nt, const unsigned char* q, bool some, int D, float c2, int lane) {
    float x[DP / 16][4];
    uint32_t amax = 0;
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk) {
        uint2 w = make_uint2(0, 0);
        if (some && kk * 16 < D) w = *reinterpret_cast<const uint2*>(q + kk * 32 + (lane & 3) * 8);
        const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y);
        x[kk][0] = a.x; x[kk][1] = a.y; x[kk][2] = b.x; x[kk][3] = b.y;
#pragma unroll
        for (int i = 0; i < 4; ++i) amax = max(amax, __float_as_uint(x[kk][i]) & 0x7fffffffu);
    }
    int up = 0;                        // what the vector is multiplied with, as a power of two
    if (!is_half<T>()) {
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        if (amax > 0 && amax < 0x7f800000u) up = 8 - max(int(amax >> 23) - 127, -110);
    }
    const float f = pow2f(up);
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk) {
        qs.f[nt][kk][0] = pack2<__half>(x[kk][held_dim<HELD>(0)] * f, x[kk][held_dim<HELD>(1)] * f);
        qs.f[nt][kk][1] = pack2<__half>(x[kk][held_dim<HELD>(2)] * f, x[kk][held_dim<HELD>(3)] * f);
    }
    const float back = c2 * pow2f(-up);
    qs.c2[nt][0] = __shfl_sync(0xffffffffu, back, (lane & 3) * 8);
    qs.c2[nt][1] = __shfl_sync(0xffffffffu, back, (lane & 3) * 8 + 4);
}

template <int DP, int NT>
struct HeldSums {                      // this thread's vectors: 2 (lane % 4) and the next of each eight
    float o[NT][DP / 16][4];           // dims 16 j + 2 (lane / 4) of the two vectors, then the next dim of both, times 2^-t
    float m[NT][2], l[NT][2];          // reference and sum of the probabilities
    float t[NT][2];                    // reference of probability times the values' power of two; from finish_held on what o is times 2^-t of
};
template <int DP, int NT>
__device__ __forceinline__ void clear_held(HeldSums<DP, NT>& a) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < DP / 16; ++j) a.o[nt][j][0] = a.o[nt][j][1] = a.o[nt][j][2] = a.o[nt][j][3] = 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) { a.m[nt][e] = a.t[nt][e] = -CUDART_INF_F; a.l[nt][e] = 0.f; }
    }
}
template <int DP, int NT>
__device__ __forceinline__ void finish_held(HeldSums<DP, NT>& a) {
#pragma unroll
    for (int x = 4; x < 32; x <<= 1)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) a.l[nt][e] += __shfl_xor_sync(0xffffffffu, a.l[nt][e], x);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) a.t[nt][e] -= HEADROOM;
}

// A block of some tokens, at least one; in[nt][e]: they are seen by this thread's vectors.  Probabilities are rounded to f16 for the second
// product; where T is f16 what that leaves out goes through a second one, so that the outputs' own rounding stays the larger.  (Two
// blocks at a time, for more independent instructions, made no difference.)
template <typename T, int DP, int HELD, int NT>
__device__ __forceinline__ void add_held_block(HeldSums<DP, NT>& acc, const HeldQueries<DP, NT>& qs, uint32_t stage, int tokens, const bool (&in)[NT][2], int lane) {
    constexpr bool TWO = is_half<T>();
    // scores, and with the values' power of two; tokens lane / 4 ([0], [1]) and 8 further ([2], [3])
    float s[NT][4], w[NT][4];
    float s2[NT][4];               // two chains of products
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[nt][i] = s2[nt][i] = 0.f;
#pragma unroll
    for (int c = 0; c < DP / 32; ++c) {
        uint32_t kf[4], x[4], y[4];
        // matrices: tokens 0-7 and 8-15 at chunk 2 c, then at chunk 2 c + 1
        ldsm4((stage + held_chunk_at<DP>(lane & 15, lane >> 4)) ^ uint32_t(c << 5), kf);
        key_codes<HELD>(kf[0], x[0], x[2]);
        key_codes<HELD>(kf[1], x[1], x[3]);
        key_codes<HELD>(kf[2], y[0], y[2]);
        key_codes<HELD>(kf[3], y[1], y[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mma16<__half>(s[nt], x, qs.f[nt][2 * c][0], qs.f[nt][2 * c][1]);
            mma16<__half>(s2[nt], y, qs.f[nt][2 * c + 1][0], qs.f[nt][2 * c + 1][1]);
        }
    }
    const uint32_t exps = stage + 2 * BLK * DP + (lane >> 2);
    int e[4];                          // keys, values; token lane / 4, 8 further
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("ld.shared.s8 %0, [%1];" : "=r"(e[i]) : "r"(exps + i * 8) : "memory");
    const float k0 = exponent_scale(e[0]), k1 = exponent_scale(e[1]);
    const float v0 = e[2] == NAN_EXP ? CUDART_NAN_F : float(e[2]), v1 = e[3] == NAN_EXP ? CUDART_NAN_F : float(e[3]);
    const bool some0 = (lane >> 2) < tokens, some1 = (lane >> 2) + 8 < tokens;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float x = (s[nt][i] + s2[nt][i]) * (qs.c2[nt][i] * k0), y = (s[nt][2 + i] + s2[nt][2 + i]) * (qs.c2[nt][i] * k1);
            const bool p = some0 && in[nt][i], q = some1 && in[nt][i];
            s[nt][i] = p ? x : -CUDART_INF_F;
            s[nt][2 + i] = q ? y : -CUDART_INF_F;
            w[nt][i] = p ? x + v0 : -CUDART_INF_F;
            w[nt][2 + i] = q ? y + v1 : -CUDART_INF_F;
        }
    bool move = false;
    float ms[NT][2], mw[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            ms[nt][i] = fmaxf(s[nt][i], s[nt][2 + i]);
            mw[nt][i] = fmaxf(w[nt][i], w[nt][2 + i]);
            move = move || ms[nt][i] > acc.m[nt][i] + SLACK || mw[nt][i] > acc.t[nt][i] + SLACK;
        }
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float a = fmaxf(acc.m[nt][i], ms[nt][i]), t = fmaxf(acc.t[nt][i], mw[nt][i]);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, x));
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
                }
                // sums without a finite reference so far are 0, or NaN
                if (acc.m[nt][i] > -CUDART_INF_F) acc.l[nt][i] *= ex2_approx(acc.m[nt][i] - a);
                const float f = acc.t[nt][i] > -CUDART_INF_F ? ex2_approx(acc.t[nt][i] - t) : 1.f;
                acc.m[nt][i] = a;
                acc.t[nt][i] = t;
#pragma unroll
                for (int j = 0; j < DP / 16; ++j) { acc.o[nt][j][i] *= f; acc.o[nt][j][2 + i] *= f; }
            }
    }
    uint32_t p0[NT], p1[NT], r0[NT], r1[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const float m0 = acc.m[nt][0] > -CUDART_INF_F ? acc.m[nt][0] : 0.f, m1 = acc.m[nt][1] > -CUDART_INF_F ? acc.m[nt][1] : 0.f;
        const float t0 = acc.t[nt][0] > -CUDART_INF_F ? acc.t[nt][0] - HEADROOM : 0.f, t1 = acc.t[nt][1] > -CUDART_INF_F ? acc.t[nt][1] - HEADROOM : 0.f;
        acc.l[nt][0] += ex2_approx(s[nt][0] - m0) + ex2_approx(s[nt][2] - m0);
        acc.l[nt][1] += ex2_approx(s[nt][1] - m1) + ex2_approx(s[nt][3] - m1);
        const float x0 = ex2_approx(w[nt][0] - t0), x1 = ex2_approx(w[nt][1] - t1), x2 = ex2_approx(w[nt][2] - t0), x3 = ex2_approx(w[nt][3] - t1);
        const uint32_t p = pack2<__half>(x0, x1), q = pack2<__half>(x2, x3);
        p0[nt] = transposed(p);
        p1[nt] = transposed(q);
        if (TWO) {
            const float2 rp = unpack2<__half>(p), rq = unpack2<__half>(q);
            r0[nt] = transposed(pack2<__half>(x0 - rp.x, x1 - rp.y));
            r1[nt] = transposed(pack2<__half>(x2 - rq.x, x3 - rq.y));
        }
    }
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) {
        uint32_t vf[4], x[4], y[4];
        // matrices: tokens 0-7 at chunks 2 j and 2 j + 1, then tokens 8-15; each register two dims of two tokens
        ldsm4t((stage + BLK * DP + held_chunk_at<DP>((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1)) ^ uint32_t(j << 5), vf);
        value_codes<HELD>(vf[0], x[0], x[1]);
        value_codes<HELD>(vf[2], x[2], x[3]);
        value_codes<HELD>(vf[1], y[0], y[1]);
        value_codes<HELD>(vf[3], y[2], y[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mma16<__half>(acc.o[nt][2 * j], x, p0[nt], p1[nt]);
            mma16<__half>(acc.o[nt][2 * j + 1], y, p0[nt], p1[nt]);
            if (TWO) {
                mma16<__half>(acc.o[nt][2 * j], x, r0[nt], r1[nt]);
                mma16<__half>(acc.o[nt][2 * j + 1], y, r0[nt], r1[nt]);
            }
        }
    }
}

}  // namespace disc
