// disc_logprobs: per row of logits the log-sum-exp, the entropy of softmax(z / T), the log-probability
// of a given token and the `top` most probable tokens with theirs; disc_logprobs_grad: the gradient of
// the log-probabilities and entropies with respect to the logits.
//
// With y_v = z_v log2(e) / T and m = max y:   S = sum 2^(y-m),  U = sum (y-m) 2^(y-m),
//   lse = ln2 (m + log2 S)     H = ln2 (log2 S - U / S)     log p_t = (z_t - max z) / T - ln2 log2 S
// so that one pass with a running maximum gives all three.  In units of y - m both sums stay between
// 0 and the number of tokens, and neither H nor a log-probability loses anything to a large lse, which fp32 holds only to 2^-24 of
// its size (2e-3 for logits near 30 at T = 1/1000; log S altogether for rows masked with a finite value).
//
// The pass is bound by the bytes of the logits.  What it may spend per logit is little: at the
// measured copy rate 11 bf16 logits arrive per SM and clock, and an SM takes 2^x sixteen times and
// any instruction 128 times per clock.  Hence packed bf16 maxima and packed fp32 pairs (about 4.5 instructions
// per logit), one comparison with the running maximum per 32 logits, and next to nothing in the loop for the
// alternatives:
//
// The alternatives come from what the pass keeps anyway, the maxima of each thread's portions of the row
// (32 logits; noted in shared memory).  The k-th largest of the block's thread maxima (k distinct elements
// reach it) is at most the k-th largest element, so that only portions whose maximum reaches it can hold one
// of the k best: as a rule k and a few, and only they are looked at again.  (Looking at all of a thread's
// portions again instead read half of the row a second time from HBM: the rows being worked on do not
// fit in L2.)  What reaches the threshold is ranked by counting in the order (larger first, -0 = +0, lower
// id first, NaN last).  Should more reach it than the lists hold (rows of equal logits), or too few (rows of
// NaN), the block selects by histograms of the order keys over its slice: exact for every input.
//
// Measured on 4096 x 128256 bf16 (1.05 GB): 167 us without alternatives, 198 with 20; the measured copy rate would be 163.
// The special-function unit is busy 66 % of the time then, the issue slots 67 %.
//
// A row is taken by one block, or, when there are too few rows to fill the device, by a cluster of up to
// 8 blocks that join their sums and lists over distributed shared memory.

#include <cuda_bf16.h>
#include <math_constants.h>

#include "disc_sm100.cuh"

namespace {

using disc::add2;
using disc::cluster_rank;
using disc::cluster_sync_all;
using disc::ex2_approx;
using disc::fma2;

constexpr int NT = 256;               // threads per block
constexpr int NW = NT / 32;
constexpr int TOP_MAX = 64;
constexpr int SHORT_ROW = 1024;       // rows up to this long are held in a warp's registers
constexpr int LIST_CAP = 2048;
constexpr int HOT_CAP = 512;          // portions of the row that are looked at again
constexpr int SLOTS = 32;             // portions of a thread
constexpr unsigned FULL = 0xffffffffu;
constexpr float LOG2E_F = 1.4426950408889634f;
constexpr float LN2_F = 0.6931471805599453f;
// 2^y is zero in fp32 (flushed) below -126
constexpr float Y_MIN = -200.f;
// Logits below `low`, y = -10^6, are taken as that: (y-m) 2^(y-m) is then 0 for them, where it would be NaN for -inf.  (y
// has to stay where fp32 still resolves whole numbers, or y-m of the floor itself would be a large rounding error.)  A row whose
// largest logit is that far out, a mask of the type's lowest value everywhere, goes through a pass of its own.
constexpr float FAR_Y = 1.0e6f;

struct LogprobParams {
    const void* logits;
    int64_t ld;
    int32_t V, top, split;
    float inv_t, c2;                  // 1/T, log2(e)/T
    float low, low_y;                 // the floor of the logits, a bf16 value, and its y
    const int32_t* targets;           // nullable
    float* logp;                      // nullable
    float* entropy;                   // nullable
    float* lse;                       // nullable
    int32_t* top_ids;                 // [n][top]
    float* top_logp;                  // [n][top] (nullable)
    uint8_t* status;
};

// the larger of the two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0u;
    uint32_t b = __float_as_uint(x);
    if (b == 0x80000000u) b = 0u;
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
    if (k == 0u) return CUDART_NAN_F;
    return (k & 0x80000000u) ? __uint_as_float(k & 0x7fffffffu) : __uint_as_float(~k);
}
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}
// the same for memory that the kernel itself may write: a gradient over its own logits
__device__ __forceinline__ uint4 ld_stream_own(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}

template <int DT>
struct Vec;
template <>
struct Vec<DISC_BF16> {
    static constexpr int E = 8;
    static constexpr int SIZE = 2;
    static __device__ __forceinline__ uint4 lowest() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
    static __device__ __forceinline__ void unpack(const uint4& v, float* x) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
    }
    // the largest of U vectors' elements, NaN only if all are
    template <int U>
    static __device__ __forceinline__ float largest(const uint4* v) {
        __nv_bfloat162 a = *reinterpret_cast<const __nv_bfloat162*>(&v[0].x);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u) a = __hmax2(a, *reinterpret_cast<const __nv_bfloat162*>(&v[u].x));
            a = __hmax2(a, *reinterpret_cast<const __nv_bfloat162*>(&v[u].y));
            a = __hmax2(a, *reinterpret_cast<const __nv_bfloat162*>(&v[u].z));
            a = __hmax2(a, *reinterpret_cast<const __nv_bfloat162*>(&v[u].w));
        }
        const uint32_t w = *reinterpret_cast<const uint32_t*>(&a);
        return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    // every element at least `low`, NaN kept
    static __device__ __forceinline__ uint4 floor_at(uint4 v, float low) {
        const __nv_bfloat162 l = __float2bfloat162_rn(low);
        uint32_t* w = &v.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(w + j), l);
            w[j] = *reinterpret_cast<const uint32_t*>(&m);
        }
        return v;
    }
    // a maximum over elements in 16 bits
    using Short = unsigned short;
    static __device__ __forceinline__ Short shorten(float x) { return Short(__float_as_uint(x) >> 16); }
    static __device__ __forceinline__ float lengthen(Short x) { return __uint_as_float(uint32_t(x) << 16); }
    static __device__ __forceinline__ float at(const char* p) { return __uint_as_float(uint32_t(*reinterpret_cast<const unsigned short*>(p)) << 16); }
    static __device__ __forceinline__ void put(char* p, float x) { *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(x); }
    static __device__ __forceinline__ uint4 pack(const float* x) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&b);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Vec<DISC_F32> {
    static constexpr int E = 4;
    static constexpr int SIZE = 4;
    static __device__ __forceinline__ uint4 lowest() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
    static __device__ __forceinline__ void unpack(const uint4& v, float* x) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    template <int U>
    static __device__ __forceinline__ float largest(const uint4* v) {
        float a = __uint_as_float(v[0].x);
#pragma unroll
        for (int u = 0; u < U; ++u)
            a = fmaxf(fmaxf(a, __uint_as_float(v[u].x)), fmaxf(__uint_as_float(v[u].y), fmaxf(__uint_as_float(v[u].z), __uint_as_float(v[u].w))));
        return a;
    }
    static __device__ __forceinline__ uint4 floor_at(uint4 v, float low) {
        uint32_t* w = &v.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(max_nan(__uint_as_float(w[j]), low));
        return v;
    }
    using Short = float;
    static __device__ __forceinline__ Short shorten(float x) { return x; }
    static __device__ __forceinline__ float lengthen(Short x) { return x; }
    static __device__ __forceinline__ float at(const char* p) { return *reinterpret_cast<const float*>(p); }
    static __device__ __forceinline__ void put(char* p, float x) { *reinterpret_cast<float*>(p) = x; }
    static __device__ __forceinline__ uint4 pack(const float* x) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

// A row as elements before the first 16-byte boundary, whole vectors, and the elements after them.
template <int DT>
struct RowShape {
    const char* base;
    int32_t head, nvec, tail;
    __device__ __forceinline__ RowShape(const void* logits, int64_t ld, int64_t row, int32_t V) {
        constexpr int E = Vec<DT>::E, SIZE = Vec<DT>::SIZE;
        base = static_cast<const char*>(logits) + row * ld * SIZE;
        head = min(V, int32_t(((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15) / SIZE));
        nvec = (V - head) / E;
        tail = V - head - nvec * E;
    }
    __device__ __forceinline__ const uint4* vecs() const { return reinterpret_cast<const uint4*>(base + size_t(head) * Vec<DT>::SIZE); }
};

struct Sums {
    float m, ref, s, u;               // largest logit, its y; sums relative to ref
};
struct Scale {
    float c2, low_y;
};
__device__ __forceinline__ float reference(float m, Scale k) {
    return fabsf(m) < CUDART_INF_F ? fminf(fmaxf(m * k.c2, k.low_y), FAR_Y) : 0.f;
}
// the sums of a, relative to a's reference, seen from another one
__device__ __forceinline__ void raise(Sums& a, float m_new, Scale k) {
    const float ref = reference(m_new, k);
    const float d = a.m > -CUDART_INF_F ? fmaxf(a.ref - ref, Y_MIN) : Y_MIN;
    const float f = ex2_approx(d);
    a.u = f * fmaf(d, a.s, a.u);
    a.s *= f;
    a.m = m_new;
    a.ref = ref;
}
__device__ __forceinline__ Sums join(Sums a, Sums b, Scale k) {
    if (b.m > a.m) { const Sums t = a; a = b; b = t; }
    raise(b, a.m, k);
    a.s += b.s;
    a.u += b.u;
    return a;
}
// over the first N lanes of the warp (a power of two); called by all of them
template <int N>
__device__ __forceinline__ Sums join_lanes(Sums a, Scale k) {
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) {
        Sums b;
        b.m = __shfl_xor_sync(FULL, a.m, o);
        b.ref = __shfl_xor_sync(FULL, a.ref, o);
        b.s = __shfl_xor_sync(FULL, a.s, o);
        b.u = __shfl_xor_sync(FULL, a.u, o);
        a = join(a, b, k);
    }
    return a;
}
// a thread's running sums, even and odd elements apart
struct Running {
    float m, ref;
    float2 s, u;
};
__device__ __forceinline__ void raise(Running& a, float m_new, Scale k) {
    const float ref = reference(m_new, k);
    const float d = a.m > -CUDART_INF_F ? fmaxf(a.ref - ref, Y_MIN) : Y_MIN;
    const float f = ex2_approx(d);
    a.u = make_float2(f * fmaf(d, a.s.x, a.u.x), f * fmaf(d, a.s.y, a.u.y));
    a.s = make_float2(a.s.x * f, a.s.y * f);
    a.m = m_new;
    a.ref = ref;
}
__device__ __forceinline__ void add(Running& a, float2 x, float2 c2, float2 down) {
    const float2 d = fma2(x, c2, down);
    const float2 e = make_float2(ex2_approx(d.x), ex2_approx(d.y));
    a.s = add2(a.s, e);
    a.u = fma2(d, e, a.u);
}

// shared memory of a block; the other blocks of the cluster read `part`, `found` and `list`
struct Smem {
    unsigned long long list[LIST_CAP + 8];             // order key << 32 | ~id : larger = better
    unsigned long long best[TOP_MAX];
    uint32_t keys[NT];
    int32_t hot[HOT_CAP];                              // portion << 8 | thread
    unsigned int hist[256];
    Sums warp_sums[NW];
    Sums part, row;                                    // of the block; of the row, in a cluster's first block
    unsigned int n_hot, n_list, threshold, found;
    unsigned int prefix, remaining;
    int scan[NW];
};

template <int DT>
struct PortionMaxima {
    typename Vec<DT>::Short at[SLOTS][NT];
};

__device__ __forceinline__ unsigned long long entry(uint32_t key, int32_t id) {
    return (static_cast<unsigned long long>(key) << 32) | uint32_t(~id);
}

__device__ __forceinline__ uint32_t remote(const void* p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(uint32_t(__cvta_generic_to_shared(p))), "r"(rank));
    return a;
}
__device__ __forceinline__ uint32_t ld_remote32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long ld_remote64(uint32_t a) {
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}

// Of the cnt entries of sm.list the `want` best, in order, into sm.best.  Entries are distinct and not 0.  Called by the
// whole block.
__device__ __forceinline__ void rank_list(Smem& sm, unsigned int cnt, unsigned int want) {
    if (threadIdx.x < 8) sm.list[cnt + threadIdx.x] = 0ull;       // up to a whole number of eights
    __syncthreads();
    for (unsigned int i = threadIdx.x; i < cnt; i += NT) {
        const unsigned long long e = sm.list[i];
        unsigned int r = 0;
        for (unsigned int j = 0; j < cnt; j += 8) {
#pragma unroll
            for (int x = 0; x < 8; x += 2) {
                const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(&sm.list[j + x]);
                r += (two.x > e) + (two.y > e);
            }
        }
        if (r < want) sm.best[r] = e;
    }
    __syncthreads();
}

// The want-th largest (want <= NT) of the block's keys, its lower 16 bits cleared: found bit by bit by one warp.
__device__ __forceinline__ uint32_t kth_key(const uint32_t* keys, unsigned int want, int lane) {
    uint32_t k[NT / 32];
#pragma unroll
    for (int j = 0; j < NT / 32; ++j) k[j] = keys[j * 32 + lane];
    uint32_t found = 0u;
#pragma unroll 1
    for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
        const uint32_t t = found | bit;
        unsigned int n = 0;
#pragma unroll
        for (int j = 0; j < NT / 32; ++j) n += k[j] >= t;
        if (__reduce_add_sync(FULL, n) >= want) found = t;
    }
    return found;
}

// The `want` best of the elements [e0, e1) of a row by histograms of the order keys, eight bits at a
// time, and the lowest ids among the keys equal to the last one.  Called by the whole block.
template <int DT>
__device__ __noinline__ void select_slice(const char* base, int32_t e0, int32_t e1, unsigned int want, Smem& sm) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __syncthreads();
    if (tid == 0) { sm.prefix = 0u; sm.remaining = want; sm.n_list = 0u; }
    __syncthreads();
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int b = tid; b < 256; b += NT) sm.hist[b] = 0u;
        __syncthreads();
        const uint32_t prefix = sm.prefix;
        unsigned int bin = 256u, run = 0u;              // equal bins in a row are counted before they are added
        for (int32_t e = e0 + tid; e < e1; e += NT) {
            const uint32_t key = order_key(Vec<DT>::at(base + size_t(e) * Vec<DT>::SIZE));
            if (shift < 24 && (key >> (shift + 8)) != (prefix >> (shift + 8))) continue;
            const unsigned int b = (key >> shift) & 255u;
            if (b != bin) {
                if (run) atomicAdd(&sm.hist[bin], run);
                bin = b;
                run = 0u;
            }
            ++run;
        }
        if (run) atomicAdd(&sm.hist[bin], run);
        __syncthreads();
        if (tid == 0) {
            unsigned int left = sm.remaining;
            int b = 255;
            for (; b > 0; --b) {
                if (sm.hist[b] >= left) break;
                left -= sm.hist[b];
            }
            sm.prefix = prefix | (uint32_t(b) << shift);
            sm.remaining = left;
        }
        __syncthreads();
    }
    const uint32_t last = sm.prefix;
    const unsigned int ties = sm.remaining;
    for (int32_t e = e0 + tid; e < e1; e += NT) {       // fewer than `want` of them
        const uint32_t key = order_key(Vec<DT>::at(base + size_t(e) * Vec<DT>::SIZE));
        if (key > last) sm.list[atomicAdd(&sm.n_list, 1u)] = entry(key, e);
    }
    unsigned int taken = 0;
    for (int32_t b0 = e0; b0 < e1 && taken < ties; b0 += NT) {
        const int32_t e = b0 + tid;
        const bool eq = e < e1 && order_key(Vec<DT>::at(base + size_t(e) * Vec<DT>::SIZE)) == last;
        const unsigned ball = __ballot_sync(FULL, eq);
        if (lane == 0) sm.scan[warp] = __popc(ball);
        __syncthreads();
        unsigned int before = taken, all = 0;
        for (int w = 0; w < NW; ++w) {
            if (w < warp) before += sm.scan[w];
            all += sm.scan[w];
        }
        before += __popc(ball & ((1u << lane) - 1u));
        if (eq && before < ties) sm.list[atomicAdd(&sm.n_list, 1u)] = entry(last, e);
        taken += all;
        __syncthreads();
    }
    __syncthreads();
}

// ---- what a row's sums give -----------------------------------------------------------------------------
struct RowResult {
    float lse, entropy;
    float m, log_sum;                 // the largest logit; ln of the sum relative to it
    uint8_t status;
};
// far: t's sums are relative to its largest logit itself, not to the clamped and rounded reference
__device__ __forceinline__ RowResult row_result(const LogprobParams& p, const Sums& t, bool far) {
    if (t.s != t.s || t.u != t.u || t.m == CUDART_INF_F)
        return {t.m == CUDART_INF_F && t.s == t.s ? CUDART_INF_F : CUDART_NAN_F, CUDART_NAN_F, 0.f, 0.f, DISC_ROW_NONFINITE};
    if (!(t.m > -CUDART_INF_F)) return {-CUDART_INF_F, 0.f, 0.f, 0.f, DISC_ROW_NOMASS};
    const float l2 = log2f(t.s);
    // the reference is m c2 rounded; what the rounding took is exact in one multiply-add
    const float log_sum = LN2_F * (far ? l2 : l2 - fmaf(t.m, p.c2, -t.ref));
    return {fmaf(t.m, p.inv_t, log_sum), fmaxf(0.f, LN2_F * (l2 - t.u / t.s)), t.m, log_sum, 0};
}
// the log-probability of a logit of the row
__device__ __forceinline__ float log_prob(const LogprobParams& p, const RowResult& r, float x) {
    if (r.status & DISC_ROW_NOMASS) return -CUDART_INF_F;
    if (r.status & DISC_ROW_NONFINITE) return x * p.inv_t - r.lse;
    const float lp = fmaf(x - r.m, p.inv_t, -r.log_sum);
    return lp > 0.f ? 0.f : lp;       // roundings of the largest one's
}
// one thread
template <int DT>
__device__ __forceinline__ void store_row(const LogprobParams& p, int64_t row, const char* base, RowResult r) {
    if (p.lse) p.lse[row] = r.lse;
    if (p.entropy) p.entropy[row] = r.entropy;
    if (p.targets) {
        const int32_t tok = p.targets[row];
        float lp = 0.f;
        if (tok >= 0 && tok < p.V) lp = log_prob(p, r, Vec<DT>::at(base + size_t(tok) * Vec<DT>::SIZE));
        else if (tok != -1) {
            lp = CUDART_NAN_F;
            r.status |= DISC_ROW_DEAD;
        }
        if (p.logp) p.logp[row] = lp;
    }
    p.status[row] = r.status;
}
// the i-th alternative; -1 where there is none
__device__ __forceinline__ void store_top(const LogprobParams& p, int64_t row, unsigned int i, unsigned long long e, bool some, const RowResult& r) {
    p.top_ids[row * p.top + i] = some ? int32_t(~uint32_t(e)) : -1;
    if (p.top_logp)
        p.top_logp[row * p.top + i] = some ? log_prob(p, r, key_value(uint32_t(e >> 32))) : -CUDART_INF_F;
}

// ---- short rows --------------------------------------------------------------------------------------------
// Up to 32 EPL logits: a warp per row, the row in registers.  (A block per row would spend its time on barriers.)  The
// alternatives are taken one after the other, each lane offering its best.
template <int DT, int EPL>
__global__ void __launch_bounds__(NT) disc_logprobs_short_kernel(const LogprobParams p, int64_t n) {
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t(blockIdx.x) * NT + threadIdx.x) >> 5;
    if (row >= n) return;
    const char* base = static_cast<const char*>(p.logits) + row * p.ld * Vec<DT>::SIZE;
    float x[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) x[j] = lane + 32 * j < p.V ? Vec<DT>::at(base + size_t(lane + 32 * j) * Vec<DT>::SIZE) : -CUDART_INF_F;
    float mx = x[0];
#pragma unroll
    for (int j = 1; j < EPL; ++j) mx = fmaxf(mx, x[j]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, o));
    // relative to the maximum itself: no logit is too far out
    const float m = fabsf(mx) < CUDART_INF_F ? mx : 0.f;
    Sums t{mx == mx ? mx : -CUDART_INF_F, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        const float d = max_nan((x[j] - m) * p.c2, Y_MIN), e = ex2_approx(d);
        t.s += e;
        t.u = fmaf(d, e, t.u);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        t.s += __shfl_xor_sync(FULL, t.s, o);
        t.u += __shfl_xor_sync(FULL, t.u, o);
    }
    const RowResult res = row_result(p, t, true);
    if (lane == 0) store_row<DT>(p, row, base, res);
    if (p.top == 0) return;
    uint32_t key[EPL];                // + 1: 0 is what has been taken or is not there
#pragma unroll
    for (int j = 0; j < EPL; ++j) key[j] = lane + 32 * j < p.V ? max(order_key(x[j]), 1u) : 0u;
    const int some = min(p.top, p.V);
    uint32_t best = 0u;
    int at = -1;
    auto offer = [&]() {
        best = 0u;
        at = -1;
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            if (key[j] > best) { best = key[j]; at = j; }
    };
    offer();
    for (int i = 0; i < p.top; ++i) {
        unsigned long long e = 0ull;
        if (i < some) {
            const uint32_t hi = __reduce_max_sync(FULL, best);
            const int32_t id = best == hi && at >= 0 ? lane + 32 * at : 0x7fffffff;
            const int32_t won = __reduce_min_sync(FULL, id);
            if (id == won) {
#pragma unroll
                for (int j = 0; j < EPL; ++j)
                    if (j == at) key[j] = 0u;
                offer();
            }
            e = entry(hi, won);
        }
        if (lane == (i & 31)) store_top(p, row, i, e, i < some, res);
    }
}

constexpr int U = 4;                  // 16-byte loads a thread keeps in flight

template <int DT, bool TOP>
__global__ void __launch_bounds__(NT, 5) disc_logprobs_kernel(const LogprobParams p) {
    constexpr int E = Vec<DT>::E, SIZE = Vec<DT>::SIZE;
    extern __shared__ unsigned char smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    PortionMaxima<DT>& pm = *reinterpret_cast<PortionMaxima<DT>*>(smem_raw + sizeof(Smem));      // only with TOP
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x / unsigned(p.split);
    const uint32_t rank = p.split > 1 ? cluster_rank() : 0u;
    const RowShape<DT> r(p.logits, p.ld, row, p.V);
    const uint4* vecs = r.vecs();

    // this block's vectors [v0, v1); the first block also takes the elements around the vectors, one per thread
    const int32_t per = (r.nvec + p.split - 1) / p.split;
    const int32_t v0 = min(r.nvec, int32_t(rank) * per), v1 = min(r.nvec, v0 + per);
    int32_t extra = -1;
    if (rank == 0) {
        if (tid < r.head) extra = tid;
        else if (tid - r.head < r.tail) extra = r.head + r.nvec * E + tid - r.head;
    }

    Running run{-CUDART_INF_F, 0.f, make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    const float2 c2 = make_float2(p.c2, p.c2);
    const Scale k{p.c2, p.low_y};
    float extra_max = -CUDART_INF_F;
    if (extra >= 0) {
        const float x = Vec<DT>::at(r.base + size_t(extra) * SIZE);
        if (x > run.m) raise(run, x, k);
        extra_max = x;
        // the same steps as for a pair, on one element
        const float d = fmaf(max_nan(x, p.low), p.c2, -run.ref), e = ex2_approx(d);
        run.s.x += e;
        run.u.x = fmaf(d, e, run.u.x);
    }
    // portions of the thread's vectors: U of them, or more when that would make too many
    const int32_t rounds = (v1 - v0 + NT * U - 1) / (NT * U);
    const int32_t per_slot = (rounds + SLOTS - 1) / SLOTS;
    int32_t in_slot = 0, slot = 0;
    float slot_max = -CUDART_INF_F;
    for (int32_t v = v0 + tid; v < v0 + rounds * (NT * U); v += NT * U) {
        uint4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = v + u * NT < v1 ? ld_stream(vecs + v + u * NT) : Vec<DT>::lowest();
        const float mx = Vec<DT>::template largest<U>(w);
        if (mx > run.m) raise(run, mx, k);
        if (TOP) {
            slot_max = fmaxf(slot_max, mx);
            if (++in_slot == per_slot) {
                pm.at[slot][tid] = Vec<DT>::shorten(slot_max);
                ++slot;
                in_slot = 0;
                slot_max = -CUDART_INF_F;
            }
        }
        const float2 down = make_float2(-run.ref, -run.ref);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[E];
            Vec<DT>::unpack(Vec<DT>::floor_at(w[u], p.low), x);
#pragma unroll
            for (int j = 0; j < E; j += 2) add(run, make_float2(x[j], x[j + 1]), c2, down);
        }
    }
    if (TOP && in_slot > 0) pm.at[slot][tid] = Vec<DT>::shorten(slot_max);
    Sums a{run.m, run.ref, run.s.x + run.s.y, run.u.x + run.u.y};

    const float own_max = run.m;
    a = join_lanes<32>(a, k);
    if (lane == 0) sm.warp_sums[warp] = a;
    const uint32_t key = v0 + tid < v1 || extra >= 0 ? order_key(own_max) : 0u;
    unsigned int found = 0;
    if (TOP) {
        sm.keys[tid] = key;
        if (tid == 0) { sm.n_hot = 0u; sm.n_list = 0u; }
    }
    __syncthreads();
    if (warp == 1) {                  // beside the selection, which the first warp begins
        const Sums t = join_lanes<NW>(sm.warp_sums[lane % NW], k);
        if (lane == 0) sm.part = t;
    }
    if (TOP) {
        const int32_t elements = (v1 - v0) * E + (rank == 0 ? r.head + r.tail : 0);
        const unsigned int want = min(unsigned(p.top), unsigned(elements));
        if (want > 0) {
            if (warp == 0) {
                const uint32_t t = kth_key(sm.keys, want, lane);
                if (lane == 0) sm.threshold = t;
            }
            __syncthreads();
            const uint32_t thr = sm.threshold;
            if (v0 + tid < v1 && key >= thr)
                for (int32_t i = 0; i * per_slot < rounds; ++i)
                    if (order_key(Vec<DT>::lengthen(pm.at[i][tid])) >= thr) {
                        const unsigned int at = atomicAdd(&sm.n_hot, 1u);
                        if (at < HOT_CAP) sm.hot[at] = i << 8 | tid;
                    }
            if (extra >= 0) {
                const uint32_t k = order_key(extra_max);
                if (k >= thr) sm.list[atomicAdd(&sm.n_list, 1u)] = entry(k, extra);
            }
            __syncthreads();
            const unsigned int n_hot = sm.n_hot;
            const int32_t each = per_slot * U, n_look = n_hot <= HOT_CAP ? int32_t(n_hot) * each : 0;
            for (int32_t i = tid; i < n_look; i += NT) {
                const int32_t h = sm.hot[i / each];
                const int32_t v = v0 + ((h >> 8) * each + i % each) * NT + (h & 255);
                if (v < v1) {
                    const uint4 w = __ldg(vecs + v);
                    float x[E];
                    Vec<DT>::unpack(w, x);
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const uint32_t k = order_key(x[j]);
                        if (k >= thr) {
                            const unsigned int at = atomicAdd(&sm.n_list, 1u);
                            if (at < LIST_CAP) sm.list[at] = entry(k, r.head + v * E + j);
                        }
                    }
                }
            }
            __syncthreads();
            unsigned int cnt = sm.n_list;
            if (n_hot > HOT_CAP || cnt > LIST_CAP || cnt < want) {
                const int32_t e0 = rank == 0 ? 0 : r.head + v0 * E;
                // the first block's slice is not one run of ids when others lie between it and the row's last
                // elements; those few are put in by hand
                const int32_t e1 = p.split == 1 ? p.V : r.head + v1 * E;
                const bool apart = rank == 0 && p.split > 1 && r.tail > 0;
                const unsigned int in_run = unsigned(e1 - e0);
                select_slice<DT>(r.base, e0, e1, min(want, in_run), sm);
                if (apart && tid < r.tail) {
                    const int32_t e = r.head + r.nvec * E + tid;
                    sm.list[atomicAdd(&sm.n_list, 1u)] = entry(order_key(Vec<DT>::at(r.base + size_t(e) * SIZE)), e);
                }
                __syncthreads();
                cnt = sm.n_list;
            }
            rank_list(sm, cnt, want);
        }
        found = want;
    }
    if (TOP && tid == 0) sm.found = found;
    if (p.split > 1) {
        cluster_sync_all();
        if (rank == 0) {
            if (warp == 1) {
                Sums t{-CUDART_INF_F, 0.f, 0.f, 0.f};
                if (lane < p.split) {
                    const uint32_t q = remote(&sm.part, lane);
                    t = Sums{__uint_as_float(ld_remote32(q)), __uint_as_float(ld_remote32(q + 4)), __uint_as_float(ld_remote32(q + 8)), __uint_as_float(ld_remote32(q + 12))};
                }
                t = join_lanes<8>(t, k);
                __syncwarp();
                if (lane == 0) sm.row = t;
            }
            if (TOP) {
                // all blocks' lists together: at most 8 x 64 entries
                const unsigned int f = lane < p.split ? ld_remote32(remote(&sm.found, lane)) : 0u;
                unsigned int upto = f;
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) {
                    const unsigned int u = __shfl_up_sync(FULL, upto, o);
                    if (lane >= o) upto += u;
                }
                const unsigned int all = __shfl_sync(FULL, upto, 7);
                for (unsigned int i = tid; i < 8 * TOP_MAX; i += NT) {
                    const int c = int(i) / TOP_MAX;
                    const unsigned int j = i % TOP_MAX;
                    const unsigned int n = __shfl_sync(FULL, f, c), before = __shfl_sync(FULL, upto, c) - n;
                    if (j < n) sm.list[before + j] = ld_remote64(remote(&sm.best[j], c));
                }
                __syncthreads();
                found = min(unsigned(p.top), all);
                rank_list(sm, all, found);
            }
        }
        cluster_sync_all();
        if (rank != 0) return;
    }
    __syncthreads();

    Sums t = p.split > 1 ? sm.row : sm.part;
    bool far = fabsf(t.m) < CUDART_INF_F && !(t.m * p.c2 > p.low_y + 256.f && t.m * p.c2 < FAR_Y) && t.s == t.s;
    if (far) {                        // the largest logit itself is that far out: once more, with differences of logits
        Sums b{t.m, 0.f, 0.f, 0.f};
        for (int32_t e = tid; e < p.V; e += NT) {
            const float d = max_nan((Vec<DT>::at(r.base + size_t(e) * SIZE) - t.m) * p.c2, Y_MIN), x = ex2_approx(d);
            b.s += x;
            b.u = fmaf(d, x, b.u);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            b.s += __shfl_xor_sync(FULL, b.s, o);
            b.u += __shfl_xor_sync(FULL, b.u, o);
        }
        if (lane == 0) sm.warp_sums[warp] = b;
        __syncthreads();
        t.s = t.u = 0.f;
        for (int w = 0; w < NW; ++w) { t.s += sm.warp_sums[w].s; t.u += sm.warp_sums[w].u; }
    }
    const RowResult res = row_result(p, t, far);
    if (tid == 0) store_row<DT>(p, row, r.base, res);
    if (TOP)
        for (unsigned int i = tid; i < unsigned(p.top); i += NT) store_top(p, row, i, i < found ? sm.best[i] : 0ull, i < found, res);
}

// ---- gradient ---------------------------------------------------------------------------------------
// With a = d logp, b = dH of the row (H = entropy, p_v = 2^(y_v - lse log2e)):
//   dz_v = (a [v = t] - p_v (a + b (log p_v + H))) / T
// One read and one write per logit; one 2^x and a handful of multiply-adds, bound by the bytes: 44 us for
// 2047 x 32000 bf16 (0.26 GB, 6.0 TB/s).
struct GradParams {
    const void* logits;
    int64_t ld;
    void* grad;
    int64_t grad_ld;
    int32_t V, teams_per_row;
    float inv_t, c2;
    const int32_t* targets;           // nullable
    const float* lse;
    const float* entropy;             // nullable when d_entropy is
    const float* d_logp;              // nullable
    const float* d_entropy;           // nullable
};

struct RowGrad {
    float l2, a_bh, b, scale, a_t;    // lse in units of y; a + b H; b ln2; 1/T; a / T
    float m;                          // ANEW: the row's maximum, and l2 its sum relative to that
    int32_t tok;
    template <bool ANEW>
    __device__ __forceinline__ float at(float x, float c2) const {
        const float y = max_nan(fmaf(ANEW ? x - m : x, c2, -l2), Y_MIN);
        return -scale * ex2_approx(y) * fmaf(y, b, a_bh);
    }
};
// a thread's vectors v0, v0 + TEAM, ... of a row
template <int DT, int TEAM>
__device__ __forceinline__ void load_vectors(const RowShape<DT>& r, int32_t v0, uint4* w) {
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (v0 + u * TEAM < r.nvec) w[u] = ld_stream_own(r.vecs() + v0 + u * TEAM);
}
template <int DT, int TEAM, bool ANEW>
__device__ __forceinline__ void grad_vectors(const RowShape<DT>& r, char* out, const RowGrad& g, float c2, int32_t v0, const uint4* w) {
    constexpr int E = Vec<DT>::E, SIZE = Vec<DT>::SIZE;
    const bool together = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(r.base)) & 15) == 0;
    char* out_vecs = out + size_t(r.head) * SIZE;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t v = v0 + u * TEAM;
        if (v < r.nvec) {
            float x[E];
            Vec<DT>::unpack(w[u], x);
            const int32_t at = g.tok - (r.head + v * E);
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = g.template at<ANEW>(x[j], c2) + (at == j ? g.a_t : 0.f);
            if (together) __stcs(reinterpret_cast<uint4*>(out_vecs) + v, Vec<DT>::pack(x));
            else
#pragma unroll
                for (int j = 0; j < E; ++j) Vec<DT>::put(out_vecs + (size_t(v) * E + j) * SIZE, x[j]);
        }
    }
}
// a thread's element before or after the vectors, -1: none
template <int DT>
__device__ __forceinline__ int32_t around_vectors(const RowShape<DT>& r, int tid) {
    if (tid < r.head) return tid;
    return tid - r.head < r.tail ? r.head + r.nvec * Vec<DT>::E + tid - r.head : -1;
}
template <int DT, bool ANEW>
__device__ __forceinline__ void grad_element(const RowShape<DT>& r, char* out, const RowGrad& g, float c2, int32_t e) {
    constexpr int SIZE = Vec<DT>::SIZE;
    if (e >= 0) Vec<DT>::put(out + size_t(e) * SIZE, g.template at<ANEW>(Vec<DT>::at(r.base + size_t(e) * SIZE), c2) + (e == g.tok ? g.a_t : 0.f));
}

// A log-sum-exp is given rounded to fp32, which puts a factor 1 +- |lse| 2^-24 on all probabilities of the row: 8e-6 up to this
// limit.  For rows beyond it (low temperatures, rows masked with a finite value, where log S would be lost) one team takes the
// whole row, forms maximum and sum anew and then the gradient; the row's other teams have nothing to do.  (4096 x 32000 bf16: 82 us
// when all rows are within the limit, 140 when all are beyond it; 16 x 128256: 12 and 28.)
constexpr float LSE_LIMIT = 128.f;

// Called by the whole team.
template <int DT, int TEAM>
__device__ __noinline__ void row_anew(const void* logits, int64_t ld, char* out, int32_t V, int64_t row, int tid, float lse, RowGrad g, float c2) {
    const RowShape<DT> r(logits, ld, row, V);
    const int32_t extra = around_vectors(r, tid);
    // the row's maximum m and its sum s of 2^((x - m) c2)
    constexpr int E = Vec<DT>::E, SIZE = Vec<DT>::SIZE, UN = 2;
    float m = -CUDART_INF_F, s = 0.f;
    auto up_to = [&](float mx) {
        if (mx > m) { s *= ex2_approx((m - mx) * c2); m = mx; }
        return m > -CUDART_INF_F ? m : 0.f;
    };
    if (extra >= 0) {
        const float x = Vec<DT>::at(r.base + size_t(extra) * SIZE), ref = up_to(x);
        s += ex2_approx((x - ref) * c2);
    }
    for (int32_t v = tid; v < r.nvec; v += UN * TEAM) {
        uint4 w[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) w[u] = v + u * TEAM < r.nvec ? r.vecs()[v + u * TEAM] : Vec<DT>::lowest();
        const float ref = up_to(Vec<DT>::template largest<UN>(w));
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            float x[E];
            Vec<DT>::unpack(w[u], x);
#pragma unroll
            for (int j = 0; j < E; ++j) s += ex2_approx((x[j] - ref) * c2);
        }
    }
    auto join = [&](float m2, float s2) {
        const float top = fmaxf(m, m2), ref = top > -CUDART_INF_F ? top : 0.f;
        s = s * ex2_approx((m - ref) * c2) + s2 * ex2_approx((m2 - ref) * c2);
        m = top;
    };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) join(__shfl_xor_sync(FULL, m, o), __shfl_xor_sync(FULL, s, o));
    if (TEAM == NT) {
        __shared__ float2 warps[NW];
        if ((tid & 31) == 0) warps[tid >> 5] = make_float2(m, s);
        __syncthreads();
        m = -CUDART_INF_F;
        s = 0.f;
        for (int w = 0; w < NW; ++w) join(warps[w].x, warps[w].y);
    }
    // A log-sum-exp that is not these logits' own, of a row that lies here only in part, say, is taken as it is given.
    const float log_sum = log2f(s), given = fmaf(-m, g.scale, lse);
    g.m = m;
    g.l2 = fabsf(fmaf(log_sum, -LN2_F, given)) <= fabsf(lse) * 4.76837158203125e-7f ? log_sum : given * LOG2E_F;      // 2^-21
    for (int32_t v = tid; v < r.nvec; v += TEAM * U) {
        uint4 w[U];
        load_vectors<DT, TEAM>(r, v, w);
        grad_vectors<DT, TEAM, true>(r, out, g, c2, v, w);
    }
    grad_element<DT, true>(r, out, g, c2, extra);
}

// TEAM threads work on a portion of a row: a block, or a warp where a warp's loads cover the row.
template <int DT, int TEAM>
__global__ void __launch_bounds__(NT, TEAM == NT ? 6 : 5) disc_logprobs_grad_kernel(const GradParams p, int64_t n) {
    const int64_t team = (int64_t(blockIdx.x) * NT + threadIdx.x) / TEAM;
    const int64_t row = TEAM == NT ? int64_t(blockIdx.x / unsigned(p.teams_per_row)) : team;
    const int32_t part = TEAM == NT ? int32_t(blockIdx.x - row * p.teams_per_row) : 0;
    const int tid = threadIdx.x % TEAM;
    if (row >= n) return;
    const RowShape<DT> r(p.logits, p.ld, row, p.V);
    char* out = static_cast<char*>(p.grad) + row * p.grad_ld * Vec<DT>::SIZE;
    const int32_t v0 = part * (TEAM * U) + tid;
    uint4 w[U];
    load_vectors<DT, TEAM>(r, v0, w);  // under way while the row's numbers come in
    RowGrad g;
    g.tok = p.targets ? p.targets[row] : -1;
    const float a = p.d_logp && g.tok >= 0 && g.tok < p.V ? p.d_logp[row] : 0.f;
    const float b = p.d_entropy ? p.d_entropy[row] : 0.f;
    const float lse = p.lse[row];
    g.l2 = lse * LOG2E_F;
    g.a_bh = b != 0.f ? fmaf(b, p.entropy[row], a) : a;
    g.b = b * LN2_F;
    g.scale = p.inv_t;
    if (lse == -CUDART_INF_F) { g.l2 = 0.f; g.scale = 0.f; }      // no mass: nothing to move
    else if (!(lse < CUDART_INF_F)) g.l2 = CUDART_NAN_F;          // +inf or NaN among the logits: no gradient is finite
    g.a_t = g.scale * a;
    if (fabsf(lse) >= LSE_LIMIT && fabsf(lse) < CUDART_INF_F) {
        if (part == 0) row_anew<DT, TEAM>(p.logits, p.ld, out, p.V, row, tid, lse, g, p.c2);
        return;
    }
    grad_vectors<DT, TEAM, false>(r, out, g, p.c2, v0, w);
    if (part == 0) grad_element<DT, false>(r, out, g, p.c2, around_vectors(r, tid));
}

template <int DT, int EPL>
int launch_short(const LogprobParams& p, int64_t n, cudaStream_t st) {
    disc_logprobs_short_kernel<DT, EPL><<<unsigned((n * 32 + NT - 1) / NT), NT, 0, st>>>(p, n);
    DISC_CUDA(cudaGetLastError());
    return DISC_OK;
}
template <int DT>
int launch_short(const LogprobParams& p, int64_t n, cudaStream_t st) {
    return p.V <= 256 ? launch_short<DT, 8>(p, n, st) : launch_short<DT, 32>(p, n, st);
}

template <int DT, bool TOP>
int launch_logprobs(const LogprobParams& p, int64_t n, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(n * p.split));
    cfg.blockDim = dim3(NT);
    constexpr int bytes = sizeof(Smem) + (TOP ? sizeof(PortionMaxima<DT>) : 0);
    static std::atomic<uint64_t> done{0};
    if (const int rc = disc::allow_smem(disc_logprobs_kernel<DT, TOP>, bytes, done)) return rc;
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(p.split);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.split > 1 ? 1 : 0;
    DISC_CUDA(cudaLaunchKernelEx(&cfg, disc_logprobs_kernel<DT, TOP>, p));
    return DISC_OK;
}

bool bad_logits(const void* logits, int dtype) { return (reinterpret_cast<uintptr_t>(logits) & (dtype == DISC_F32 ? 3u : 1u)) != 0; }

}  // namespace

extern "C" {

int disc_logprobs(const void* logits, disc_dtype_t dtype, int64_t ld, int64_t n, int32_t vocab_size, float inv_temperature,
                  const int32_t* targets, int32_t top, float* logp_out, float* entropy_out, float* lse_out,
                  int32_t* top_ids_out, float* top_logp_out, uint8_t* status_out, void* stream) {
    if (n < 0 || vocab_size <= 0 || ld < vocab_size || top < 0) return DISC_ERR_ARG;
    if (dtype != DISC_F32 && dtype != DISC_BF16) return DISC_ERR_UNSUPPORTED;
    if (top > TOP_MAX || n > (int64_t(1) << 27)) return DISC_ERR_UNSUPPORTED;
    if (!(inv_temperature > 0.f) || !(inv_temperature <= 3.0e38f)) return DISC_ERR_ARG;
    if (n == 0) return DISC_OK;
    if (!logits || !status_out || (top > 0 && !top_ids_out) || (targets && !logp_out)) return DISC_ERR_ARG;
    if (bad_logits(logits, dtype)) return DISC_ERR_ARG;
    int sms = 0;
    if (const int rc = disc::device_sms(&sms)) return rc;
    LogprobParams p;
    p.logits = logits; p.ld = ld; p.V = vocab_size; p.top = top;
    p.inv_t = inv_temperature; p.c2 = inv_temperature * LOG2E_F;
    p.low = __bfloat162float(__float2bfloat16_rn(fmaxf(-FAR_Y / p.c2, -1.0e37f)));
    p.low_y = p.low * p.c2;
    p.targets = targets; p.logp = logp_out; p.entropy = entropy_out; p.lse = lse_out;
    p.top_ids = top_ids_out; p.top_logp = top_logp_out; p.status = status_out;
    // too few rows to put a block on every SM: a row is shared by a cluster, as long as every block still has
    // some vectors for each of its threads
    p.split = 1;
    const int64_t vecs = vocab_size / (dtype == DISC_F32 ? 4 : 8);
    while (p.split < 8 && n * p.split * 2 <= 2 * sms && vecs / (p.split * 2) >= NT) p.split *= 2;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // Short rows, a warp per row or a block per row (us, bf16, warps / blocks; f32 crosses at the same places):
    //   4096 rows of 256    1 alternative  5 / 37    20  17 / 40    64   45 / 74
    //   4096 rows of 1000   1             14 / 37    16  39 / 40    20   45 / 41    64  116 / 50
    //   32 rows of 256      8              5 / 6     12   6 / 6     20    8 / 6     64   19 / 7
    //   32 rows of 1000     1              6 / 6      4   8 / 6     20   16 / 6     64   37 / 7
    // Alternatives cost a warp 0.25 to 0.6 us each, one after the other, whatever the number of rows, and blocks next to
    // nothing as long as all of them run at once.
    const bool wave = n <= int64_t(sms) * 5;
    if (vocab_size <= 256 ? !wave || top <= 12 : vocab_size <= SHORT_ROW && !wave && top <= 16) return dtype == DISC_F32 ? launch_short<DISC_F32>(p, n, st) : launch_short<DISC_BF16>(p, n, st);
    if (dtype == DISC_F32) return top ? launch_logprobs<DISC_F32, true>(p, n, st) : launch_logprobs<DISC_F32, false>(p, n, st);
    return top ? launch_logprobs<DISC_BF16, true>(p, n, st) : launch_logprobs<DISC_BF16, false>(p, n, st);
}

int disc_logprobs_grad(const void* logits, disc_dtype_t dtype, int64_t ld, int64_t n, int32_t vocab_size, float inv_temperature,
                       const int32_t* targets, const float* lse, const float* entropy, const float* d_logp, const float* d_entropy,
                       void* grad_out, int64_t grad_ld, void* stream) {
    if (n < 0 || vocab_size <= 0 || ld < vocab_size || grad_ld < vocab_size) return DISC_ERR_ARG;
    if (dtype != DISC_F32 && dtype != DISC_BF16) return DISC_ERR_UNSUPPORTED;
    if (!(inv_temperature > 0.f) || !(inv_temperature <= 3.0e38f)) return DISC_ERR_ARG;
    if (n == 0) return DISC_OK;
    if (!logits || !lse || !grad_out || (d_logp && !targets) || (d_entropy && !entropy)) return DISC_ERR_ARG;
    if (bad_logits(logits, dtype) || bad_logits(grad_out, dtype)) return DISC_ERR_ARG;
    // in place is fine; rows that overlap in any other way are not
    if (grad_out == logits && grad_ld != ld) return DISC_ERR_ARG;
    const int64_t vecs = vocab_size / (dtype == DISC_F32 ? 4 : 8);
    GradParams p;
    p.logits = logits; p.ld = ld; p.grad = grad_out; p.grad_ld = grad_ld; p.V = vocab_size;
    p.inv_t = inv_temperature; p.c2 = inv_temperature * LOG2E_F;
    p.targets = targets; p.lse = lse; p.entropy = entropy; p.d_logp = d_logp; p.d_entropy = d_entropy;
    const bool warps = vecs <= 32 * U;
    p.teams_per_row = warps ? 1 : int32_t(vecs / (NT * U) + 1);
    if (n * p.teams_per_row > 0x7fffffff) return DISC_ERR_UNSUPPORTED;
    const unsigned grid = warps ? unsigned((n + NW - 1) / NW) : unsigned(n * p.teams_per_row);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == DISC_F32) {
        if (warps) disc_logprobs_grad_kernel<DISC_F32, 32><<<grid, NT, 0, st>>>(p, n);
        else disc_logprobs_grad_kernel<DISC_F32, NT><<<grid, NT, 0, st>>>(p, n);
    } else {
        if (warps) disc_logprobs_grad_kernel<DISC_BF16, 32><<<grid, NT, 0, st>>>(p, n);
        else disc_logprobs_grad_kernel<DISC_BF16, NT><<<grid, NT, 0, st>>>(p, n);
    }
    DISC_CUDA(cudaGetLastError());
    return DISC_OK;
}

}  // extern "C"
