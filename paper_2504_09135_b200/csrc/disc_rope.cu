// Queries and keys on their way to attention: each head's RMS norm and the rotation by the token's position in one pass
// (disc_norm_rope), its gradient (disc_norm_rope_grad), and, with the keys and values going straight into a cache's pages,
// disc_norm_rope_write.
//
//   u = w x r,  r = 1 / sqrt(mean(x^2) + eps);   y_a = u_a cos t_i - u_b sin t_i,  y_b = u_b cos t_i + u_a sin t_i,
//   t_i = position inv_freq_i,  (a, b) = (i, i + rot / 2) or (2 i, 2 i + 1)
//
// Backward, with g = dy rotated by -t, c = w g and z = x r:  dw = sum g z,  dx = r (c - z mean(c z)).  The vectors are normed first: r^3, which
// r c - x r^3 mean(c x) has, leaves the range of fp32 where |x| is 10^15, or 10^-13 with eps = 0.
//
// Bound by the bytes: every vector is read once and written once, and what stands in the way are the instructions around them.  So a
// lane holds 16 values of a vector, two runs of 8 that are rotated into one another (8 or 4 lanes a vector, 4 or 8 vectors side by side
// in a warp; vectors that cannot be cut like that have runs of 4): loads and stores of 16 bytes, three or two shuffles for a sum of
// squares.  A warp's vectors are all of one kind, queries, keys or values, and it goes from token to token, the next ones on their way
// into a ring in shared memory, of which every lane fills and reads places of its own, while the present ones are worked on.  What a
// token's vectors have in common, weight times cosine and weight times sine, is formed once for all of them: y = r (P x + Q x'), x' the
// other value of the pair.
//
// Angles: the fraction of a turn, position x inv_freq / 2 pi less its whole turns, is the product of two whole numbers modulo 2^64 (the
// frequency as a 64-bit fraction of a turn, which wraps by itself), so that a position of a million is as exact as one of ten; an fp32
// product would be off by 0.03 there.  Then sin and cos of that fraction in fp32, each pair's by one lane, and through shared memory to the lanes
// that turn it.
//
// Measured, bf16, heads of 128: 16384 tokens x 40 heads 57 to 60 us (336 MB, 5.6 to 5.9 TB/s), the gradient of 8191 tokens x 40 heads 51 us (252 MB,
// 4.9 TB/s).  Heads of 80 take as long as heads of 96, 56 and 51 us: five or six of a vector's eight lanes have values.

#include "disc_held.cuh"

namespace {

using namespace disc;

constexpr unsigned FULL = 0xffffffffu;
constexpr int THREADS = 128;           // of a block of the gradient
constexpr int WARPS = THREADS / 32;
constexpr int DEPTH = 6;               // steps of a warp in flight, and the one it is at
constexpr int GRAD_DEPTH = 4;
constexpr int FORWARD_WARPS = 20;      // blocks of one warp, on an SM
constexpr int GRAD_BLOCKS = 3;         // on an SM
constexpr int SMS = 148;
constexpr int MAX_GRAD_BLOCKS = SMS * GRAD_BLOCKS;     // which each leave sums of their own
constexpr int MOST_TOKENS = 32;        // of a warp, whose lanes look up one each
constexpr int MOST_STEPS = 8;

struct Vectors {                       // strides in bytes
    unsigned char* at;
    int64_t token, head;
};
struct RopeParams {
    Vectors x[3];                      // queries, keys; values, which are only written
    Vectors y[2];
    int32_t n, D, rot, interleaved, norm, weights_f32;
    float inv_D;
    int32_t heads[3];
    const void* w[2];
    float eps;
    const int32_t* pos;                // nullable with a cache: the place in the row
    const float* inv_freq;
};
struct CacheParams {
    unsigned char* plane[2];
    const int32_t* table;
    const int32_t* len;
    int32_t rows, width, pages, page_size, shift, held, token_bytes, head_bytes;
    const int32_t* cu;                 // nullable: one token per sequence
    const int32_t* seq_rows;           // nullable: sequence i is row i
    const uint8_t* status;             // nullable
    int32_t n_seqs;
};

// Queries, keys or values: by selection, as an index into the parameters would put them on the stack.
__device__ __forceinline__ Vectors pick(const Vectors* v, int kind) { return kind == 0 ? v[0] : kind == 1 ? v[1] : v[2]; }
__device__ __forceinline__ Vectors pick2(const Vectors* v, int kind) { return kind == 0 ? v[0] : v[1]; }

__device__ __forceinline__ float2 swapped(float2 a) { return make_float2(a.y, a.x); }

// Where a lane's two runs of RUN values begin.  Rotated: the pairs (a + i, b + i), i < RUN, or, interleaved, neighbours in both.
struct Place {
    int32_t a, b;
    bool some, turned;
};
template <int RUN>
__device__ __forceinline__ Place place_of(const RopeParams& p, int c) {
    Place at;
    at.some = c * 2 * RUN < p.D;
    at.turned = c * 2 * RUN < p.rot;
    const bool split = at.turned && !p.interleaved;
    at.a = split ? RUN * c : 2 * RUN * c;
    at.b = split ? p.rot / 2 + RUN * c : 2 * RUN * c + RUN;
    return at;
}
// A lane's values: 16-bit words as they lie in memory, or pairs of neighbours in fp32, run a, then run b.
template <int RUN>
struct Raw {
    uint32_t w[RUN];
};
template <int RUN>
__device__ __forceinline__ Raw<RUN> load_raw(const unsigned char* a_run, const unsigned char* b_run) {
    Raw<RUN> r;
    if constexpr (RUN == 8) {
        const uint4 a = *reinterpret_cast<const uint4*>(a_run), b = *reinterpret_cast<const uint4*>(b_run);
        r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w; r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
    } else {
        const uint2 a = *reinterpret_cast<const uint2*>(a_run), b = *reinterpret_cast<const uint2*>(b_run);
        r.w[0] = a.x; r.w[1] = a.y; r.w[2] = b.x; r.w[3] = b.y;
    }
    return r;
}
// a lane's two runs of a vector into its places of a step in shared memory; zeros when !some
template <int RUN>
__host__ __device__ constexpr int step_bytes() { return 32 * RUN * 4; }
template <int RUN>
__device__ __forceinline__ void copy_in(uint32_t step, const unsigned char* v, const Place& at, bool some, int lane) {
    const uint32_t to = step + lane * (RUN * 2);
    const int n = some ? RUN * 2 : 0;
    const unsigned char *a = v + at.a * 2, *b = v + at.b * 2;
    if constexpr (RUN == 8) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(a), "r"(n) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + 32 * 16), "l"(b), "r"(n) : "memory");
    } else {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to), "l"(a), "r"(n) : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to + 32 * 8), "l"(b), "r"(n) : "memory");
    }
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_for_all_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int RUN>
__device__ __forceinline__ void store_raw(unsigned char* v, const Place& at, const Raw<RUN>& r) {
    if constexpr (RUN == 8) {
        *reinterpret_cast<uint4*>(v + at.a * 2) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
        *reinterpret_cast<uint4*>(v + at.b * 2) = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
    } else {
        *reinterpret_cast<uint2*>(v + at.a * 2) = make_uint2(r.w[0], r.w[1]);
        *reinterpret_cast<uint2*>(v + at.b * 2) = make_uint2(r.w[2], r.w[3]);
    }
}
template <typename T, int RUN>
__device__ __forceinline__ void unpack(const Raw<RUN>& r, float2* x) {
#pragma unroll
    for (int i = 0; i < RUN; ++i) x[i] = unpack2<T>(r.w[i]);
}
template <typename T, int RUN>
__device__ __forceinline__ Raw<RUN> pack(const float2* x) {
    Raw<RUN> r;
#pragma unroll
    for (int i = 0; i < RUN; ++i) r.w[i] = pack2<T>(x[i].x, x[i].y);
    return r;
}
template <typename T, int RUN>
__device__ __forceinline__ void load_weights(const RopeParams& p, int kind, const Place& at, float2* w) {
#pragma unroll
    for (int i = 0; i < RUN; ++i) w[i] = make_float2(1.f, 1.f);
    const void* from = kind ? p.w[1] : p.w[0];
    if (!from || !at.some) return;
    if (p.weights_f32) {
        const float* f = static_cast<const float*>(from);
#pragma unroll
        for (int i = 0; i < RUN; i += 2) {
            const float4 v = *reinterpret_cast<const float4*>(f + (i < RUN / 2 ? at.a + 2 * i : at.b + 2 * i - RUN));
            w[i] = make_float2(v.x, v.y);
            w[i + 1] = make_float2(v.z, v.w);
        }
    } else {
        const unsigned char* v = static_cast<const unsigned char*>(from);
        unpack<T, RUN>(load_raw<RUN>(v + at.a * 2, v + at.b * 2), w);
    }
}

// Cosines and sines of a warp's token: each of the rot / 2 <= 64 pairs by one lane, through shared memory.
struct __align__(16) Turns {           // read four at a time
    float c[64], s[64];
};
static_assert(alignof(Turns) == 16 && sizeof(Turns) % 16 == 0, "read_turns");
struct Frequencies {
    uint64_t f[2];                     // of pairs lane and lane + 32, as fractions of a turn of 63 bits; the last bit says that it is not finite
};
__device__ __forceinline__ Frequencies frequencies_of(const RopeParams& p, int lane) {
    Frequencies q;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        q.f[i] = 0;
        if (2 * (lane + 32 * i) >= p.rot) continue;
        const float inv_freq = p.inv_freq[lane + 32 * i];
        const double turns = double(inv_freq) * 0.15915494309189533577;          // 1 / 2 pi
        q.f[i] = fabsf(inv_freq) < CUDART_INF_F ? uint64_t((turns - floor(turns)) * 18446744073709551616.0) & ~uint64_t(1) : 1;
    }
    return q;
}
__device__ __forceinline__ void turn_to(const RopeParams& p, int32_t pos, const Frequencies& q, Turns& out, int lane) {
    __syncwarp();                      // the token before has been read by all lanes
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (64 * i >= p.rot) break;
        const int32_t part = int32_t(uint32_t((uint64_t(int64_t(pos)) * q.f[i]) >> 32));          // of 2^32, from -1/2 to 1/2 of a turn
        float s, c;
        sincospif(q.f[i] & 1 ? CUDART_NAN_F : float(part) * 0x1p-31f, &s, &c);
        out.c[lane + 32 * i] = c;
        out.s[lane + 32 * i] = s;
    }
    __syncwarp();
}
// the lane's RUN pairs
template <int RUN>
__device__ __forceinline__ void read_turns(const Turns& t, int c, float* cs, float* sn) {
#pragma unroll
    for (int i = 0; i < RUN; i += 4) {
        const float4 a = *reinterpret_cast<const float4*>(t.c + RUN * c + i), b = *reinterpret_cast<const float4*>(t.s + RUN * c + i);
        cs[i] = a.x; cs[i + 1] = a.y; cs[i + 2] = a.z; cs[i + 3] = a.w;
        sn[i] = b.x; sn[i + 1] = b.y; sn[i + 2] = b.z; sn[i + 3] = b.w;
    }
}
// y_i = x_i P_i + x'_i Q_i, x' the pairs' other values: of the other run, or, interleaved, the neighbours
template <int RUN>
__device__ __forceinline__ void turn(float2* x, const float2* P, const float2* Q, bool interleaved) {
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < RUN; ++i) x[i] = fma2(x[i], P[i], mul2(swapped(x[i]), Q[i]));
    } else {
#pragma unroll
        for (int i = 0; i < RUN / 2; ++i) {
            const float2 u = x[i], v = x[i + RUN / 2];
            x[i] = fma2(u, P[i], mul2(v, Q[i]));
            x[i + RUN / 2] = fma2(v, P[i + RUN / 2], mul2(u, Q[i + RUN / 2]));
        }
    }
}
// P and Q for weights w: y_a = w_a x_a c - w_b x_b s, y_b = w_b x_b c + w_a x_a s
template <int RUN>
__device__ __forceinline__ void coefficients(const Turns& t, int c, const float2* w, bool interleaved, float2* P, float2* Q) {
    float cs[RUN], sn[RUN];
    read_turns<RUN>(t, c, cs, sn);
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            const float s = sn[i];
            P[i] = make_float2(w[i].x * cs[i], w[i].y * cs[i]);
            Q[i] = make_float2(-w[i].y * s, w[i].x * s);
        }
    } else {
        constexpr int H = RUN / 2;
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const float2 cc = make_float2(cs[2 * i], cs[2 * i + 1]), ss = make_float2(sn[2 * i], sn[2 * i + 1]);
            P[i] = mul2(w[i], cc);
            P[i + H] = mul2(w[i + H], cc);
            Q[i] = mul2(w[i + H], make_float2(-ss.x, -ss.y));
            Q[i + H] = mul2(w[i], ss);
        }
    }
}
// back by the angles, without weights: half the registers of P and Q
template <int RUN>
__device__ __forceinline__ void turn_back(float2* x, const float* cs, const float* sn, bool interleaved) {
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < RUN; ++i) x[i] = fma2(x[i], make_float2(cs[i], cs[i]), mul2(swapped(x[i]), make_float2(sn[i], -sn[i])));
    } else {
#pragma unroll
        for (int i = 0; i < RUN / 2; ++i) {
            const float2 c = make_float2(cs[2 * i], cs[2 * i + 1]), t = make_float2(sn[2 * i], sn[2 * i + 1]), u = x[i], v = x[i + RUN / 2];
            x[i] = fma2(u, c, mul2(v, t));
            x[i + RUN / 2] = fma2(v, c, mul2(u, make_float2(-t.x, -t.y)));
        }
    }
}
template <int LPV>
__device__ __forceinline__ float sum_of(float x) {
#pragma unroll
    for (int o = 1; o < LPV; o <<= 1) x += __shfl_xor_sync(FULL, x, o);
    return x;
}
template <int LPV, int RUN>
__device__ __forceinline__ float inverse_norm(const RopeParams& p, const float2* x) {
    float2 s = mul2(x[0], x[0]);
#pragma unroll
    for (int i = 1; i < RUN; ++i) s = fma2(x[i], x[i], s);
    return rsqrtf(fmaf(sum_of<LPV>(s.x + s.y), p.inv_D, p.eps));
}

// The page of a token and its place in it (page -1: it is not written), and its position.  A lane per token.
struct Spot {
    int32_t page, off, pos;            // page -1: not written
};
__device__ __forceinline__ Spot spot_of(const CacheParams& w, int32_t t) {
    Spot at = {-1, 0, 0};
    int32_t seq = t, back = 1;                         // the token is the back-th from the end of its sequence
    if (w.cu) {
        if (t < w.cu[0] || t >= w.cu[w.n_seqs]) return at;
        int32_t lo = 0, hi = w.n_seqs;                 // cu[lo] <= t < cu[hi]
        while (hi - lo > 1) {
            const int32_t m = lo + (hi - lo) / 2;
            if (w.cu[m] <= t) lo = m; else hi = m;
        }
        seq = lo;
        back = w.cu[lo + 1] - t;
    }
    const int32_t row = w.seq_rows ? w.seq_rows[seq] : seq;
    if (row < 0 || row >= w.rows) return at;
    const int32_t place = w.len[row] - back;
    at.pos = max(place, 0);
    if (place < 0 || (place >> w.shift) >= w.width || (w.status && w.status[row])) return at;
    at.page = w.table[size_t(row) * w.width + (place >> w.shift)];
    at.off = place & (w.page_size - 1);
    if (at.page >= w.pages) at.page = -1;
    return at;
}

// How the vectors are dealt out: a warp has `per` steps (of SIDE vectors each) of one kind of `tokens` tokens.
struct Cut {
    int64_t end[3];                    // warps up to the last of queries, keys, values
    int32_t per[3], chunks[3], tokens[3];
};
struct Share {
    int kind, h0, h1;                  // vectors h0 .. h1-1 of it
    int32_t t0, tokens;                // of tokens t0, t0 + 1, ...
};
__device__ __forceinline__ bool share_of(const Cut& cut, const RopeParams& p, int64_t id, int side_by_side, Share* s) {
    const int kind = id < cut.end[0] ? 0 : id < cut.end[1] ? 1 : 2;
    if (id >= cut.end[2]) return false;
    id -= kind == 0 ? 0 : kind == 1 ? cut.end[0] : cut.end[1];
    const int chunks = kind == 0 ? cut.chunks[0] : kind == 1 ? cut.chunks[1] : cut.chunks[2];
    const int per = (kind == 0 ? cut.per[0] : kind == 1 ? cut.per[1] : cut.per[2]) * side_by_side;
    s->kind = kind;
    const int tokens = kind == 0 ? cut.tokens[0] : kind == 1 ? cut.tokens[1] : cut.tokens[2];
    s->t0 = int32_t(id / chunks * tokens);
    s->tokens = min(tokens, p.n - s->t0);
    s->h0 = int(id % chunks) * per;
    s->h1 = min(kind == 0 ? p.heads[0] : kind == 1 ? p.heads[1] : p.heads[2], s->h0 + per);
    return true;
}

// HELD: -1 without a cache, else how it holds its vectors.  Blocks of one warp: all that is the same for its lanes then goes by the block's number
// and through the uniform registers (four warps to a block: 7 % longer for 16384 tokens x 40 heads).
template <typename T, int LPV, int RUN, int HELD>
__global__ void __launch_bounds__(32, FORWARD_WARPS) norm_rope_kernel(const RopeParams p, const CacheParams w, const Cut cut) {
    let_later_in();
    wait_for_earlier();
    constexpr int STEP = step_bytes<RUN>();
    __shared__ __align__(16) unsigned char ring[DEPTH * STEP];
    __shared__ Turns turns;
    constexpr int SIDE = 32 / LPV;     // vectors side by side
    constexpr bool CACHE = HELD >= 0;
    const int lane = threadIdx.x, c = lane % LPV, side = lane / LPV;
    Share sh;
    if (!share_of(cut, p, blockIdx.x, SIDE, &sh)) return;
    const int kind = sh.kind;
    const Place at = place_of<RUN>(p, c);
    const bool rotated = p.rot > 0 && kind < 2, normed = p.norm && kind < 2;
    const int steps = (sh.h1 - sh.h0 + SIDE - 1) / SIDE;           // of a token

    // loads, DEPTH - 1 steps ahead
    const uint32_t ring_at = smem_u32(ring);
    const Vectors src = CACHE ? pick(p.x, kind) : pick2(p.x, kind);
    const unsigned char* in = src.at + sh.t0 * src.token + (sh.h0 + side) * src.head;
    const int64_t in_step = SIDE * src.head, in_token = src.token - steps * in_step;
    int in_h = sh.h0 + side, left = sh.tokens * steps;             // steps not yet asked for
    uint32_t in_at = 0, at_step = 0;   // places in the ring
    auto fetch = [&]() {
        if (left > 0) {
            // for lanes without a vector any address will do: nothing is read
            const bool some = at.some && in_h < sh.h1;
            copy_in<RUN>(ring_at + in_at, some ? in : src.at, at, some, lane);
            --left;
            in += in_step;
            in_h += SIDE;
            if (in_h - side >= sh.h1) {
                in += in_token;
                in_h = sh.h0 + side;
            }
        }
        commit();
        in_at = in_at == (DEPTH - 1) * STEP ? 0 : in_at + STEP;
    };
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) fetch();

    Spot spots = {-1, 0, 0};           // of the lane-th token
    if (lane < sh.tokens) {
        const int32_t t = sh.t0 + lane;
        if (CACHE) spots = spot_of(w, t);
        if (rotated && p.pos) spots.pos = p.pos[t];
    }
    Frequencies freq;
    if (rotated) freq = frequencies_of(p, lane);

    float2 P[RUN], Q[RUN];
    const bool to_cache = CACHE && kind > 0;
    const Vectors dst = CACHE ? p.y[0] : pick2(p.y, kind);
    const int64_t out_step = to_cache ? int64_t(SIDE) * w.head_bytes : SIDE * dst.head;
    unsigned char* out = nullptr;
    int32_t off = 0;
    bool written = true;
    const int64_t page_bytes = to_cache ? int64_t(p.heads[1]) * w.head_bytes : 0, first_out = to_cache ? int64_t(sh.h0 + side) * w.head_bytes : (sh.h0 + side) * dst.head;
    unsigned char* const plane = CACHE ? (kind == 2 ? w.plane[1] : w.plane[0]) : nullptr;
    int h = sh.h1 + side;              // at a token's end: the next begins
    int from = -1;                     // which of the warp's tokens
    for (int todo = sh.tokens * steps; todo > 0; --todo) {
        if (h - side >= sh.h1) {
            ++from;
            h = sh.h0 + side;
            if (to_cache) {
                const int32_t page = __shfl_sync(FULL, spots.page, from);
                off = __shfl_sync(FULL, spots.off, from);
                written = page >= 0;
                out = plane + max(page, 0) * page_bytes + first_out;
            } else {
                out = dst.at + (int64_t(sh.t0) + from) * dst.token + first_out;
            }
            if (rotated) turn_to(p, __shfl_sync(FULL, spots.pos, from), freq, turns, lane);
            // what the weights and the angles come to, where they change
            if (rotated || (normed && from == 0)) {
                float2 f[RUN];
                load_weights<T, RUN>(p, kind, at, f);
                if (at.turned) {
                    coefficients<RUN>(turns, c, f, p.interleaved, P, Q);
                } else {
#pragma unroll
                    for (int j = 0; j < RUN; ++j) P[j] = f[j];
                }
            }
        }
        wait_for_all_but<DEPTH - 2>();
        Raw<RUN> y = load_raw<RUN>(ring + at_step + lane * (RUN * 2), ring + at_step + (32 + lane) * (RUN * 2));
        at_step = at_step == (DEPTH - 1) * STEP ? 0 : at_step + STEP;
        fetch();
        if (normed || rotated) {
            float2 x[RUN];
            unpack<T, RUN>(y, x);
            if (normed) {
                const float r = inverse_norm<LPV, RUN>(p, x);
#pragma unroll
                for (int j = 0; j < RUN; ++j) x[j] = mul2(x[j], make_float2(r, r));
            }
            if (at.turned && rotated) {
                turn<RUN>(x, P, Q, p.interleaved);
            } else if (normed) {
#pragma unroll
                for (int j = 0; j < RUN; ++j) x[j] = mul2(x[j], P[j]);
            }
            y = pack<T, RUN>(x);
        }
        const bool real = h < sh.h1 && at.some;
        if (!to_cache) {
            if (real) store_raw<RUN>(out, at, y);
        } else if (HELD <= HELD_PLAIN) {
            if (real && written) store_raw<RUN>(out + off * w.token_bytes, at, y);
        } else {
            // what is held is a vector of the type T
            float inv;
            const int e = hold_exponent<HELD>(largest_bits<T, LPV, RUN>(y.w), &inv);
            float2 x[RUN];
            unpack<T, RUN>(y, x);
            uint32_t code[RUN / 2];
#pragma unroll
            for (int j = 0; j < RUN / 2; ++j) code[j] = hold4<HELD>(x[2 * j], x[2 * j + 1], inv);
            if (e == NAN_EXP) {
#pragma unroll
                for (int j = 0; j < RUN / 2; ++j) code[j] = 0;
            }
            if (real && written) {
                unsigned char* to = out + off * p.D;
                if constexpr (RUN == 8) {
                    *reinterpret_cast<uint2*>(to + at.a) = make_uint2(code[0], code[1]);
                    *reinterpret_cast<uint2*>(to + at.b) = make_uint2(code[2], code[3]);
                } else {
                    *reinterpret_cast<uint32_t*>(to + at.a) = code[0];
                    *reinterpret_cast<uint32_t*>(to + at.b) = code[1];
                }
                if (c == 0) out[w.page_size * p.D + off] = uint8_t(e);
            }
        }
        h += SIDE;
        out += out_step;
    }
}

// ---- gradient ------------------------------------------------------------------------------------------
// x: the inputs, y: the gradient of the outputs, dx: contiguous.  A block's warps work on one kind, go through its tokens' vectors in a
// fixed order and keep the weights' gradients of their lanes; a block leaves one sum for each weight in part[block][D].
template <typename T, int LPV, int RUN>
__global__ void __launch_bounds__(THREADS, GRAD_BLOCKS) norm_rope_grad_kernel(const RopeParams p, unsigned char* dq, unsigned char* dk, float* part, int q_blocks,
                                                                           const Cut cut) {
    let_later_in();
    wait_for_earlier();
    constexpr int STEP = step_bytes<RUN>();
    __shared__ __align__(16) unsigned char s_ring[WARPS][GRAD_DEPTH * 2 * STEP];
    __shared__ Turns s_turns[WARPS];
    __shared__ float sums[WARPS][128];
    constexpr int SIDE = 32 / LPV;
    const int lane = threadIdx.x & 31, warp = __shfl_sync(FULL, int(threadIdx.x >> 5), 0), c = lane % LPV, side = lane / LPV;
    Turns& turns = s_turns[warp];
    const Place at = place_of<RUN>(p, c);
    const int kind = int(blockIdx.x) < q_blocks ? 0 : 1, heads = kind ? p.heads[1] : p.heads[0];
    const int chunks = kind ? cut.chunks[1] : cut.chunks[0], per = (kind ? cut.per[1] : cut.per[0]) * SIDE;
    const int64_t items = int64_t(p.n) * chunks, stride = int64_t(kind ? gridDim.x - q_blocks : q_blocks) * WARPS;
    const int64_t first = int64_t(kind ? blockIdx.x - q_blocks : blockIdx.x) * WARPS + warp;
    const Vectors xs = pick2(p.x, kind), gs = pick2(p.y, kind);
    const bool rotated = p.rot > 0;
    Frequencies freq;
    if (rotated) freq = frequencies_of(p, lane);
    float2 f[RUN], acc[RUN];
    load_weights<T, RUN>(p, kind, at, f);
#pragma unroll
    for (int j = 0; j < RUN; ++j) acc[j] = make_float2(0.f, 0.f);

    // loads, GRAD_DEPTH - 1 steps ahead: vectors and gradients
    unsigned char* ring = s_ring[warp];
    const uint32_t ring_at = smem_u32(ring);
    int64_t in_id = first;
    const unsigned char *in_x = xs.at, *in_g = gs.at;
    int in_h = 0, in_last = 0;
    uint32_t in_at = 0, at_step = 0;
    auto begin = [&]() {
        in_last = 0;
        if (in_id < items) {
            const int32_t t = int32_t(in_id / chunks);
            in_h = int(in_id % chunks) * per;
            in_last = min(heads, in_h + per);
            in_h += side;
            in_x = xs.at + t * xs.token + in_h * xs.head;
            in_g = gs.at + t * gs.token + in_h * gs.head;
        }
    };
    auto fetch = [&]() {
        if (in_last > 0) {             // by the whole warp
            const bool some = at.some && in_h < in_last;
            copy_in<RUN>(ring_at + in_at, some ? in_x : xs.at, at, some, lane);
            copy_in<RUN>(ring_at + in_at + STEP, some ? in_g : gs.at, at, some, lane);
            in_h += SIDE;
            in_x += SIDE * xs.head;
            in_g += SIDE * gs.head;
            if (in_h - side >= in_last) {
                in_id += stride;
                begin();
            }
        }
        commit();
        in_at = in_at == (GRAD_DEPTH - 1) * 2 * STEP ? 0 : in_at + 2 * STEP;
    };
    begin();
#pragma unroll
    for (int i = 0; i < GRAD_DEPTH - 1; ++i) fetch();
    for (int64_t id = first; id < items; id += stride) {
        const int32_t t = int32_t(id / chunks);
        const int h0 = int(id % chunks) * per, h1 = min(heads, h0 + per);
        float cs[RUN], sn[RUN];
        if (rotated) {
            turn_to(p, p.pos[t], freq, turns, lane);
            if (at.turned) read_turns<RUN>(turns, c, cs, sn);
        }
        unsigned char* to = (kind ? dk : dq) + (int64_t(t) * heads + h0 + side) * p.D * 2;
        for (int h = h0 + side; h - side < h1; h += SIDE, to += SIDE * p.D * 2) {
            float2 x[RUN], g[RUN];
            wait_for_all_but<GRAD_DEPTH - 2>();
            const unsigned char* mine = ring + at_step + lane * (RUN * 2);
            unpack<T, RUN>(load_raw<RUN>(mine, mine + 32 * RUN * 2), x);
            unpack<T, RUN>(load_raw<RUN>(mine + STEP, mine + STEP + 32 * RUN * 2), g);
            at_step = at_step == (GRAD_DEPTH - 1) * 2 * STEP ? 0 : at_step + 2 * STEP;
            fetch();
            if (rotated && at.turned) turn_back<RUN>(g, cs, sn, p.interleaved);
            if (p.norm) {
                const float r = inverse_norm<LPV, RUN>(p, x);
                // vectors that are not there are zeros, but 0 times an infinite r (eps = 0) is not
                const float ra = h < h1 ? r : 0.f;
                float2 dot = make_float2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < RUN; ++j) {
                    x[j] = mul2(x[j], make_float2(ra, ra));
                    acc[j] = fma2(g[j], x[j], acc[j]);
                    g[j] = mul2(g[j], f[j]);
                    dot = fma2(g[j], x[j], dot);
                }
                const float m = -sum_of<LPV>(dot.x + dot.y) * p.inv_D;
#pragma unroll
                for (int j = 0; j < RUN; ++j) g[j] = mul2(fma2(x[j], make_float2(m, m), g[j]), make_float2(r, r));
            }
            if (h < h1 && at.some) store_raw<RUN>(to, at, pack<T, RUN>(g));
        }
    }
    if (!part) return;
#pragma unroll
    for (int j = 0; j < RUN; ++j) {
#pragma unroll
        for (int o = LPV; o < 32; o <<= 1) {
            acc[j].x += __shfl_xor_sync(FULL, acc[j].x, o);
            acc[j].y += __shfl_xor_sync(FULL, acc[j].y, o);
        }
        if (lane < LPV && at.some) {
            const int d = j < RUN / 2 ? at.a + 2 * j : at.b + 2 * j - RUN;
            sums[warp][d] = acc[j].x;
            sums[warp][d + 1] = acc[j].y;
        }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < p.D; d += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += sums[w][d];
        part[int64_t(blockIdx.x) * p.D + d] = s;
    }
}
// the blocks' sums, in a fixed order: a block of threads per 32 weights, 32 runs of blocks side by side
__global__ void __launch_bounds__(1024) weight_grad_kernel(const float* part, int q_blocks, int blocks, int D, float* dqw, float* dkw) {
    let_later_in();
    wait_for_earlier();
    __shared__ float sums[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, groups = (D + 31) / 32, kind = blockIdx.x / groups, d = blockIdx.x % groups * 32 + x;
    float s = 0.f;
    if (d < D)
        for (int b = (kind ? q_blocks : 0) + y; b < (kind ? blocks : q_blocks); b += 32) s += part[int64_t(b) * D + d];
    sums[y][x] = s;
    __syncthreads();
    if (y == 0 && d < D) {
        s = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) s += sums[r][x];
        float* to = kind ? dkw : dqw;
        if (to) to[d] = s;
    }
}

// ---- launches ------------------------------------------------------------------------------------------
// Runs of 8 values where both halves of what is rotated and the whole vector are made of them.
bool long_runs(int32_t D, int32_t rot) { return D % 16 == 0 && rot % 16 == 0; }
int side_by_side(int32_t D, int32_t rot) { return (D <= 64 ? 4 : 2) * (long_runs(D, rot) ? 2 : 1); }

// Equal shares of all steps for the warps that run at a time, as long as that is at least two steps and at most MOST_STEPS (then several
// shares one after the other): with many steps the warps that end late are then short ones (16384 tokens x 40 heads: with one round of 55
// steps 6 % longer, with 4 steps, half of a token's queries, 12 %).  A share is several tokens, or a part of one.
Cut cut_of(int64_t n, const int32_t* heads, int side, int64_t warps) {
    Cut cut = {};
    int64_t steps[3], all = 0, end = 0;
    for (int k = 0; k < 3; ++k) all += n * (steps[k] = (heads[k] + side - 1) / side);
    int64_t share = (all + warps - 1) / warps;
    share = share < 2 ? 2 : share > MOST_STEPS ? MOST_STEPS : share;
    for (int k = 0; k < 3; ++k) {
        cut.tokens[k] = cut.per[k] = 1;
        if (steps[k] > 0) {
            const int64_t chunks = steps[k] / share > 1 ? steps[k] / share : 1, tokens = (share + steps[k] - 1) / steps[k];
            cut.tokens[k] = int32_t(chunks > 1 ? 1 : tokens > MOST_TOKENS ? MOST_TOKENS : tokens);
            cut.per[k] = int32_t((steps[k] + chunks - 1) / chunks);
        }
        cut.chunks[k] = int32_t((steps[k] + cut.per[k] - 1) / cut.per[k]);
        end += (n + cut.tokens[k] - 1) / cut.tokens[k] * cut.chunks[k];
        cut.end[k] = end;
    }
    return cut;
}

template <typename T, int HELD>
int launch(const RopeParams& p, const CacheParams& w, cudaStream_t st) {
    const Cut cut = cut_of(p.n, p.heads, side_by_side(p.D, p.rot), SMS * FORWARD_WARPS);
    if (cut.end[2] >= (int64_t(1) << 31)) return DISC_ERR_UNSUPPORTED;
    auto kernel = long_runs(p.D, p.rot) ? (p.D <= 64 ? norm_rope_kernel<T, 4, 8, HELD> : norm_rope_kernel<T, 8, 8, HELD>)
                                        : (p.D <= 64 ? norm_rope_kernel<T, 8, 4, HELD> : norm_rope_kernel<T, 16, 4, HELD>);
    return launch_after(kernel, unsigned(cut.end[2]), 32, 0, st, p, w, cut);
}
template <int HELD>
int launch(int type, const RopeParams& p, const CacheParams& w, cudaStream_t st) {
    return type == DISC_BF16 ? launch<__nv_bfloat16, HELD>(p, w, st) : launch<__half, HELD>(p, w, st);
}
int launch_cache(const disc_cache_t* c, const RopeParams& p, const CacheParams& w, cudaStream_t st) {
    const int held = cache_held(c), type = cache_type(c);
    return held == HELD_PLAIN ? launch<HELD_PLAIN>(type, p, w, st) : held == HELD_E4M3 ? launch<HELD_E4M3>(type, p, w, st) : launch<HELD_I8>(type, p, w, st);
}

bool misaligned(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) != 0; }

// what is done to the vectors; DISC_OK and p filled in, or an error
int check_how(const disc_norm_rope_t* a, int32_t dtype, int32_t D, RopeParams* p) {
    if (dtype != DISC_BF16 && dtype != DISC_F16) return DISC_ERR_UNSUPPORTED;
    if (D <= 0 || a->rot < 0 || a->rot > D || (a->rot > 0 && !a->inv_freq)) return DISC_ERR_ARG;
    if (D % 8 || D > DISC_MAX_HEAD_DIM || a->rot % 8) return DISC_ERR_UNSUPPORTED;
    if (a->norm && !(a->eps >= 0.f && a->eps <= 3.0e38f)) return DISC_ERR_ARG;
    const bool weights = a->norm && (a->q_weight || a->k_weight);
    if (weights && a->weight_dtype != DISC_F32 && a->weight_dtype != dtype) return DISC_ERR_UNSUPPORTED;
    if (weights && (misaligned(a->q_weight) || misaligned(a->k_weight))) return DISC_ERR_ARG;
    if (a->n_q_heads < 0 || a->n_q_heads > (1 << 16) || a->n_kv_heads < 0 || a->n_kv_heads > (1 << 16) || a->n_tokens < 0 || a->n_tokens > (int64_t(1) << 30)) return DISC_ERR_ARG;
    p->D = D; p->rot = a->rot; p->interleaved = a->interleaved != 0; p->norm = a->norm != 0;
    p->weights_f32 = a->weight_dtype == DISC_F32;
    p->w[0] = p->norm ? a->q_weight : nullptr; p->w[1] = p->norm ? a->k_weight : nullptr;
    p->inv_D = 1.f / float(D);
    p->eps = a->eps; p->inv_freq = a->inv_freq; p->pos = a->positions; p->n = int32_t(a->n_tokens);
    return DISC_OK;
}
// vectors [n][heads][D]: 16-byte boundaries, strides multiples of 8 values
int check_vectors(const void* x, int64_t token, int64_t head, int64_t n, int32_t heads, Vectors* v) {
    *v = Vectors{nullptr, 0, 0};
    if (heads == 0) return DISC_OK;
    if (!x || misaligned(x)) return DISC_ERR_ARG;
    if (n == 1) token = 0;
    if (heads == 1) head = 0;
    if ((token | head) & 7) return DISC_ERR_UNSUPPORTED;
    *v = Vectors{static_cast<unsigned char*>(const_cast<void*>(x)), token * 2, head * 2};
    return DISC_OK;
}

// An output may lie on its own input, place for place; on another one it would be written while that is still read.  Told by where they begin.
int check_places(const RopeParams& p) {
    for (int k = 0; k < 2; ++k) {
        const Vectors &y = p.y[k], &x = p.x[k];
        if (!y.at) continue;
        if (y.at == x.at && (y.token != x.token || y.head != x.head)) return DISC_ERR_ARG;
        if (y.at == p.x[1 - k].at || y.at == p.x[2].at || y.at == p.y[1 - k].at) return DISC_ERR_ARG;
    }
    return DISC_OK;
}

void cache_params(const disc_cache_t* c, int32_t layer, const int32_t* cu, int32_t n_seqs, const int32_t* rows, const uint8_t* status, CacheParams* w) {
    w->plane[0] = static_cast<unsigned char*>(c->pool) + 2 * int64_t(layer) * cache_plane_bytes(c);
    w->plane[1] = w->plane[0] + cache_plane_bytes(c);
    w->table = c->table; w->len = c->len; w->rows = c->n_rows; w->width = c->table_width; w->pages = c->n_pages; w->page_size = c->page_size;
    w->shift = 0;
    while ((1 << w->shift) < c->page_size) ++w->shift;
    w->held = cache_held(c); w->token_bytes = cache_token_bytes(c); w->head_bytes = cache_head_bytes(c);
    w->cu = cu; w->seq_rows = rows; w->status = status; w->n_seqs = n_seqs;
}

// The gradient's items and blocks for each kind of vectors.  An item: the vectors of a kind of a token, or, with few tokens, a part of them,
// so that there are four items for a warp.
struct GradCut {
    Cut cut;
    int64_t items[2];
    int q_blocks, blocks;
};
GradCut grad_items(int64_t n, int32_t hq, int32_t hkv, int side) {
    GradCut g = {};
    const int32_t heads[2] = {hq, hkv};
    const int64_t wanted = n > 0 ? (int64_t(MAX_GRAD_BLOCKS) * WARPS * 4 + n - 1) / n : 1;
    for (int k = 0; k < 2; ++k) {
        const int steps = (heads[k] + side - 1) / side, chunks = wanted < (steps + 1) / 2 ? int(wanted) : (steps + 1) / 2;
        g.cut.per[k] = chunks ? (steps + chunks - 1) / chunks : 1;
        g.cut.chunks[k] = (steps + g.cut.per[k] - 1) / g.cut.per[k];
        g.items[k] = n * g.cut.chunks[k];
    }
    // as many blocks as there can be
    const int64_t need = (g.items[0] + WARPS - 1) / WARPS + (g.items[1] + WARPS - 1) / WARPS;
    g.blocks = int(need < MAX_GRAD_BLOCKS ? need : MAX_GRAD_BLOCKS);
    return g;
}
GradCut grad_cut(int64_t n, int32_t hq, int32_t hkv, int side) {
    GradCut g = grad_items(n, hq, hkv, side);
    const int64_t need_q = (g.items[0] + WARPS - 1) / WARPS, need_k = (g.items[1] + WARPS - 1) / WARPS;
    if (need_q + need_k <= MAX_GRAD_BLOCKS) {
        g.q_blocks = int(need_q);
        return g;
    }
    // dealt out so that the kind whose warps end last ends soonest; beginning an item costs as much as a step and a half
    const double cost[2] = {g.cut.per[0] + 1.5, g.cut.per[1] + 1.5};
    double best = 1e300;
    g.q_blocks = hkv ? 0 : MAX_GRAD_BLOCKS;
    for (int x = 4; hq && hkv && x < MAX_GRAD_BLOCKS; x += 8) {
        const double cq = ceil(double(g.items[0]) / (x * WARPS)) * cost[0], ck = ceil(double(g.items[1]) / ((MAX_GRAD_BLOCKS - x) * WARPS)) * cost[1];
        const double end = cq > ck ? cq : ck;
        if (end < best) { best = end; g.q_blocks = x; }
    }
    return g;
}

}  // namespace

extern "C" {

int disc_norm_rope(const disc_norm_rope_t* a, void* stream) {
    RopeParams p = {};
    if (!a) return DISC_ERR_ARG;
    if (const int rc = check_how(a, a->dtype, a->head_dim, &p)) return rc;
    const int64_t n = a->n_tokens;
    if (a->n_q_heads + a->n_kv_heads == 0) return DISC_ERR_ARG;
    if (n == 0) return DISC_OK;
    if (p.rot > 0 && !a->positions) return DISC_ERR_ARG;
    if (const int rc = check_vectors(a->q, a->q_token, a->q_head, n, a->n_q_heads, &p.x[0])) return rc;
    if (const int rc = check_vectors(a->k, a->k_token, a->k_head, n, a->n_kv_heads, &p.x[1])) return rc;
    if (const int rc = check_vectors(a->q_out, a->q_out_token, a->q_out_head, n, a->n_q_heads, &p.y[0])) return rc;
    if (const int rc = check_vectors(a->k_out, a->k_out_token, a->k_out_head, n, a->n_kv_heads, &p.y[1])) return rc;
    if (const int rc = check_places(p)) return rc;
    p.heads[0] = a->n_q_heads; p.heads[1] = a->n_kv_heads;
    return launch<-1>(a->dtype, p, CacheParams{}, static_cast<cudaStream_t>(stream));
}

int disc_norm_rope_write(const disc_cache_t* c, int32_t layer, const disc_norm_rope_t* a, void* stream) {
    if (!a || !c || !c->pool || !c->table || !c->len) return DISC_ERR_ARG;
    if (const int rc = disc::cache_sizes(c)) return rc;
    RopeParams p = {};
    if (const int rc = check_how(a, cache_type(c), c->head_dim, &p)) return rc;
    const int64_t n = a->n_tokens;
    if (layer < 0 || layer >= c->n_layers || a->n_seqs < 0 || a->dtype != cache_type(c) || a->head_dim != c->head_dim || a->n_kv_heads != c->n_kv_heads) return DISC_ERR_ARG;
    if (!a->cu && n != a->n_seqs) return DISC_ERR_ARG;
    if (!a->rows && a->n_seqs > c->n_rows) return DISC_ERR_ARG;
    if (n == 0 || a->n_seqs == 0) return DISC_OK;
    if (const int rc = check_vectors(a->q, a->q_token, a->q_head, n, a->n_q_heads, &p.x[0])) return rc;
    if (const int rc = check_vectors(a->k, a->k_token, a->k_head, n, c->n_kv_heads, &p.x[1])) return rc;
    if (const int rc = check_vectors(a->v, a->v_token, a->v_head, n, c->n_kv_heads, &p.x[2])) return rc;
    if (const int rc = check_vectors(a->q_out, a->q_out_token, a->q_out_head, n, a->n_q_heads, &p.y[0])) return rc;
    if (const int rc = check_places(p)) return rc;
    p.heads[0] = a->n_q_heads; p.heads[1] = p.heads[2] = c->n_kv_heads;
    CacheParams w;
    cache_params(c, layer, a->cu, a->n_seqs, a->rows, a->status, &w);
    return launch_cache(c, p, w, static_cast<cudaStream_t>(stream));
}

int64_t disc_norm_rope_scratch_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_tokens) {
    if (n_q_heads < 0 || n_kv_heads < 0 || n_q_heads > (1 << 16) || n_kv_heads > (1 << 16) || n_q_heads + n_kv_heads == 0 || head_dim <= 0 || head_dim > DISC_MAX_HEAD_DIM || n_tokens < 0 || n_tokens > (int64_t(1) << 30))
        return DISC_ERR_ARG;
    const int a = grad_items(n_tokens, n_q_heads, n_kv_heads, side_by_side(head_dim, 0)).blocks, b = grad_items(n_tokens, n_q_heads, n_kv_heads, side_by_side(head_dim, 8)).blocks;
    return int64_t(a > b ? a : b) * head_dim * 4;
}

int disc_norm_rope_grad(const disc_norm_rope_t* a, void* d_q, void* d_k, float* d_q_weight, float* d_k_weight, void* scratch, int64_t scratch_bytes, void* stream) {
    RopeParams p = {};
    if (!a) return DISC_ERR_ARG;
    if (const int rc = check_how(a, a->dtype, a->head_dim, &p)) return rc;
    const int32_t head_dim = a->head_dim, n_q_heads = a->n_q_heads, n_kv_heads = a->n_kv_heads;
    const int64_t n_tokens = a->n_tokens, need = disc_norm_rope_scratch_bytes(n_q_heads, n_kv_heads, head_dim, n_tokens);
    if (need < 0) return int(need);
    if (n_tokens > 0 && p.rot > 0 && !a->positions) return DISC_ERR_ARG;
    const bool weights = d_q_weight || d_k_weight;
    if (weights && (!p.norm || (n_tokens > 0 && (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 3u) || scratch_bytes < need)))) return DISC_ERR_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n_tokens == 0) {
        if (d_q_weight) DISC_CUDA(cudaMemsetAsync(d_q_weight, 0, size_t(head_dim) * 4, st));
        if (d_k_weight) DISC_CUDA(cudaMemsetAsync(d_k_weight, 0, size_t(head_dim) * 4, st));
        return DISC_OK;
    }
    if (const int rc = check_vectors(a->q, a->q_token, a->q_head, n_tokens, n_q_heads, &p.x[0])) return rc;
    if (const int rc = check_vectors(a->k, a->k_token, a->k_head, n_tokens, n_kv_heads, &p.x[1])) return rc;
    if (const int rc = check_vectors(a->q_out, a->q_out_token, a->q_out_head, n_tokens, n_q_heads, &p.y[0])) return rc;
    if (const int rc = check_vectors(a->k_out, a->k_out_token, a->k_out_head, n_tokens, n_kv_heads, &p.y[1])) return rc;
    if ((n_q_heads && (!d_q || misaligned(d_q))) || (n_kv_heads && (!d_k || misaligned(d_k)))) return DISC_ERR_ARG;
    p.heads[0] = n_q_heads; p.heads[1] = n_kv_heads;
    const GradCut g = grad_cut(n_tokens, n_q_heads, n_kv_heads, side_by_side(head_dim, p.rot));
    float* part = weights ? static_cast<float*>(scratch) : nullptr;
    const bool bf = a->dtype == DISC_BF16, small = head_dim <= 64;
    auto kernel = long_runs(head_dim, p.rot) ? (bf ? (small ? norm_rope_grad_kernel<__nv_bfloat16, 4, 8> : norm_rope_grad_kernel<__nv_bfloat16, 8, 8>)
                                                   : (small ? norm_rope_grad_kernel<__half, 4, 8> : norm_rope_grad_kernel<__half, 8, 8>))
                                             : (bf ? (small ? norm_rope_grad_kernel<__nv_bfloat16, 8, 4> : norm_rope_grad_kernel<__nv_bfloat16, 16, 4>)
                                                   : (small ? norm_rope_grad_kernel<__half, 8, 4> : norm_rope_grad_kernel<__half, 16, 4>));
    if (const int rc = launch_after(kernel, unsigned(g.blocks), THREADS, 0, st, p, static_cast<unsigned char*>(d_q), static_cast<unsigned char*>(d_k), part, g.q_blocks, g.cut)) return rc;
    if (!weights) return DISC_OK;
    return launch_after(weight_grad_kernel, unsigned(2 * ((head_dim + 31) / 32)), 1024, 0, st, static_cast<const float*>(part), g.q_blocks, g.blocks, int(head_dim), d_q_weight, d_k_weight);
}

}  // extern "C"
