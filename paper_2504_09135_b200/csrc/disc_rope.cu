// Queries and keys on their way to attention: each head's RMS norm and the rotation by the token's position in one pass
// (disc_norm_rope), its gradient (disc_norm_rope_grad), and, with the keys and values going straight into a cache's pages,
// disc_norm_rope_write.  The last is also how a cache held in 8 bits is written (disc_cache_write).
//
//   u = w x r,  r = 1 / sqrt(mean(x^2) + eps);   y_a = u_a cos t_i - u_b sin t_i,  y_b = u_b cos t_i + u_a sin t_i,
//   t_i = position inv_freq_i,  (a, b) = (i, i + rot / 2) or (2 i, 2 i + 1)
//
// Backward, with g = dy rotated by -t and c = w g:  dw = sum g x r,  dx = r c - x r^3 mean(c x).
//
// Bound by the bytes: every vector is read once and written once.  8 or 16 lanes hold a vector, 8 values each, so that a pair
// that is rotated lies in one lane and the sum of squares is three or four shuffles; a warp has the vectors of one token, four
// loads of each lane in flight.  The angles of a lane's four pairs are formed once for the token's vectors: position x
// inv_freq / 2 pi in 64 bits, less its whole turns, so that a position of a million is as exact as one of ten (in 32 bits its
// angle is off by 0.03), then sin and cos of a fraction of a turn in 32 bits.

#include "disc_held.cuh"

namespace {

using namespace disc;

constexpr unsigned FULL = 0xffffffffu;
constexpr int THREADS = 128;
constexpr int AT_ONCE = 4;             // vectors of a lane in flight
constexpr int MAX_BLOCKS = 148 * 8;    // of the gradient, whose blocks each leave sums of their own

struct Vectors {                       // strides in bytes
    unsigned char* at;
    int64_t token, head;
};
struct RopeParams {
    Vectors x[3];                      // queries, keys; values, which are only written
    Vectors y[2];
    int32_t n, D, rot, interleaved, norm, weights_f32;
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
__device__ __forceinline__ Vectors pick(const Vectors* v, int which) { return which == 0 ? v[0] : which == 1 ? v[1] : v[2]; }
__device__ __forceinline__ Vectors pick2(const Vectors* v, int which) { return which == 0 ? v[0] : v[1]; }

// Where a lane's two runs of four values begin.  Rotated: the four pairs (a + i, b + i), or (a, a+1), (a+2, a+3), (b, b+1), (b+2, b+3).
struct Place {
    int32_t a, b;
    bool some, turned;
};
__device__ __forceinline__ Place place_of(const RopeParams& p, int c) {
    Place at;
    at.some = c * 8 < p.D;
    at.turned = c * 8 < p.rot;
    const bool split = at.turned && !p.interleaved;
    at.a = split ? 4 * c : 8 * c;
    at.b = split ? p.rot / 2 + 4 * c : 8 * c + 4;
    return at;
}
__device__ __forceinline__ void angles(const RopeParams& p, int32_t pos, int c, float* cs, float* sn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        double turns = double(pos) * (double(p.inv_freq[4 * c + i]) * 0.15915494309189533577);
        turns -= rint(turns);
        sincospif(2.f * float(turns), sn + i, cs + i);
    }
}
// by the angles, or back with sign = -1
__device__ __forceinline__ void turn(float* x, const float* cs, const float* sn, bool interleaved, float sign) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float s = sign * sn[i];
        float* a = interleaved ? x + 2 * i : x + i;
        float* b = interleaved ? x + 2 * i + 1 : x + 4 + i;
        const float u = *a, v = *b;
        *a = u * cs[i] - v * s;
        *b = v * cs[i] + u * s;
    }
}
template <typename T>
__device__ __forceinline__ void load8(const unsigned char* v, const Place& at, float* x) {
    const uint2 a = at.some ? *reinterpret_cast<const uint2*>(v + at.a * 2) : make_uint2(0, 0), b = at.some ? *reinterpret_cast<const uint2*>(v + at.b * 2) : make_uint2(0, 0);
    const float2 f[4] = {unpack2<T>(a.x), unpack2<T>(a.y), unpack2<T>(b.x), unpack2<T>(b.y)};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = f[i].x; x[2 * i + 1] = f[i].y; }
}
template <typename T>
__device__ __forceinline__ void store8(unsigned char* v, const Place& at, const float* x) {
    if (!at.some) return;
    *reinterpret_cast<uint2*>(v + at.a * 2) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
    *reinterpret_cast<uint2*>(v + at.b * 2) = make_uint2(pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
}
template <typename T>
__device__ __forceinline__ void load_weights(const RopeParams& p, int which, const Place& at, float* w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    const void* from = which ? p.w[1] : p.w[0];
    if (!from || !at.some) return;
    if (p.weights_f32) {
        const float* f = static_cast<const float*>(from);
        const float4 a = *reinterpret_cast<const float4*>(f + at.a), b = *reinterpret_cast<const float4*>(f + at.b);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    } else {
        load8<T>(static_cast<const unsigned char*>(from), at, w);
    }
}
template <int LPV>
__device__ __forceinline__ float sum_of(float x) {
#pragma unroll
    for (int o = 1; o < LPV; o <<= 1) x += __shfl_xor_sync(FULL, x, o);
    return x;
}
template <int LPV>
__device__ __forceinline__ float inverse_norm(const RopeParams& p, const float* x) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
    return rsqrtf(sum_of<LPV>(s) / float(p.D) + p.eps);
}

// the last i with cu[i] <= t, for cu[0] <= t < cu[n]; by a whole warp, 32 places at a time
__device__ __forceinline__ int32_t sequence_of(const int32_t* cu, int32_t n, int32_t t, int lane) {
    int32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const int32_t step = int32_t((uint32_t(hi - lo) + 31) / 32);
        const int64_t at = lo + int64_t(lane + 1) * step;
        const unsigned before = __ballot_sync(FULL, at < hi && cu[min(at, int64_t(n))] <= t);
        lo += __popc(before) * step;
        hi = hi - lo > step ? lo + step : hi;
    }
    return lo;
}

// A warp per token and LOADS x 32 / LPV of its vectors: queries, then keys, then (with a cache) values.
template <typename T, int LPV, bool CACHE>
__global__ void __launch_bounds__(THREADS) norm_rope_kernel(const RopeParams p, const CacheParams w, int chunks) {
    let_later_in();
    wait_for_earlier();
    constexpr int SIDE = 32 / LPV;     // vectors side by side
    const int lane = threadIdx.x & 31, c = lane % LPV;
    const int64_t id = int64_t(blockIdx.x) * (THREADS / 32) + (threadIdx.x >> 5);
    const int32_t t = int32_t(id / chunks);
    if (t >= p.n) return;
    const int first = int(id % chunks) * (AT_ONCE * SIDE) + lane / LPV;
    const int hq = p.heads[0], hk = hq + p.heads[1], all = CACHE ? hk + p.heads[2] : hk;
    const Place at = place_of(p, c);

    float x[AT_ONCE][8];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const int h = first + i * SIDE, which = h < hq ? 0 : h < hk ? 1 : 2;
        const Vectors v = CACHE ? pick(p.x, which) : pick2(p.x, which);
        Place here = at;
        here.some = at.some && h < all;
        load8<T>(v.at + t * v.token + (h - (which == 0 ? 0 : which == 1 ? hq : hk)) * v.head, here, x[i]);
    }

    int32_t pos = 0, page = -1, off = 0;
    if (CACHE) {
        int32_t seq = t, back = 1;                     // the token is the back-th from the end of its sequence
        bool some = true;
        if (w.cu) {
            some = t >= w.cu[0] && t < w.cu[w.n_seqs];
            if (some) {
                seq = sequence_of(w.cu, w.n_seqs, t, lane);
                back = w.cu[seq + 1] - t;
            }
        }
        const int32_t row = !some ? -1 : w.seq_rows ? w.seq_rows[seq] : seq;
        if (row >= 0 && row < w.rows) {
            const int32_t place = w.len[row] - back;
            pos = max(place, 0);
            if (place >= 0 && !(w.status && w.status[row])) {
                page = w.table[size_t(row) * w.width + (place >> w.shift)];
                off = place & (w.page_size - 1);
                if (page >= w.pages) page = -1;
            }
        }
    }
    if (!CACHE || p.pos) pos = p.pos ? p.pos[t] : 0;
    float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
    if (at.turned) angles(p, pos, c, cs, sn);

#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const int h = first + i * SIDE, which = h < hq ? 0 : h < hk ? 1 : 2;
        if (__all_sync(FULL, h >= all)) break;
        if (p.norm) {
            const float r = inverse_norm<LPV>(p, x[i]);
            float f[8];
            if (which < 2) {
                load_weights<T>(p, which, at, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = x[i][j] * r * f[j];
            }
        }
        if (at.turned && which < 2) {
            if (p.interleaved) turn(x[i], cs, sn, true, 1.f); else turn(x[i], cs, sn, false, 1.f);
        }
        const int head = h - (which == 0 ? 0 : which == 1 ? hq : hk);
        if (!CACHE || which == 0) {
            const Vectors v = CACHE ? p.y[0] : pick2(p.y, which);
            if (h < all) store8<T>(v.at + t * v.token + head * v.head, at, x[i]);
        }
        if (CACHE) {
            // by all lanes, also those whose vector is a query: the maximum is formed by shuffles
            const bool to_page = which > 0 && h < all && page >= 0;
            unsigned char* to = (which == 2 ? w.plane[1] : w.plane[0]) + (int64_t(max(page, 0)) * p.heads[1] + head) * w.head_bytes;
            if (w.held == HELD_PLAIN) {
                if (to_page) store8<T>(to + int64_t(off) * w.token_bytes, at, x[i]);
                continue;
            }
            // what is held is a vector of the type T
            uint32_t amax = 0;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2 r = unpack2<T>(pack2<T>(x[i][j], x[i][j + 1]));
                x[i][j] = r.x;
                x[i][j + 1] = r.y;
                amax = max(amax, max(__float_as_uint(r.x) & 0x7fffffffu, __float_as_uint(r.y) & 0x7fffffffu));
            }
#pragma unroll
            for (int o = 1; o < LPV; o <<= 1) amax = max(amax, __shfl_xor_sync(FULL, amax, o));
            float inv;
            const int e = w.held == HELD_E4M3 ? hold_exponent<HELD_E4M3>(amax, &inv) : hold_exponent<HELD_I8>(amax, &inv);
            const uint32_t lo = w.held == HELD_E4M3 ? hold4<HELD_E4M3>(x[i], inv) : hold4<HELD_I8>(x[i], inv);
            const uint32_t hi = w.held == HELD_E4M3 ? hold4<HELD_E4M3>(x[i] + 4, inv) : hold4<HELD_I8>(x[i] + 4, inv);
            if (to_page && at.some) {
                *reinterpret_cast<uint32_t*>(to + off * p.D + at.a) = lo;
                *reinterpret_cast<uint32_t*>(to + off * p.D + at.b) = hi;
                if (c == 0) to[w.page_size * p.D + off] = uint8_t(e);
            }
        }
    }
}

// ---- gradient ------------------------------------------------------------------------------------------
// x: the inputs, y: the gradient of the outputs, dx: contiguous.  Warps go through the tokens' vectors in a fixed order and keep the
// weights' gradients of their lanes; a block leaves one sum for each weight in part[block][2][D].
template <typename T, int LPV>
__global__ void __launch_bounds__(THREADS) norm_rope_grad_kernel(const RopeParams p, unsigned char* dq, unsigned char* dk, float* part, int chunks) {
    let_later_in();
    wait_for_earlier();
    constexpr int SIDE = 32 / LPV, WARPS = THREADS / 32, STEPS = 2;
    __shared__ float sums[WARPS][2][128];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane % LPV;
    const int hq = p.heads[0], all = hq + p.heads[1];
    const Place at = place_of(p, c);
    float acc[2][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[0][j] = acc[1][j] = 0.f;
    for (int64_t id = int64_t(blockIdx.x) * WARPS + warp; id < int64_t(p.n) * chunks; id += int64_t(gridDim.x) * WARPS) {
        const int32_t t = int32_t(id / chunks);
        const int first = int(id % chunks) * (AT_ONCE * SIDE) + lane / LPV;
        float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
        if (at.turned) angles(p, p.pos ? p.pos[t] : 0, c, cs, sn);
#pragma unroll
        for (int i0 = 0; i0 < AT_ONCE; i0 += STEPS) {
            float x[STEPS][8], g[STEPS][8];
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int h = first + (i0 + i) * SIDE, which = h < hq ? 0 : 1;
                Place here = at;
                here.some = at.some && h < all;
                const Vectors xv = pick2(p.x, which), gv = pick2(p.y, which);
                load8<T>(xv.at + t * xv.token + (h - which * hq) * xv.head, here, x[i]);
                load8<T>(gv.at + t * gv.token + (h - which * hq) * gv.head, here, g[i]);
            }
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int h = first + (i0 + i) * SIDE, which = h < hq ? 0 : 1, head = h - which * hq;
                if (at.turned) {
                    if (p.interleaved) turn(g[i], cs, sn, true, -1.f); else turn(g[i], cs, sn, false, -1.f);
                }
                if (p.norm) {
                    const float r = inverse_norm<LPV>(p, x[i]);
                    float f[8];
                    load_weights<T>(p, which, at, f);
                    float dot = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float dw = h < all ? g[i][j] * x[i][j] * r : 0.f;
                        if (which == 0) acc[0][j] += dw; else acc[1][j] += dw;
                        g[i][j] *= f[j];
                        dot = fmaf(g[i][j], x[i][j], dot);
                    }
                    const float m = sum_of<LPV>(dot) / float(p.D) * (r * r * r);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[i][j] = r * g[i][j] - x[i][j] * m;
                }
                if (h < all) store8<T>((which ? dk : dq) + (int64_t(t) * (which ? p.heads[1] : hq) + head) * p.D * 2, at, g[i]);
            }
        }
    }
    if (!part) return;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int o = LPV; o < 32; o <<= 1) acc[k][j] += __shfl_xor_sync(FULL, acc[k][j], o);
            if (lane < LPV && at.some) sums[warp][k][j < 4 ? at.a + j : at.b + j - 4] = acc[k][j];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.D; i += THREADS) {
        const int k = i / p.D, d = i % p.D;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += sums[w][k][d];
        part[(int64_t(blockIdx.x) * 2 + k) * p.D + d] = s;
    }
}
// the blocks' sums, in a fixed order: a block of threads per 32 weights, 32 runs of blocks side by side
__global__ void __launch_bounds__(1024) weight_grad_kernel(const float* part, int blocks, int D, float* dqw, float* dkw) {
    let_later_in();
    wait_for_earlier();
    __shared__ float sums[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, i = blockIdx.x * 32 + x;
    float s = 0.f;
    if (i < 2 * D)
        for (int b = y; b < blocks; b += 32) s += part[int64_t(b) * 2 * D + i];
    sums[y][x] = s;
    __syncthreads();
    if (y == 0 && i < 2 * D) {
        s = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) s += sums[r][x];
        float* to = i < D ? dqw : dkw;
        if (to) to[i % D] = s;
    }
}

// ---- launches ------------------------------------------------------------------------------------------
int chunks_of(int vectors, int D) {
    const int per = AT_ONCE * (D <= 64 ? 4 : 2);
    return (vectors + per - 1) / per;
}
template <typename T, bool CACHE>
int launch(const RopeParams& p, const CacheParams& w, cudaStream_t st) {
    const int chunks = chunks_of(p.heads[0] + p.heads[1] + (CACHE ? p.heads[2] : 0), p.D);
    const int64_t blocks = (int64_t(p.n) * chunks + THREADS / 32 - 1) / (THREADS / 32);
    if (blocks >= (int64_t(1) << 31)) return DISC_ERR_UNSUPPORTED;
    if (p.D <= 64) return launch_after(norm_rope_kernel<T, 8, CACHE>, unsigned(blocks), THREADS, 0, st, p, w, chunks);
    return launch_after(norm_rope_kernel<T, 16, CACHE>, unsigned(blocks), THREADS, 0, st, p, w, chunks);
}

bool misaligned(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) != 0; }

// what is done to the vectors; DISC_OK and p filled in, or an error
int check_how(const disc_rope_t* how, disc_dtype_t dtype, int32_t D, RopeParams* p) {
    if (!how) return DISC_ERR_ARG;
    if (dtype != DISC_BF16 && dtype != DISC_F16) return DISC_ERR_UNSUPPORTED;
    if (D <= 0 || how->rot < 0 || how->rot > D || (how->rot > 0 && !how->inv_freq)) return DISC_ERR_ARG;
    if (D % 8 || D > DISC_MAX_HEAD_DIM || how->rot % 8) return DISC_ERR_UNSUPPORTED;
    if (how->norm && !(how->eps >= 0.f && how->eps <= 3.0e38f)) return DISC_ERR_ARG;
    const bool weights = how->norm && (how->q_weight || how->k_weight);
    if (weights && how->weight_dtype != DISC_F32 && how->weight_dtype != int32_t(dtype)) return DISC_ERR_UNSUPPORTED;
    if (weights && (misaligned(how->q_weight) || misaligned(how->k_weight))) return DISC_ERR_ARG;
    p->D = D; p->rot = how->rot; p->interleaved = how->interleaved != 0; p->norm = how->norm != 0;
    p->weights_f32 = how->weight_dtype == DISC_F32;
    p->w[0] = p->norm ? how->q_weight : nullptr; p->w[1] = p->norm ? how->k_weight : nullptr;
    p->eps = how->eps; p->inv_freq = how->inv_freq;
    return DISC_OK;
}
// vectors [n][heads][D]: 16-byte boundaries, strides multiples of 8 values
int check_vectors(const void* x, int64_t token, int64_t head, int64_t n, int32_t heads, Vectors* v) {
    *v = Vectors{nullptr, 0, 0};
    if (heads == 0) return DISC_OK;
    if (!x || misaligned(x)) return DISC_ERR_ARG;
    // the stride over an axis of one is never used
    if (n == 1) token = 0;
    if (heads == 1) head = 0;
    if ((token | head) & 7) return DISC_ERR_UNSUPPORTED;
    *v = Vectors{static_cast<unsigned char*>(const_cast<void*>(x)), token * 2, head * 2};
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

int64_t grad_blocks(int64_t n, int32_t vectors, int32_t D) {
    const int64_t need = (n * chunks_of(vectors, D) + THREADS / 32 - 1) / (THREADS / 32);
    return need < MAX_BLOCKS ? need : MAX_BLOCKS;
}

}  // namespace

int disc::write_held(const disc_cache_t* c, int32_t layer, const void* k, int64_t k_token, int64_t k_head, const void* v, int64_t v_token, int64_t v_head,
                     int32_t n_tokens, const int32_t* cu, int32_t n_seqs, const int32_t* rows, const uint8_t* status, cudaStream_t st) {
    RopeParams p = {};
    CacheParams w;
    p.n = n_tokens; p.D = c->head_dim;
    p.heads[1] = p.heads[2] = c->n_kv_heads;
    p.x[1] = Vectors{static_cast<unsigned char*>(const_cast<void*>(k)), k_token * 2, k_head * 2};
    p.x[2] = Vectors{static_cast<unsigned char*>(const_cast<void*>(v)), v_token * 2, v_head * 2};
    cache_params(c, layer, cu, n_seqs, rows, status, &w);
    return cache_type(c) == DISC_BF16 ? launch<__nv_bfloat16, true>(p, w, st) : launch<__half, true>(p, w, st);
}

extern "C" {

int disc_norm_rope(const disc_rope_t* how, const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                   int64_t k_head_stride, disc_dtype_t dtype, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_tokens,
                   const int32_t* positions, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void* k_out,
                   int64_t k_out_token_stride, int64_t k_out_head_stride, void* stream) {
    RopeParams p = {};
    if (const int rc = check_how(how, dtype, head_dim, &p)) return rc;
    if (n_q_heads < 0 || n_kv_heads < 0 || n_q_heads > (1 << 16) || n_kv_heads > (1 << 16) || n_q_heads + n_kv_heads == 0 || n_tokens < 0 || n_tokens > (int64_t(1) << 30)) return DISC_ERR_ARG;
    if (n_tokens == 0) return DISC_OK;
    if (p.rot > 0 && !positions) return DISC_ERR_ARG;
    if (const int rc = check_vectors(q, q_token_stride, q_head_stride, n_tokens, n_q_heads, &p.x[0])) return rc;
    if (const int rc = check_vectors(k, k_token_stride, k_head_stride, n_tokens, n_kv_heads, &p.x[1])) return rc;
    if (const int rc = check_vectors(q_out, q_out_token_stride, q_out_head_stride, n_tokens, n_q_heads, &p.y[0])) return rc;
    if (const int rc = check_vectors(k_out, k_out_token_stride, k_out_head_stride, n_tokens, n_kv_heads, &p.y[1])) return rc;
    p.n = int32_t(n_tokens); p.heads[0] = n_q_heads; p.heads[1] = n_kv_heads; p.pos = positions;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const CacheParams none = {};
    return dtype == DISC_BF16 ? launch<__nv_bfloat16, false>(p, none, st) : launch<__half, false>(p, none, st);
}

int disc_norm_rope_write(const disc_cache_t* c, int32_t layer, const disc_rope_t* how, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                         int32_t n_q_heads, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                         int64_t v_head_stride, int64_t n_tokens, const int32_t* positions, const int32_t* cu, int32_t n_seqs, const int32_t* rows,
                         const uint8_t* status, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void* stream) {
    if (!c || !c->pool || !c->table || !c->len) return DISC_ERR_ARG;
    if (const int rc = disc::cache_sizes(c)) return rc;
    RopeParams p = {};
    if (const int rc = check_how(how, disc_dtype_t(cache_type(c)), c->head_dim, &p)) return rc;
    if (layer < 0 || layer >= c->n_layers || n_q_heads < 0 || n_q_heads > (1 << 16) || n_tokens < 0 || n_seqs < 0 || n_tokens > (int64_t(1) << 30)) return DISC_ERR_ARG;
    if (!cu && n_tokens != n_seqs) return DISC_ERR_ARG;
    if (!rows && n_seqs > c->n_rows) return DISC_ERR_ARG;
    if (n_tokens == 0 || n_seqs == 0) return DISC_OK;
    if (const int rc = check_vectors(q, q_token_stride, q_head_stride, n_tokens, n_q_heads, &p.x[0])) return rc;
    if (const int rc = check_vectors(k, k_token_stride, k_head_stride, n_tokens, c->n_kv_heads, &p.x[1])) return rc;
    if (const int rc = check_vectors(v, v_token_stride, v_head_stride, n_tokens, c->n_kv_heads, &p.x[2])) return rc;
    if (const int rc = check_vectors(q_out, q_out_token_stride, q_out_head_stride, n_tokens, n_q_heads, &p.y[0])) return rc;
    p.n = int32_t(n_tokens); p.heads[0] = n_q_heads; p.heads[1] = p.heads[2] = c->n_kv_heads; p.pos = positions;
    CacheParams w;
    cache_params(c, layer, cu, n_seqs, rows, status, &w);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cache_type(c) == DISC_BF16 ? launch<__nv_bfloat16, true>(p, w, st) : launch<__half, true>(p, w, st);
}

int64_t disc_norm_rope_scratch_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_tokens) {
    if (n_q_heads < 0 || n_kv_heads < 0 || n_q_heads > (1 << 16) || n_kv_heads > (1 << 16) || head_dim <= 0 || head_dim > DISC_MAX_HEAD_DIM || n_tokens < 0 || n_tokens > (int64_t(1) << 30))
        return DISC_ERR_ARG;
    return grad_blocks(n_tokens, n_q_heads + n_kv_heads, head_dim) * 2 * head_dim * 4;
}

int disc_norm_rope_grad(const disc_rope_t* how, const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                        int64_t k_head_stride, disc_dtype_t dtype, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_tokens,
                        const int32_t* positions, const void* d_q_out, int64_t dq_token_stride, int64_t dq_head_stride, const void* d_k_out,
                        int64_t dk_token_stride, int64_t dk_head_stride, void* d_q, void* d_k, float* d_q_weight, float* d_k_weight, void* scratch,
                        int64_t scratch_bytes, void* stream) {
    RopeParams p = {};
    if (const int rc = check_how(how, dtype, head_dim, &p)) return rc;
    const int64_t need = disc_norm_rope_scratch_bytes(n_q_heads, n_kv_heads, head_dim, n_tokens);
    if (need < 0) return int(need);
    if (n_q_heads + n_kv_heads == 0 || (n_tokens > 0 && p.rot > 0 && !positions)) return DISC_ERR_ARG;
    const bool weights = d_q_weight || d_k_weight;
    if (weights && (!p.norm || (n_tokens > 0 && (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 3u) || scratch_bytes < need)))) return DISC_ERR_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n_tokens == 0) {
        if (d_q_weight) DISC_CUDA(cudaMemsetAsync(d_q_weight, 0, size_t(head_dim) * 4, st));
        if (d_k_weight) DISC_CUDA(cudaMemsetAsync(d_k_weight, 0, size_t(head_dim) * 4, st));
        return DISC_OK;
    }
    if (const int rc = check_vectors(q, q_token_stride, q_head_stride, n_tokens, n_q_heads, &p.x[0])) return rc;
    if (const int rc = check_vectors(k, k_token_stride, k_head_stride, n_tokens, n_kv_heads, &p.x[1])) return rc;
    if (const int rc = check_vectors(d_q_out, dq_token_stride, dq_head_stride, n_tokens, n_q_heads, &p.y[0])) return rc;
    if (const int rc = check_vectors(d_k_out, dk_token_stride, dk_head_stride, n_tokens, n_kv_heads, &p.y[1])) return rc;
    if ((n_q_heads && (!d_q || misaligned(d_q))) || (n_kv_heads && (!d_k || misaligned(d_k)))) return DISC_ERR_ARG;
    p.n = int32_t(n_tokens); p.heads[0] = n_q_heads; p.heads[1] = n_kv_heads; p.pos = positions;
    const int chunks = chunks_of(n_q_heads + n_kv_heads, head_dim), blocks = int(grad_blocks(n_tokens, n_q_heads + n_kv_heads, head_dim));
    float* part = weights ? static_cast<float*>(scratch) : nullptr;
    auto kernel = dtype == DISC_BF16 ? (head_dim <= 64 ? norm_rope_grad_kernel<__nv_bfloat16, 8> : norm_rope_grad_kernel<__nv_bfloat16, 16>)
                                     : (head_dim <= 64 ? norm_rope_grad_kernel<__half, 8> : norm_rope_grad_kernel<__half, 16>);
    if (const int rc = launch_after(kernel, unsigned(blocks), THREADS, 0, st, p, static_cast<unsigned char*>(d_q), static_cast<unsigned char*>(d_k), part, chunks)) return rc;
    if (!weights) return DISC_OK;
    return launch_after(weight_grad_kernel, unsigned((2 * head_dim + 31) / 32), 1024, 0, st, static_cast<const float*>(part), blocks, int(head_dim), d_q_weight, d_k_weight);
}

}  // extern "C"
