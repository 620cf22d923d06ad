// disc_attend_cached over a cache held in 8 bits, where up to 16 query vectors read the same pages.  The plan is that of
// disc_attend.cu.
//
//   out[r] = sum_j p_j v_j,  p = softmax_j(scale q[r] k_j),  k_j = 2^e_j kc_j,  v_j = 2^f_j vc_j
//
// The codes kc, vc become f16 exactly and go into the products as they are; the
// powers of two stay outside: scale 2^e_j multiplies a token's scores, and what multiplies a token's value codes is
// 2^(s_j + f_j - t) with a running maximum t of the exponents s_j + f_j of its own, so that the factors are at most 2^SLACK (and HEADROOM more, up to
// the end of f16's range) however much the values' sizes differ from token to token.  The queries become f16 too, a bf16 vector after a power of two that brings its
// largest value to 2^8 (what is lost is below 2^-32 of the largest value).
//
// Bound by the bytes of the distinct pages while the conversion keeps up.  So the products are taken with the tokens (S^T = K Q^T) and
// the value dims (O^T = V^T P^T) as the wide side of mma.sync m16n8k16 and the query vectors as the narrow one, eight at a
// time: a converted register is used whole, and once for each eight query vectors.  ldmatrix with transposition moves 16-bit units, which
// are two value dims of a token here; the two become two rows of the product (dims 2 i and 2 i + 1 are rows i and i + 8).
//
// A block of 4 warps per share and key head as in disc_attend.cu: every warp brings in blocks of 16 tokens for itself, several in
// flight, and the warps' results are joined at the end.  The maxima move only when a score exceeds them by SLACK, which is what one
// vote of the warp costs, instead of shuffles for every block.
//
// Measured on 64 rows of 1 to 8191 tokens, 32 / 8 heads of 128, bf16 in e4m3: 98 us for 0.53 GB (5.4 TB/s; the copy rate would be 81).  Neither
// DRAM (82 %) nor issue (52 %) nor a pipe (ALU 57 %, 212 of 380 instructions for a block of 16 tokens) is full; 8 or 12 warps to an SM,
// one block at a time or two, three or five blocks in flight make no difference.

#include "disc_attend.cuh"
#include "disc_held_mma.cuh"

namespace {

using namespace disc;

constexpr int AT = 128;
constexpr int WARPS = AT / 32;

template <int DP, int NT>
struct HeldSmem {
    static constexpr int STAGES = DP == 128 ? 4 : 8;               // blocks on their way to a warp, and the one it is at
    static constexpr int STAGE = held_stage_bytes<DP>();           // in its spare place: the block's tokens and owner
    static constexpr int RING = STAGES * STAGE;                    // of a warp
    static constexpr int SUMS = WARPS * NT * 8 * DP * 4;           // at the end, over the rings
    static constexpr int BYTES = WARPS * RING > SUMS ? WARPS * RING : SUMS;
};

// Up to 8 query vectors fit three blocks' registers; with 16 they spilled there and took more than twice as long.  The 64 rows with 16 heads
// on each of 4 key heads: 77 us for 0.27 GB, which the copy rate would move in 41; eight warps to an SM are too few for the chain of a block.
template <typename T, int DP, int HELD, int NT>
__global__ void __launch_bounds__(AT, NT == 1 ? HELD_BLOCKS : 2) attend_held_kernel(const AttendParams p) {
    let_later_in();
    wait_for_earlier();
    using S = HeldSmem<DP, NT>;
    constexpr int STAGES = S::STAGES, STAGE = S::STAGE;
    constexpr int CH = DP / 16;                                    // 16-byte chunks of a token's codes
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float w_m[WARPS][NT * 8], w_l[WARPS][NT * 8], w_t[WARPS][NT * 8];
    __shared__ int s_last;

    // by shuffle: the compiler then knows that the warp's number is the same for its lanes, and what hangs on it goes through uniform registers
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const PlanShape& sh = p.shape;
    const int G = sh.G, blk_shift = 31 - __clz(sh.blks_per_page);  // pages are powers of two
    const int lane_of = blockIdx.x / p.kv_heads, head = blockIdx.x % p.kv_heads;
    const int item_end = p.plan.first[lane_of + 1];
    unsigned char* const ring = smem + warp * S::RING;
    const uint32_t ring_at = smem_u32(ring);

    for (int n = p.plan.first[lane_of]; n < item_end; ++n) {
        const int4 item = *reinterpret_cast<const int4*>(p.plan.items + n), more = *(reinterpret_cast<const int4*>(p.plan.items + n) + 1);
        const int g = item.x, r0 = more.x, n_rows = more.y, splits = more.z;
        const int M = n_rows * G;
        const int2* list = p.plan.list + int64_t(g) * sh.list_ld;
        const int32_t* table = p.table + int64_t(r0) * p.width;
        const int32_t len = p.len[r0];
        const int blocks = (item.z - item.y - warp + WARPS - 1) / WARPS;       // of this warp: warp, warp + 4, ...

        __syncthreads();                                           // the item before is done with the shared memory
        auto entry = [&](int t) {
            const int i = item.y + t * WARPS + warp;
            if (i >= item.z) return make_int2(0, 0);
            if (sh.per_group > 1) return list[i];
            return make_int2(table[i >> blk_shift], (i & (sh.blks_per_page - 1)) | max(0, min(BLK, len - i * BLK)) << 8);
        };
        auto load = [&](uint32_t stage, int2 e) {
            // a plan older than the books: rows may have let go of their pages since, and -1 is no place to read from
            if (unsigned(e.x) >= unsigned(p.pages)) e = make_int2(0, 0);
            const int tokens = (e.y >> 8) & 255;
            const int64_t off = (int64_t(e.x) * p.kv_heads + head) * p.head_bytes;
            if (tokens) load_held_block<DP>(ring_at + stage, p.k + off, p.v + off, e.y & 255, tokens, p.D, p.page_size, lane);
            if (lane == 0) *reinterpret_cast<volatile int*>(ring + stage + 2 * BLK * DP + HELD_SPARE) = e.y >> 8;
        };
        int2 first[STAGES];
#pragma unroll
        for (int t = 0; t < STAGES; ++t) first[t] = entry(t);
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t) {
            if (t < blocks) load(t * STAGE, first[t]);
            cp_commit();
        }
        int2 next = first[STAGES - 1];

        // query vectors: vector m is head m % G of row m / G
        HeldQueries<DP, NT> qs;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int m = nt * 8 + (lane >> 2);
            load_held_queries<T, DP, HELD>(qs, nt, p.q + (r0 + m / G) * p.q_row + (head * G + m % G) * p.q_head, m < M, p.D, p.c2, lane);
        }
        HeldSums<DP, NT> acc;
        clear_held(acc);
        int owner_of[NT][2];                                       // whose vectors this thread's columns are
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) owner_of[nt][e] = (nt * 8 + (lane & 3) * 2 + e) / G + 1;

        uint32_t stage = 0;
#pragma unroll 1
        for (int t = 0; t < blocks; ++t) {
            cp_wait<STAGES - 2>();
            __syncwarp();                                          // a warp works on what it has brought in itself
            if (t + STAGES - 1 < blocks) load(stage == 0 ? (STAGES - 1) * STAGE : stage - STAGE, next);
            cp_commit();
            next = entry(t + STAGES);
            const int meta = *reinterpret_cast<volatile int*>(ring + stage + 2 * BLK * DP + HELD_SPARE), owner = meta >> 8, tokens = meta & 255;
            bool in[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) in[nt][e] = !owner || owner == owner_of[nt][e];
            if (tokens) add_held_block<T, DP, HELD, NT>(acc, qs, ring_at + stage, tokens, in, lane);
            stage = stage == (STAGES - 1) * STAGE ? 0 : stage + STAGE;
        }
        finish_held(acc);
        cp_wait<0>();
        __syncthreads();                                           // every warp is done with the tiles
        // sums to shared memory, [warps x vectors][DP] fp32
        float* os = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int m = nt * 8 + (lane & 3) * 2 + e;
                float* a = os + (warp * NT * 8 + m) * DP + (lane >> 2) * 2;
#pragma unroll
                for (int j = 0; j < CH; ++j) *reinterpret_cast<float2*>(a + 16 * j) = make_float2(acc.o[nt][j][e], acc.o[nt][j][2 + e]);
                if (lane < 4) { w_m[warp][m] = acc.m[nt][e]; w_l[warp][m] = acc.l[nt][e]; w_t[warp][m] = acc.t[nt][e]; }
            }
        __syncthreads();

        const int64_t slot = splits > 1 ? (int64_t(more.w + item.w) * p.kv_heads + head) * sh.M : 0;
        constexpr int DV = DP / 4;
        for (int i = tid; i < M * DV; i += AT) {
            const int m = i / DV, d = (i % DV) * 4;
            if (d >= p.D) continue;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            float mm = w_m[0][m], tt = w_t[0][m];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) { mm = fmaxf(mm, w_m[w][m]); tt = fmaxf(tt, w_t[w][m]); }
            float ll = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float f = w_t[w][m] > -CUDART_INF_F ? ex2_approx(w_t[w][m] - tt) : 0.f;
                const float4 y = *reinterpret_cast<const float4*>(os + (w * NT * 8 + m) * DP + d);
                // a sum without a finite maximum is 0, or NaN from a score or a vector that is
                x.x += w_t[w][m] > -CUDART_INF_F ? f * y.x : y.x; x.y += w_t[w][m] > -CUDART_INF_F ? f * y.y : y.y;
                x.z += w_t[w][m] > -CUDART_INF_F ? f * y.z : y.z; x.w += w_t[w][m] > -CUDART_INF_F ? f * y.w : y.w;
                ll += w_m[w][m] > -CUDART_INF_F ? ex2_approx(w_m[w][m] - mm) * w_l[w][m] : w_l[w][m];
            }
            const float inv = ll > 0.f ? 1.f / ll : (ll == 0.f ? 0.f : ll);
            // in two halves: with the smallest of the values' powers of two the factor itself has few digits
            const float f = tt > -CUDART_INF_F && ll > 0.f ? exp2f(0.5f * (tt - mm)) : 1.f;
            x.x = x.x * inv * f * f; x.y = x.y * inv * f * f; x.z = x.z * inv * f * f; x.w = x.w * inv * f * f;
            float lse2 = ll > 0.f ? mm + log2f(ll) : (ll == 0.f ? -CUDART_INF_F : ll);
            if (n_rows > 1 && p.len[r0 + m / G] == 0) {           // beside rows whose shared pages it does not hold
                x = make_float4(0.f, 0.f, 0.f, 0.f);
                lse2 = -CUDART_INF_F;
            }
            if (splits > 1) {
                *reinterpret_cast<float4*>(p.plan.part + (slot + m) * p.D + d) = x;
                if (d == 0) p.plan.part_lse[slot + m] = lse2;
            } else {
                const int64_t at = int64_t(r0 + m / G) * p.kv_heads * G + head * G + m % G;
                *reinterpret_cast<uint2*>(p.out + (at * p.D + d) * 2) = make_uint2(pack_out<T>(x.x, x.y), pack_out<T>(x.z, x.w));
                if (d == 0 && p.lse) p.lse[at] = lse2 * LN2_F;
            }
        }
        if (splits > 1) {
            // the last of the group's items joins them all, in their order
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                int32_t* cnt = p.plan.arrived + int64_t(g) * p.kv_heads + head;
                s_last = atomicAdd(cnt, 1) == splits - 1;
                if (s_last) *cnt = 0;
            }
            __syncthreads();
            if (s_last) {
                __threadfence();
                join_items<T, DP, AT>(p, more.w, splits, head, M, r0);
            }
        }
    }
}

template <typename T, int DP, int HELD, int NT>
int launch(const AttendParams& p, cudaStream_t st) {
    constexpr int bytes = HeldSmem<DP, NT>::BYTES;
    static std::atomic<uint64_t> done{0};
    if (const int rc = allow_smem(attend_held_kernel<T, DP, HELD, NT>, bytes, done)) return rc;
    return launch_after(attend_held_kernel<T, DP, HELD, NT>, unsigned(p.shape.lanes * p.kv_heads), AT, bytes, st, p);
}
template <typename T, int HELD>
int launch(const AttendParams& p, cudaStream_t st) {
    if (p.shape.M <= HELD_FEW) return p.D <= 64 ? launch<T, 64, HELD, 1>(p, st) : launch<T, 128, HELD, 1>(p, st);
    return p.D <= 64 ? launch<T, 64, HELD, 2>(p, st) : launch<T, 128, HELD, 2>(p, st);
}

}  // namespace

int disc::attend_held(const AttendParams& p, int32_t dtype, cudaStream_t st) {
    if ((dtype & 15) == DISC_BF16) return (dtype >> 4) == HELD_E4M3 ? launch<__nv_bfloat16, HELD_E4M3>(p, st) : launch<__nv_bfloat16, HELD_I8>(p, st);
    return (dtype >> 4) == HELD_E4M3 ? launch<__half, HELD_E4M3>(p, st) : launch<__half, HELD_I8>(p, st);
}
