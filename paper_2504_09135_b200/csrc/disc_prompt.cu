// disc_attend_prompt: attention over whole prompts, packed sequences, causal or full, grouped heads.
//
//   S = scale Q K^T (masked),  P = softmax(S) row by row,  O = P V
//
// 4 D flops per query, key and query head: bound by the tensor cores once a sequence has some
// hundred tokens.  An SM's tensor cores take 8192 bf16 flops a clock and its special-function units 16
// exponentials; a block of 128 queries x 128 keys at D = 128 needs 1024 clocks of either, so that both
// have to be kept busy at once.
//
// A block works on two tiles of 128 query vectors against a stream of key/value blocks of 128 tokens.
// The vectors of a tile are TQ = 128 / G consecutive tokens times the G query heads that read the
// same key head: K and V are read once for all G, and the staircase of the causal mask costs one masked block
// per tile whatever G is.
//   warps 0-3, 4-7   one thread per query vector of tile 0 and tile 1: reads its 128 scores from tensor memory,
//                    masks, exponentiates relative to a running reference and writes P back as bf16 / f16
//                    over the scores, the first 96 keys before the rest
//   warp 8           TMA loads of Q, then K and V blocks in turn into a ring
//   warp 9           issues the MMAs (tcgen05, cta_group::1, M 128): S_i = Q_i K^T from shared memory, then
//                    O_i += P_i V with P_i as the operand in tensor memory.  While the threads of one tile
//                    exponentiate, the tensor cores run the other tile's P V and next Q K^T.
//   warp 10          what to work on next: the block takes over the places of blocks that have not started yet (cluster
//                    launch control), so that the next item's loads and first scores run under the last one's output
//                    (64 prompts of 350 tokens: 92 us with a block per item, 73 so)
// Tensor memory, 512 columns: S_0 | S_1 | O_0 | O_1.
//
// The reference a row is exponentiated against moves only when the row's maximum exceeds it by more than 2^8: until then
// the sums just grow (up to 2^8 times, fp32 has room), and the accumulated O need not be touched.  When it moves, the
// row's own thread rescales O in tensor memory; the product before has completed by then, since it was issued
// before the scores the thread has just read.  Sums l are of the unrounded probabilities, in fp32; P is
// rounded to the inputs' type because the second product takes it in that type; O is rounded once at the end.
//
// The rows of V beyond the end of a sequence belong to the next one: P is 0 there, but 0 times a non-finite
// value is not, so the last block's foreign rows are overwritten with zeros before the product.  Within a sequence the same
// would let a query's output be spoilt by tokens that it does not see: a row that comes out non-finite beside such a token
// is done once more by its thread alone (row_alone; the look at every output value costs 64 ragged prompts 88.9 us
// against 88.0, 2 x 8192 tokens 513 against 510).
// All waits are bounded; one that runs out sets the error word and every role leaves.
//
// Measured on 2 x 8192 tokens, 16 / 4 heads of 128: 457 us (1.20 PFLOP/s, 0.71 of cuBLAS' measured rate) in a short run, 515 us
// under the power cap; 2,820 clocks per 256 x 128 block of scores, of which the products take 2,080 and the exponentials as many.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "disc_sm100.cuh"

namespace {

using namespace disc;

constexpr float LN2_F = 0.6931471805599453f;
constexpr float LOG2E_F = 1.4426950408889634f;
constexpr int TM = 128;                  // query vectors of a tile
constexpr int TN = 128;                  // keys of a block
constexpr int THREADS = 384;
constexpr int BOX = 64;                  // values of a row in one 128-byte swizzled box
constexpr int FIRST = 96;                // keys whose probabilities are handed over first

template <int DP>
struct Shape {
    static constexpr int BOXES = DP / BOX;
    static constexpr int BOX_BYTES = TN * BOX * 2;                 // 16 KB
    static constexpr int TILE_BYTES = BOXES * BOX_BYTES;
    static constexpr int STAGES = DP == 128 ? 4 : 6;
    static constexpr int SMEM = 2 * TILE_BYTES + STAGES * TILE_BYTES + 1024 + 256;
};

struct PromptParams {
    const int32_t* cu_q;
    const int32_t* cu_k;
    int32_t n_seqs, hq, hkv, G, TQ, D, causal;
    float c2;                             // scale log2(e)
    const unsigned char* q;               // for row_alone; strides in bytes
    const unsigned char* k;
    const unsigned char* v;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head;
    unsigned char* out;
    float* lse;
    uint32_t* error;
    uint32_t idesc_qk, idesc_pv;
};

// One item of work, put together by the scheduling warp for the others.
struct Item {
    int q0, lq, k0, lk;                   // the sequence's tokens in q and in k / v
    int first, head;                      // first query token of the two tiles, key head
    int nb[2];                            // blocks of keys that each tile sees
    int some;                             // 0: no more items
};
constexpr int ITEMS = 2;

// Cluster launch control: a block that is already running takes over the place of one that has not started yet.
__device__ __forceinline__ void ask_for_block(void* answer, uint64_t* bar) {
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(smem_u32(answer)), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ bool taken_block(const void* answer, unsigned& block) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .b128 h;\n\t.reg .pred p;\n\t"
        "ld.shared.b128 h, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "mov.u32 %1, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, h;\n\t}"
        : "=r"(ok), "=r"(block)
        : "r"(smem_u32(answer))
        : "memory");
    return ok != 0;
}

template <typename T>
__device__ __forceinline__ void unpack8(const unsigned char* src, float* x) {
    const uint4 w = *reinterpret_cast<const uint4*>(src);
    const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y), c = unpack2<T>(w.z), d = unpack2<T>(w.w);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
}
// A query's output that is not finite.  Its blocks of keys end at `end`, and it sees the first `sees` of them.  Values that a
// token of its last blocks makes non-finite which it does not see, and none there that it sees, are formed again from what it
// sees: by one thread, 8 at a time, against the reference and the sum that are known.
template <typename T>
__device__ __noinline__ void row_alone(const PromptParams& p, int64_t q_tok, int q_head, int k_head, int64_t k0, int sees, int end, float ref, float inv,
                                       unsigned char* dst) {
    const unsigned char* q = p.q + q_tok * p.q_token + q_head * p.q_head;
    const unsigned char* k = p.k + k0 * p.k_token + k_head * p.k_head;
    const unsigned char* v = p.v + k0 * p.v_token + k_head * p.v_head;
    for (int c = 0; c < p.D; c += 8) {
        unsigned hidden = 0u, seen = 0u;               // a bit per value
        for (int j = sees / TN * TN; j < end; ++j) {
            float x[8];
            unpack8<T>(v + j * p.v_token + c * 2, x);
            unsigned bad = 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) bad |= unsigned(!(fabsf(x[e]) < CUDART_INF_F)) << e;
            if (j < sees) seen |= bad;
            else hidden |= bad;
        }
        if (!(hidden & ~seen)) continue;
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < sees; ++j) {
            float s = 0.f, x[8], y[8];
            for (int d = 0; d < p.D; d += 8) {
                unpack8<T>(q + d * 2, x);
                unpack8<T>(k + j * p.k_token + d * 2, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
            }
            const float pr = ex2_approx(fmaf(s, p.c2, -ref));
            unpack8<T>(v + j * p.v_token + c * 2, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(pr, x[e], o[e]);
        }
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack2<T>(o[2 * e] * inv, o[2 * e + 1] * inv);
        *reinterpret_cast<uint4*>(dst + c * 2) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS, 1)
attend_prompt_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PromptParams p) {
    using S = Shape<DP>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* tiles = reinterpret_cast<unsigned char*>((uintptr_t(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char* ring = tiles + 2 * S::TILE_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + S::STAGES * S::TILE_BYTES);
    uint64_t* q_full = bars;                          // [2]
    uint64_t* q_empty = bars + 2;                     // [2] the last scores of an item's tile are done
    uint64_t* s_full = bars + 4;                      // [2] scores of a tile (and the product before) done
    uint64_t* o_full = bars + 6;                      // [2] the last product of an item's tile done
    uint64_t* p_full = bars + 8;                      // [2][2] probabilities of a tile written: the first 96 keys, the last 32
    uint64_t* item_full = bars + 12;                  // [ITEMS]
    uint64_t* item_empty = bars + 14;                 // [ITEMS]
    uint64_t* answer_full = bars + 16;
    uint64_t* kv_full = bars + 17;                    // [STAGES]
    uint64_t* kv_empty = bars + 17 + S::STAGES;       // [STAGES]
    static_assert((17 + 2 * S::STAGES) * 8 <= 256, "room for the barriers");
    __shared__ __align__(16) unsigned char answer[16];
    __shared__ Item items[ITEMS];
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    volatile int* abort = &s_abort;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full + i, 1); mbar_init(q_empty + i, 1); mbar_init(s_full + i, 1); mbar_init(o_full + i, 1);
            mbar_init(p_full + 2 * i, TM / 32); mbar_init(p_full + 2 * i + 1, TM / 32);
        }
        for (int i = 0; i < ITEMS; ++i) { mbar_init(item_full + i, 1); mbar_init(item_empty + i, 10); }
        mbar_init(answer_full, 1);
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(kv_full + s, 1); mbar_init(kv_empty + s, 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_slot);

    // the n-th item of this block, null when there is none (or a wait ran out); it stays in its place until the warp lets go of it
    auto get_item = [&](int n) -> const volatile Item* {
        if (!mbar_wait_all(item_full + n % ITEMS, (n / ITEMS) & 1, abort)) return nullptr;
        const volatile Item* it = &items[n % ITEMS];
        return it->some ? it : nullptr;
    };
    auto let_go = [&](int n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(item_empty + n % ITEMS);
    };

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (warp == 10) {
            // ---- scheduling.  Block b stands for key head b % hkv of the (b / hkv)-th pair of tiles, counted through the
            // sequences, the tiles late in a sequence, which see the most keys, first; neighbouring blocks share keys
            // and values.  The launch has room for the most pairs there can be; what lies beyond the last is skipped.
            unsigned block = blockIdx.x;
            int base = 0, chunk = 0;                   // pairs before the chunk-th 32 sequences
            for (int n = 0;; ++n) {
                Item it;
                it.some = 0;
                bool more = true;
                while (more) {
                    const int pair = int(block / unsigned(p.hkv));
                    bool beyond = false;
                    if (pair < base) base = chunk = 0;
                    for (;;) {
                        const int seq = chunk * 32 + lane;
                        const int q0 = p.cu_q[min(seq, p.n_seqs)], q1 = p.cu_q[min(seq + 1, p.n_seqs)];
                        const int pairs = (q1 - q0 + 2 * p.TQ - 1) / (2 * p.TQ);
                        int upto = pairs;
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
                            const int u = __shfl_up_sync(0xffffffffu, upto, o);
                            if (lane >= o) upto += u;
                        }
                        const unsigned in = __ballot_sync(0xffffffffu, pair < base + upto);
                        if (in) {
                            const int who = __ffs(in) - 1;
                            it.q0 = __shfl_sync(0xffffffffu, q0, who);
                            it.lq = __shfl_sync(0xffffffffu, q1, who) - it.q0;
                            const int before = base + __shfl_sync(0xffffffffu, upto - pairs, who);
                            it.first = (__shfl_sync(0xffffffffu, pairs, who) - 1 - (pair - before)) * 2 * p.TQ;
                            const int seq_of = chunk * 32 + who;
                            it.k0 = p.cu_k[seq_of];
                            it.lk = p.cu_k[seq_of + 1] - it.k0;
                            break;
                        }
                        base += __shfl_sync(0xffffffffu, upto, 31);
                        ++chunk;
                        if (chunk * 32 >= p.n_seqs) { beyond = true; break; }
                    }
                    if (!beyond) {
                        it.head = int(block % unsigned(p.hkv));
                        it.some = 1;
                        const int shift = it.lk - it.lq;          // query j sees the keys 0 .. j + shift
                        for (int i = 0; i < 2; ++i) {
                            const int t0 = it.first + i * p.TQ, t1 = min(it.lq, t0 + p.TQ);
                            const int keys = t0 < t1 ? (p.causal ? min(it.lk, t1 + shift) : it.lk) : 0;
                            it.nb[i] = keys > 0 ? (keys + TN - 1) / TN : 0;
                        }
                    }
                    // the place in the ring was read by everybody before it is written again
                    if (it.some) {
                        if (n >= ITEMS && !mbar_wait_all(item_empty + n % ITEMS, (n / ITEMS - 1) & 1, abort)) { it.some = 0; more = false; break; }
                        if (lane == 0) {
                            items[n % ITEMS] = it;
                            mbar_arrive(item_full + n % ITEMS);
                        }
                        __syncwarp();
                        break;
                    }
                    more = false;                      // nothing lies beyond the last pair
                }
                if (!it.some) {
                    if (n >= ITEMS) mbar_wait_all(item_empty + n % ITEMS, (n / ITEMS - 1) & 1, abort);
                    if (lane == 0) {
                        items[n % ITEMS].some = 0;
                        mbar_arrive(item_full + n % ITEMS);
                    }
                    break;
                }
                if (lane == 0) {
                    mbar_expect_tx(answer_full, 16);
                    ask_for_block(answer, answer_full);
                }
                __syncwarp();
                if (!mbar_wait_all(answer_full, n & 1, abort)) break;
                const bool got = taken_block(answer, block);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (!got) {
                    ++n;
                    if (n >= ITEMS) mbar_wait_all(item_empty + n % ITEMS, (n / ITEMS - 1) & 1, abort);
                    if (lane == 0) {
                        items[n % ITEMS].some = 0;
                        mbar_arrive(item_full + n % ITEMS);
                    }
                    break;
                }
            }
        } else if (warp == 8) {
            // ---- loads
            int load = 0, uses[2] = {0, 0};
            bool ok = true;
            for (int n = 0; ok; ++n) {
                const volatile Item* it = get_item(n);
                if (!it) break;
                if (lane == 0) {
                    const int n_blk = max(it->nb[0], it->nb[1]), head = it->head, k0 = it->k0;
                    const uint32_t q_bytes = uint32_t(S::BOXES) * p.G * p.TQ * BOX * 2;
                    for (int i = 0; i < 2 && ok; ++i)
                        if (it->nb[i] > 0) {
                            if (uses[i] > 0) ok = mbar_wait(q_empty + i, (uses[i] - 1) & 1, abort);
                            if (!ok) break;
                            ++uses[i];
                            mbar_expect_tx(q_full + i, q_bytes);
                            for (int b = 0; b < S::BOXES; ++b)
                                tma_load_3d(tiles + i * S::TILE_BYTES + b * S::BOX_BYTES, &map_q, b * BOX, head * p.G, it->q0 + it->first + i * p.TQ, q_full + i);
                        }
                    for (int j = 0; j < 2 * n_blk && ok; ++j, ++load) {            // K_0 V_0 K_1 V_1 ...
                        const int s = load % S::STAGES, round = load / S::STAGES;
                        if (round > 0) ok = mbar_wait(kv_empty + s, (round - 1) & 1, abort);
                        if (!ok) break;
                        mbar_expect_tx(kv_full + s, S::TILE_BYTES);
                        for (int b = 0; b < S::BOXES; ++b)
                            tma_load_3d(ring + s * S::TILE_BYTES + b * S::BOX_BYTES, j & 1 ? &map_v : &map_k, b * BOX, head, k0 + (j >> 1) * TN, kv_full + s);
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                let_go(n);
            }
        } else if (warp == 9) {
            // ---- MMAs
            const uint64_t q_desc[2] = {smem_desc_sw128(tiles), smem_desc_sw128(tiles + S::TILE_BYTES)};
            const uint64_t kv_desc = smem_desc_sw128(ring), v_desc = smem_desc_n_major(ring, S::BOX_BYTES);
            constexpr uint64_t TILE16 = S::TILE_BYTES >> 4;
            // S_i = Q_i K^T with the keys in place `stage` of the ring
            auto scores = [&](int i, int stage) {
                const uint64_t kd = kv_desc + uint64_t(stage) * TILE16;
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) {
                    const uint64_t off = uint64_t((kk / 4) * (S::BOX_BYTES >> 4) + (kk % 4) * 2);
                    umma_ss(tmem + i * TN, q_desc[i] + off, kd + off, p.idesc_qk, kk > 0);
                }
            };
            int load = 0, uses[2] = {0, 0}, done[2] = {0, 0};      // loads taken; items and blocks of each tile
            bool ok = true;
            for (int n = 0; ok; ++n) {
                const volatile Item* it = get_item(n);
                if (!it) break;
                const int nb[2] = {it->nb[0], it->nb[1]}, lk = it->lk;
                let_go(n);
                const int n_blk = max(nb[0], nb[1]);
                if (n_blk == 0) continue;
                ok = mbar_wait_all(kv_full + load % S::STAGES, (load / S::STAGES) & 1, abort);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (nb[i] == 0 || !ok) continue;
                    ok = mbar_wait_all(q_full + i, uses[i] & 1, abort);
                    if (!ok) continue;
                    ++uses[i];
                    tc_fence_after();
                    if (elect_one()) {
                        scores(i, load % S::STAGES);
                        umma_commit(s_full + i);
                        if (nb[i] == 1) umma_commit(q_empty + i);
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (elect_one()) umma_commit(kv_empty + load % S::STAGES);
                __syncwarp();
                ++load;
                for (int j = 0; j < n_blk && ok; ++j) {
                    const bool more = j + 1 < n_blk;
                    const int v_stage = load % S::STAGES, k_stage = (load + 1) % S::STAGES;
                    ok = mbar_wait_all(kv_full + v_stage, (load / S::STAGES) & 1, abort);
                    if (ok && more) ok = mbar_wait_all(kv_full + k_stage, ((load + 1) / S::STAGES) & 1, abort);
                    if (!ok) break;
                    const int left = lk - j * TN;
                    if (left < TN) {                   // rows beyond the sequence: zeros
                        unsigned char* v_tile = ring + v_stage * S::TILE_BYTES;
                        for (int r = left + (lane >> 3); r < TN; r += 4)
#pragma unroll
                            for (int b = 0; b < S::BOXES; ++b)
                                *reinterpret_cast<uint4*>(v_tile + b * S::BOX_BYTES + r * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    const uint64_t vd = v_desc + uint64_t(v_stage) * TILE16;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (j >= nb[i] || !ok) continue;
                        auto values = [&](int from, int to) {
#pragma unroll
                            for (int kk = from; kk < to; ++kk)
                                umma_ts(tmem + 2 * TN + i * DP, tmem + i * TN + kk * 8, vd + uint64_t(kk * (16 * 128 >> 4)), p.idesc_pv, j > 0 || kk > 0);
                        };
                        ok = mbar_wait_all(p_full + 2 * i, done[i] & 1, abort);
                        if (!ok) continue;
                        tc_fence_after();
                        if (elect_one()) values(0, FIRST / 16);
                        __syncwarp();
                        ok = mbar_wait_all(p_full + 2 * i + 1, done[i] & 1, abort);
                        if (!ok) continue;
                        ++done[i];
                        tc_fence_after();
                        if (elect_one()) {
                            values(FIRST / 16, TN / 16);
                            if (j + 1 < nb[i]) {
                                scores(i, k_stage);
                                umma_commit(s_full + i);
                                if (j + 2 == nb[i]) umma_commit(q_empty + i);
                            } else umma_commit(o_full + i);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect_one()) {
                        umma_commit(kv_empty + v_stage);
                        if (more) umma_commit(kv_empty + k_stage);
                    }
                    __syncwarp();
                    load += more ? 2 : 1;
                }
            }
            // the last reports of free places have arrived before the block leaves
            for (int back = 0; back < S::STAGES && back < load && ok; ++back)
                ok = mbar_wait_all(kv_empty + (load - 1 - back) % S::STAGES, ((load - 1 - back) / S::STAGES) & 1, abort);
            for (int i = 0; i < 2 && ok; ++i)
                if (uses[i] > 0) ok = mbar_wait_all(q_empty + i, (uses[i] - 1) & 1, abort);
        }
    } else {
        // ---- softmax: this thread's query vector
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int i = warp >> 2;
        const int m = (warp & 3) * 32 + lane;
        const int row_tok = i * p.TQ + m / p.G, g = m % p.G;
        const bool used = m < p.TQ * p.G;
        const uint32_t lane_bits = uint32_t((warp & 3) * 32) << 16;
        const uint32_t s_tm = tmem + lane_bits + i * TN, o_tm = tmem + lane_bits + 2 * TN + i * DP;
        const float2 c2 = make_float2(p.c2, p.c2);
        // output rows on 32-byte boundaries are written 32 bytes at a time
        const bool wide = p.D % 16 == 0 && (reinterpret_cast<uintptr_t>(p.out) & 31) == 0;
        int seen = 0, ends = 0;                       // blocks and items of this tile so far
        for (int n = 0;; ++n) {
            const volatile Item* it = get_item(n);
            if (!it) break;
            const int nb = it->nb[i];
            int sees = 0;                             // keys that the row sees
            if (used && it->first + row_tok < it->lq) sees = p.causal ? max(0, min(it->lk, it->first + row_tok + it->lk - it->lq + 1)) : it->lk;
            float ref = -CUDART_INF_F;                // in units of log2
            float2 l = make_float2(0.f, 0.f);
            bool bad = false;                         // a score is NaN
            bool ok = true;
            for (int j = 0; j < nb; ++j) {
                ok = mbar_wait_all(s_full + i, seen & 1, abort);
                if (!ok) break;
                ++seen;
                tc_fence_after();
                float s[TN];
                tmem_ld128(s_tm, s);
                const int left = sees - j * TN;       // keys of this block that the row sees
                if (__any_sync(0xffffffffu, left < TN)) {
#pragma unroll
                    for (int c = 0; c < TN; ++c) s[c] = c < left ? s[c] : -CUDART_INF_F;
                }
                uint32_t pk[16];
                float2 la;
                first_scores<T, DP, TN>(s, c2, ref, l, bad, o_tm, j > 0, la, pk);
                tmem_st16(s_tm, pk);
                const float base = ref > -CUDART_INF_F ? ref : 0.f;
                const float2 down = make_float2(-base, -base);
                exp_chunk<T>(s + 32, c2, down, la, pk);
                tmem_st16(s_tm + 16, pk);
                exp_chunk<T>(s + 64, c2, down, la, pk);
                tmem_st16(s_tm + 32, pk);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 2 * i);
                exp_chunk<T>(s + 96, c2, down, la, pk);
                tmem_st16(s_tm + 48, pk);
                l = add2(l, la);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 2 * i + 1);
            }
            const float total = bad ? CUDART_NAN_F : l.x + l.y;
            if (!ok) break;
            if (nb > 0) {
                if (!mbar_wait_all(o_full + i, ends & 1, abort)) break;
                ++ends;
                tc_fence_after();
            }
            const float inv = total > 0.f ? 1.f / total : (total == 0.f ? 0.f : total);
            const int tok = it->first + row_tok;
            const bool live = used && tok < it->lq;
            const int64_t at = int64_t(it->q0 + tok) * p.hq + it->head * p.G + g;
            unsigned char* dst = p.out + at * p.D * 2;
            float2 finite[4] = {};                    // NaN once a value is not
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
                uint32_t o[32];
                if (nb > 0) tmem_ld32(o_tm + c, o);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    finite[e % 4] = fma2(make_float2(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1])), make_float2(0.f, 0.f), finite[e % 4]);
#pragma unroll
                for (int e = 0; e < 32; e += 16) {
                    uint32_t w[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        w[x] = sees > 0 ? pack2<T>(__uint_as_float(o[e + 2 * x]) * inv, __uint_as_float(o[e + 2 * x + 1]) * inv) : 0u;
                    if (live && c + e < p.D) {
                        if (wide) st_global32(dst + (c + e) * 2, w);
                        else {
                            *reinterpret_cast<uint4*>(dst + (c + e) * 2) = make_uint4(w[0], w[1], w[2], w[3]);
                            if (c + e + 8 < p.D) *reinterpret_cast<uint4*>(dst + (c + e) * 2 + 16) = make_uint4(w[4], w[5], w[6], w[7]);
                        }
                    }
                }
            }
            finite[0] = add2(add2(finite[0], finite[1]), add2(finite[2], finite[3]));
            if (finite[0].x + finite[0].y != 0.f && live && sees > 0 && sees < min(it->lk, nb * TN) && total < CUDART_INF_F)
                row_alone<T>(p, it->q0 + tok, it->head * p.G + g, it->head, it->k0, sees, min(it->lk, nb * TN), ref > -CUDART_INF_F ? ref : 0.f, inv, dst);
            let_go(n);
            if (live && p.lse) p.lse[at] = total > 0.f ? (ref + log2f(total)) * LN2_F : (total == 0.f ? -CUDART_INF_F : total);
            tc_fence_before();                        // O has been read before the next item's first probabilities are reported
        }
    }

    tc_fence_before();
    __syncthreads();
    if (s_abort && threadIdx.x == 0) {
        atomicExch(p.error, 1u);
        for (int i = 0; i < 200; ++i) __nanosleep(1000);          // copies in flight land before the memory is given up
    }
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// [tokens][heads][D] as a 3-D tensor map, innermost first
int make_map3(EncodeTiled enc, CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t tokens, int32_t heads, int32_t D,
              int64_t token_stride, int64_t head_stride, int box_heads, int box_tokens) {
    const cuuint64_t dims[3] = {cuuint64_t(D), cuuint64_t(heads), cuuint64_t(tokens)};
    const cuuint64_t strides[2] = {cuuint64_t(head_stride) * 2, cuuint64_t(token_stride) * 2};
    const cuuint32_t box[3] = {cuuint32_t(BOX), cuuint32_t(box_heads), cuuint32_t(box_tokens)};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = enc(map, type, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DISC_OK : DISC_ERR_UNSUPPORTED;
}

template <typename T, int DP>
int launch_prompt(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const PromptParams& p, unsigned grid, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    if (const int rc = allow_smem(attend_prompt_kernel<T, DP>, Shape<DP>::SMEM, done)) return rc;
    attend_prompt_kernel<T, DP><<<grid, THREADS, Shape<DP>::SMEM, st>>>(q, k, v, p);
    DISC_CUDA(cudaGetLastError());
    return DISC_OK;
}

}  // namespace

extern "C" {

int disc_attend_prompt(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                       int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride, disc_dtype_t dtype,
                       int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_q, int64_t n_k, const int32_t* cu_q,
                       const int32_t* cu_k, int32_t n_seqs, int32_t max_q, int32_t causal, float scale, void* out, float* lse_out,
                       uint32_t* error, void* stream) {
    if (n_q_heads <= 0 || n_kv_heads <= 0 || head_dim <= 0 || n_q < 0 || n_k < 0 || n_seqs < 0 || max_q < 0) return DISC_ERR_ARG;
    if (dtype != DISC_BF16 && dtype != DISC_F16) return DISC_ERR_UNSUPPORTED;
    if (n_q_heads % n_kv_heads || !(scale > 0.f) || !(scale <= 3.0e38f)) return DISC_ERR_ARG;
    if (head_dim % 8 || head_dim > DISC_MAX_HEAD_DIM || n_q_heads / n_kv_heads > TM || n_q >= (int64_t(1) << 31) - 512 ||
        n_k >= (int64_t(1) << 31) - 512)
        return DISC_ERR_UNSUPPORTED;
    if (n_q == 0 || n_seqs == 0 || max_q == 0) return DISC_OK;
    if (!q || !out || !cu_q || !error || (n_k > 0 && (!k || !v))) return DISC_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(out)) & 15u)
        return DISC_ERR_ARG;
    // without the keys' own offsets they are the queries'
    if (!cu_k && n_k != n_q) return DISC_ERR_ARG;
    // TMA: strides in multiples of 16 bytes.  The stride over an axis of one is never used; any valid one will do.
    const int64_t fit = (int64_t(head_dim) + 7) / 8 * 8;
    if (n_q_heads == 1) q_head_stride = fit;
    if (n_kv_heads == 1) k_head_stride = v_head_stride = fit;
    if (n_q == 1) q_token_stride = fit * n_q_heads;
    if (n_k <= 1) k_token_stride = v_token_stride = fit * n_kv_heads;
    if ((q_token_stride | q_head_stride | k_token_stride | k_head_stride | v_token_stride | v_head_stride) & 7) return DISC_ERR_UNSUPPORTED;
    if (q_token_stride <= 0 || q_head_stride <= 0 || k_token_stride <= 0 || k_head_stride <= 0 || v_token_stride <= 0 || v_head_stride <= 0)
        return DISC_ERR_UNSUPPORTED;
    const int G = n_q_heads / n_kv_heads, TQ = TM / G;
    PromptParams p;
    p.cu_q = cu_q; p.cu_k = cu_k ? cu_k : cu_q; p.n_seqs = n_seqs; p.hq = n_q_heads; p.hkv = n_kv_heads; p.G = G; p.TQ = TQ; p.D = head_dim;
    p.q = static_cast<const unsigned char*>(q); p.k = static_cast<const unsigned char*>(k); p.v = static_cast<const unsigned char*>(v);
    p.q_token = q_token_stride * 2; p.q_head = q_head_stride * 2; p.k_token = k_token_stride * 2; p.k_head = k_head_stride * 2;
    p.v_token = v_token_stride * 2; p.v_head = v_head_stride * 2;
    p.causal = causal != 0; p.c2 = scale * LOG2E_F; p.out = static_cast<unsigned char*>(out); p.lse = lse_out; p.error = error;
    // pairs of tiles: a sequence of n queries has n / (2 TQ) of them, rounded up
    const int64_t longest = max_q < n_q ? max_q : n_q;
    const int64_t by_seq = (longest + 2 * TQ - 1) / (2 * TQ) * n_seqs, by_sum = n_q / (2 * TQ) + n_seqs;
    const int64_t grid = (by_seq < by_sum ? by_seq : by_sum) * n_kv_heads;
    if (grid > 0x7fffffff) return DISC_ERR_UNSUPPORTED;
    const int DP = head_dim <= 64 ? 64 : 128;
    // instruction descriptors: D fp32 (bits 4-5 = 1), A and B f16 = 0 / bf16 = 1 (bits 7-9, 10-12), B of the second
    // product N-major (bit 16), N >> 3 at bit 17, M >> 4 at bit 24
    const uint32_t ty = dtype == DISC_BF16 ? 1u : 0u;
    const uint32_t idesc = (1u << 4) | (ty << 7) | (ty << 10) | (uint32_t(TM >> 4) << 24);
    p.idesc_qk = idesc | (uint32_t(TN >> 3) << 17);
    p.idesc_pv = idesc | (uint32_t(DP >> 3) << 17) | (1u << 16);

    EncodeTiled enc = nullptr;
    if (const int rc = tensor_map_encoder(&enc)) return rc;
    const CUtensorMapDataType type = dtype == DISC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    alignas(64) CUtensorMap map_q, map_k, map_v;
    if (const int rc = make_map3(enc, &map_q, type, q, n_q, n_q_heads, head_dim, q_token_stride, q_head_stride, G, TQ)) return rc;
    // no keys at all: no load is issued, and any valid map will do
    const bool none = n_k == 0;
    if (const int rc = make_map3(enc, &map_k, type, none ? q : k, none ? 1 : n_k, n_kv_heads, head_dim, k_token_stride, k_head_stride, 1, TN)) return rc;
    if (const int rc = make_map3(enc, &map_v, type, none ? q : v, none ? 1 : n_k, n_kv_heads, head_dim, v_token_stride, v_head_stride, 1, TN)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == DISC_BF16)
        return DP == 64 ? launch_prompt<__nv_bfloat16, 64>(map_q, map_k, map_v, p, unsigned(grid), st)
                        : launch_prompt<__nv_bfloat16, 128>(map_q, map_k, map_v, p, unsigned(grid), st);
    return DP == 64 ? launch_prompt<__half, 64>(map_q, map_k, map_v, p, unsigned(grid), st)
                    : launch_prompt<__half, 128>(map_q, map_k, map_v, p, unsigned(grid), st);
}

int disc_attend_error(const uint32_t* error, void* stream) {
    if (!error) return DISC_ERR_ARG;
    uint32_t e = 0;
    DISC_CUDA(cudaMemcpyAsync(&e, error, 4, cudaMemcpyDeviceToHost, static_cast<cudaStream_t>(stream)));
    DISC_CUDA(cudaStreamSynchronize(static_cast<cudaStream_t>(stream)));
    return e ? DISC_ERR_CUDA : DISC_OK;
}

}  // extern "C"
