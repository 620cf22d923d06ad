// disc_attend_cached where more than 16 query vectors read the same pages: K candidates of a query over its
// prompt, or many query heads on one key head.
//
// Per token and key head there are 4 D bytes to read and 4 M D flops to do, for M = 128 as many flops per
// byte as the tensor cores can do while the bytes come from HBM at half their rate.  That is tcgen05's work
// (mma.sync reached a sixth of the bytes' rate here), in two kernels after a plan:
//
//   1. A group's rows x query heads, up to 128, are one tile of query vectors.  The blocks of 16 tokens that all
//      the rows hold in full go through the tensor cores as in the attention over prompts: S = Q K^T, a thread
//      per query vector for the softmax, O += P V.  A row that has more than 8 full blocks of its own after those
//      gets items of its own.  The whole is cut into equal shares.  Every item leaves normalised sums and log-sum-exps in fp32.
//   2. A warp per row and one or two key heads joins them, in order, with what is left of the row: up to 8 full blocks of its own
//      and the partly filled one, by mma.sync.  Here, where rows have nothing in common, no row's values come near
//      another row's sums.
//
// Kernel 1: blocks of 6 warps, two to an SM, so that one's softmax runs beside the other's products; 4 warps one
// thread per query vector, one warp the loads (a TMA box of 16 tokens x 64 values per block, page by page),
// one the MMAs.  Tensor memory: S 64 columns | O.  Tiles of 64 tokens, so that five of keys or values are on their way at a
// time (with two of 128 tokens the loads came too late: 54 us against 50 on 128 prompts of 500 to 1024 tokens).  A last tile of fewer than 4 blocks takes fewer steps of the
// second product, and its missing scores are masked, so that nothing stale is ever multiplied.  P is rounded to the inputs' type, the
// operand type of the second product; sums of the remainders apart from O, as the rows form has them, would need 320 of the 256
// columns of tensor memory that a block can have with two to an SM.

#include "disc_attend.cuh"

namespace {

using namespace disc;

constexpr unsigned FULL = 0xffffffffu;
constexpr float LN2_F = 0.6931471805599453f;
constexpr int TN = 64;                 // tokens of a tile
constexpr int TILE_BLKS = TN / BLK;
constexpr int BOX = 64;
constexpr int Q_BOX_BYTES = GROUP_M * BOX * 2;
constexpr int MIN_SHARED = 4;          // blocks: less is not worth an item
constexpr int MAX_TAIL = 8;            // full blocks that kernel 2 takes along

// ---- the plan ---------------------------------------------------------------------------------------
// A block per group: the leading pages that its rows share, and what rows have left.  Rows without tokens need no pages and are
// left out; what the tile of the group adds up for them is not joined.
__global__ void __launch_bounds__(256) group_shared_kernel(const PlanParams p) {
    let_later_in();
    wait_for_earlier();
    __shared__ int32_t s_shared, s_lead[8], s_len[GROUP_M];
    const PlanShape& sh = p.shape;
    const int g = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t r0 = g / sh.sub * sh.group + g % sh.sub * sh.per_group;
    const int32_t r1 = min(p.rows, min(r0 + sh.per_group, g / sh.sub * sh.group + sh.group));
    if (threadIdx.x == 0) s_shared = 0x7fffffff;
    const int32_t own = r0 + int32_t(threadIdx.x), own_len = own < r1 ? p.len[own] : 0;      // at most GROUP_M rows
    if (own < r1) s_len[threadIdx.x] = own_len;
    const int32_t warp_lead = __reduce_min_sync(FULL, own_len > 0 ? own : max(r0, r1));
    if (lane == 0) s_lead[warp] = warp_lead;
    __syncthreads();
    const int32_t lead = __reduce_min_sync(FULL, s_lead[lane & 7]);
    const int32_t* first = p.table + int64_t(lead) * p.width;
    for (int32_t r = r0 + warp; r < r1; r += 8) {
        const int32_t len = s_len[r - r0];
        if (len == 0) continue;
        const int32_t full = min(s_len[lead - r0], len) >> p.shift;
        int32_t same = full;
        if (r > lead) {
            const int32_t* row = p.table + int64_t(r) * p.width;
            for (int32_t j0 = 0; j0 < full; j0 += 64) {
                const int32_t j = j0 + lane, j2 = j + 32;
                const bool a = j >= full || first[j] == row[j], b = j2 >= full || first[j2] == row[j2];
                const unsigned da = __ballot_sync(FULL, !a), db = __ballot_sync(FULL, !b);
                if (da | db) {
                    same = da ? j0 + __ffs(da) - 1 : j0 + 31 + __ffs(db);
                    break;
                }
            }
        }
        if (lane == 0) atomicMin(&s_shared, same);
    }
    __syncthreads();
    int32_t blks = lead < r1 ? s_shared * sh.blks_per_page : 0;
    if (blks < MIN_SHARED) blks = 0;
    if (threadIdx.x == 0) { p.plan.shared[g] = blks; p.plan.lead[g] = lead; }
    if (own < r1) {
        const int32_t left = own_len / BLK - blks;
        p.plan.alone[own] = left > MAX_TAIL ? left : 0;
    }
}

// Exclusive sums over the block of two numbers; all: the whole sums.  Called by the whole block.
constexpr int PT = 1024;
__device__ __forceinline__ int2 block_sums(int32_t a, int32_t b, int2 (*sums), int2* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t ia = a, ib = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t ua = __shfl_up_sync(FULL, ia, o), ub = __shfl_up_sync(FULL, ib, o);
        if (lane >= o) { ia += ua; ib += ub; }
    }
    __syncthreads();
    if (lane == 31) sums[warp] = make_int2(ia, ib);
    __syncthreads();
    int2 w = sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t ua = __shfl_up_sync(FULL, w.x, o), ub = __shfl_up_sync(FULL, w.y, o);
        if (lane >= o) { w.x += ua; w.y += ub; }
    }
    *all = make_int2(__shfl_sync(FULL, w.x, 31), __shfl_sync(FULL, w.y, 31));
    const int32_t ba = __shfl_sync(FULL, w.x, max(warp - 1, 0)), bb = __shfl_sync(FULL, w.y, max(warp - 1, 0));
    return make_int2(ia - a + (warp ? ba : 0), ib - b + (warp ? bb : 0));
}

// One block: a lane's share, and the items, groups first, then rows.
__global__ void __launch_bounds__(PT) group_items_kernel(const PlanParams p) {
    let_later_in();
    wait_for_earlier();
    __shared__ int2 sums[32];
    __shared__ int32_t s_all;
    const PlanShape& sh = p.shape;
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid == 0) s_all = 0;
    __syncthreads();
    int32_t mine = 0, alone = 0;
    auto place = [](int32_t blks) { return blks > 0 ? blks + START : 0; };
    for (int32_t g = tid; g < sh.groups; g += PT) mine += place(p.plan.shared[g]);
    for (int32_t r = tid; r < p.rows; r += PT) alone += place(p.plan.alone[r]);
    mine += alone;
    const int any_alone = __syncthreads_or(alone > 0);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(FULL, mine, o);
    if (lane == 0 && mine) atomicAdd(&s_all, mine);
    __syncthreads();
    const int32_t all = s_all;
    const int32_t share = max(TILE_BLKS, ((all - 1) / sh.lanes + TILE_BLKS) / TILE_BLKS * TILE_BLKS);
    const int32_t lanes = all / share + (all % share > 0);
    int32_t items = 0, part = 0, blocks = 0;
    for (int kind = 0; kind < 2; ++kind) {
        const int32_t n = kind == 0 ? sh.groups : p.rows;
        for (int32_t i0 = 0; i0 < n; i0 += PT) {
            const int32_t i = i0 + tid;
            if (kind == 1 && !any_alone) {
                if (i < n) p.plan.row_part[i] = make_int2(0, 0);
                continue;
            }
            int32_t blks = 0, row = 0, rows = 1, first = 0, lead = 0;
            if (i < n) {
                if (kind == 0) {
                    blks = p.plan.shared[i];
                    lead = p.plan.lead[i];
                    row = i / sh.sub * sh.group + i % sh.sub * sh.per_group;
                    rows = max(0, min(p.rows, min(row + sh.per_group, i / sh.sub * sh.group + sh.group)) - row);
                } else {
                    blks = p.plan.alone[i];
                    row = lead = i;
                    if (blks) first = p.plan.shared[i / sh.group * sh.sub + i % sh.group / sh.per_group];
                }
            }
            int2 total;
            const int32_t at = blocks + block_sums(place(blks), 0, sums, &total).x;
            blocks += total.x;
            const Cut cut = cut_group(at, blks, share);
            const int32_t parts = cut.splits * rows * sh.G * p.kv_heads;
            const int2 before = block_sums(cut.splits, parts, sums, &total);
            const int32_t item0 = items + before.x, part0 = part + before.y;
            items += total.x;
            part += total.y;
            if (i < n) (kind == 0 ? p.plan.group_part : p.plan.row_part)[i] = make_int2(part0, cut.splits);
            for (int32_t x = 0; x < cut.splits; ++x) {
                const int32_t border = (cut.from + x) * share - at, begin = max(0, border), end = min(blks, border + share);
                p.plan.group_items[item0 + x] = GroupItem{row, rows, first + begin, first + end, part0 + x * rows * sh.G * p.kv_heads, lead, {0, 0}};
            }
            if (blks > 0) first_items(p.plan.first, at, blks, share, cut, item0, cut.splits);
        }
    }
    __syncthreads();
    for (int32_t i = lanes + tid; i <= sh.lanes; i += PT) p.plan.first[i] = items;
}

// ---- kernel 1 -----------------------------------------------------------------------------------------
constexpr int THREADS = 192;
template <int DP>
struct Shape {
    static constexpr int BOXES = DP / BOX;
    static constexpr int BOX_BYTES = TN * BOX * 2;
    static constexpr int TILE_BYTES = BOXES * BOX_BYTES;
    static constexpr int Q_BYTES = BOXES * Q_BOX_BYTES;
    static constexpr int STAGES = DP == 128 ? 5 : 10;              // with Q as much as two blocks fit into an SM
    static constexpr int TMEM = 256;                               // columns: S 64, O up to 128
    static constexpr int BARRIERS = 5 + 2 * STAGES;
    static constexpr int SMEM = Q_BYTES + STAGES * TILE_BYTES + BARRIERS * 8 + 16;
};

struct GroupParams {
    Plan plan;
    const int32_t* table;
    int32_t width, kv_heads, G, per_group, D, page_size, blks_per_page;
    float c2;
    uint32_t* error;
    uint32_t idesc_qk, idesc_pv;
};

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS, 2)
attend_group_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v, const GroupParams p) {
    using S = Shape<DP>;
    extern __shared__ __align__(1024) unsigned char q_tile[];      // nothing else is in shared memory: it begins on a swizzle atom
    unsigned char* ring = q_tile + S::Q_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + S::STAGES * S::TILE_BYTES);
    uint64_t* q_full = bars;
    uint64_t* q_empty = bars + 1;
    uint64_t* s_full = bars + 2;
    uint64_t* o_full = bars + 3;
    uint64_t* p_full = bars + 4;
    uint64_t* kv_full = bars + 5;
    uint64_t* kv_empty = bars + 5 + S::STAGES;
    uint32_t& tmem_slot = *reinterpret_cast<uint32_t*>(bars + S::BARRIERS);
    int& s_abort = *reinterpret_cast<int*>(bars + S::BARRIERS + 1);
    volatile int* abort = &s_abort;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        s_abort = 0;
        mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(s_full, 1); mbar_init(o_full, 1); mbar_init(p_full, 4);
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(kv_full + s, 1); mbar_init(kv_empty + s, 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(S::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_slot);

    let_later_in();
    wait_for_earlier();
    // this block's lane and key head
    const int lane_of = blockIdx.x / p.kv_heads, head = blockIdx.x % p.kv_heads;
    const int item0 = p.plan.first[lane_of], item1 = p.plan.first[lane_of + 1];

    if (warp >= 4) {
        if (warp == 4) {
            // ---- loads
            int load = 0, n = 0;
            bool ok = true;
            for (; item0 + n < item1 && ok; ++n) {
                const GroupItem* it = p.plan.group_items + item0 + n;
                const int row = it->row, begin = it->begin, blks = it->end - begin;
                const int32_t* table = p.table + int64_t(it->lead) * p.width;
                if (n > 0) ok = mbar_wait_all(q_empty, (n - 1) & 1, abort);
                if (ok && lane == 0) {
                    mbar_expect_tx(q_full, uint32_t(S::BOXES) * p.G * p.per_group * BOX * 2);
                    for (int b = 0; b < S::BOXES; ++b) tma_load_3d(q_tile + b * Q_BOX_BYTES, &map_q, b * BOX, head * p.G, row, q_full);
                }
                for (int t = 0; t < blks && ok; t += TILE_BLKS) {
                    const int here = min(TILE_BLKS, blks - t);
                    // lane l brings in block l % 4: its keys, then its values
                    const int b = lane % TILE_BLKS, blk = begin + t + b;
                    int y = 0;
                    if (b < here) y = (table[blk / p.blks_per_page] * p.kv_heads + head) * p.page_size + blk % p.blks_per_page * BLK;
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv, ++load) {
                        const int s = load % S::STAGES, round = load / S::STAGES;
                        if (round > 0 && ok) ok = mbar_wait_all(kv_empty + s, (round - 1) & 1, abort);
                        if (!ok) continue;
                        if (lane == 0) mbar_expect_tx(kv_full + s, uint32_t(here) * S::BOXES * BLK * BOX * 2);
                        __syncwarp();
                        if (lane < TILE_BLKS && b < here)
                            for (int x = 0; x < S::BOXES; ++x)
                                tma_load_2d(ring + s * S::TILE_BYTES + x * S::BOX_BYTES + b * (BLK * BOX * 2), kv ? &map_v : &map_k, x * BOX, y, kv_full + s);
                        __syncwarp();
                    }
                }
            }
        } else if (warp == 5) {
            // ---- MMAs
            const uint64_t q_desc = smem_desc_sw128(q_tile), kv_desc = smem_desc_sw128(ring), v_desc = smem_desc_n_major(ring, S::BOX_BYTES);
            constexpr uint64_t TILE16 = S::TILE_BYTES >> 4;
            auto scores = [&](int stage) {
                const uint64_t kd = kv_desc + uint64_t(stage) * TILE16;
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) {
                    umma_ss(tmem, q_desc + uint64_t((kk / 4) * (Q_BOX_BYTES >> 4) + (kk % 4) * 2), kd + uint64_t((kk / 4) * (S::BOX_BYTES >> 4) + (kk % 4) * 2),
                            p.idesc_qk, kk > 0);
                }
            };
            int load = 0, n = 0, tile = 0;
            bool ok = true;
            for (; item0 + n < item1 && ok; ++n) {
                const GroupItem* it = p.plan.group_items + item0 + n;
                const int blks = it->end - it->begin;
                ok = mbar_wait_all(q_full, n & 1, abort) && mbar_wait_all(kv_full + load % S::STAGES, (load / S::STAGES) & 1, abort);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    scores(load % S::STAGES);
                    umma_commit(s_full);
                    umma_commit(kv_empty + load % S::STAGES);
                    if (blks <= TILE_BLKS) umma_commit(q_empty);
                }
                __syncwarp();
                ++load;
                for (int t = 0; t < blks && ok; t += TILE_BLKS, ++tile) {
                    const int here = min(TILE_BLKS, blks - t);
                    const bool more = t + TILE_BLKS < blks;
                    const int v_stage = load % S::STAGES, k_stage = (load + 1) % S::STAGES;
                    ok = mbar_wait_all(kv_full + v_stage, (load / S::STAGES) & 1, abort);
                    if (ok) ok = mbar_wait_all(p_full, tile & 1, abort);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t vd = v_desc + uint64_t(v_stage) * TILE16;
                        for (int kk = 0; kk < here; ++kk)
                            umma_ts(tmem + TN, tmem + kk * 8, vd + uint64_t(kk * (BLK * 128 >> 4)), p.idesc_pv, t > 0 || kk > 0);
                        umma_commit(kv_empty + v_stage);
                        if (!more) umma_commit(o_full);
                    }
                    __syncwarp();
                    ++load;
                    if (more) {
                        ok = mbar_wait_all(kv_full + k_stage, (load / S::STAGES) & 1, abort);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
                            scores(k_stage);
                            umma_commit(s_full);
                            umma_commit(kv_empty + k_stage);
                            if (t + 2 * TILE_BLKS >= blks) umma_commit(q_empty);
                        }
                        __syncwarp();
                        ++load;
                    }
                }
            }
            // the last reports of free places have arrived before the block leaves
            for (int back = 0; back < S::STAGES && back < load && ok; ++back)
                ok = mbar_wait_all(kv_empty + (load - 1 - back) % S::STAGES, ((load - 1 - back) / S::STAGES) & 1, abort);
            if (ok && n > 0) mbar_wait_all(q_empty, (n - 1) & 1, abort);
        }
    } else {
        // ---- softmax: this thread's query vector
        const int m = warp * 32 + lane;
        const uint32_t lane_bits = uint32_t(warp * 32) << 16;
        const uint32_t s_tm = tmem + lane_bits, o_tm = tmem + lane_bits + TN;
        const float2 c2 = make_float2(p.c2, p.c2);
        int tile = 0, n = 0;
        bool ok = true;
        for (; item0 + n < item1 && ok; ++n) {
            const GroupItem* it = p.plan.group_items + item0 + n;
            const int blks = it->end - it->begin;
            float ref = -CUDART_INF_F;
            float2 l = make_float2(0.f, 0.f);
            bool bad = false;
            for (int t = 0; t < blks; t += TILE_BLKS, ++tile) {
                ok = mbar_wait_all(s_full, tile & 1, abort);
                if (!ok) break;
                tc_fence_after();
                float s[TN];
                tmem_ld64(s_tm, s);
                const int here = min(TILE_BLKS, blks - t) * BLK;
                if (here < TN) {
#pragma unroll
                    for (int c = 0; c < TN; ++c) s[c] = c < here ? s[c] : -CUDART_INF_F;
                }
                uint32_t pk[16];
                float2 la;
                first_scores<T, DP, TN>(s, c2, ref, l, bad, o_tm, t > 0, la, pk);
                tmem_st16(s_tm, pk);
                const float base = ref > -CUDART_INF_F ? ref : 0.f;
                exp_chunk<T>(s + 32, c2, make_float2(-base, -base), la, pk);
                tmem_st16(s_tm + 16, pk);
                l = add2(l, la);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full);
            }
            if (!ok) break;
            ok = mbar_wait_all(o_full, n & 1, abort);
            if (!ok) break;
            tc_fence_after();
            const float total = bad ? CUDART_NAN_F : l.x + l.y;
            const float inv = total > 0.f ? 1.f / total : (total == 0.f ? 0.f : total);
            const int rows = it->rows * p.G;
            const int64_t at = int64_t(it->part) + head * rows + m;
            float* dst = p.plan.part + at * p.D;
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
                uint32_t o[32];
                tmem_ld32(o_tm + c, o);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * inv);
#pragma unroll
                for (int e = 0; e < 32; e += 8)
                    if (m < rows && c + e < p.D) st_global32(dst + c + e, o + e);
            }
            if (m < rows) p.plan.part_lse[at] = total > 0.f ? ref + log2f(total) : (total == 0.f ? -CUDART_INF_F : total);
            tc_fence_before();                        // O has been read before the next unit's first probabilities are reported
        }
    }

    tc_fence_before();
    __syncthreads();
    if (s_abort && threadIdx.x == 0) {
        atomicExch(p.error, 1u);
        for (int i = 0; i < 200; ++i) __nanosleep(1000);          // copies in flight land before the memory is given up
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM) : "memory");
    }
}

// ---- kernel 2 -----------------------------------------------------------------------------------------
constexpr int JT = 128;                // threads of a block: 4 warps, each with a row and key head of its own

// an 8 x 8 matrix of 16-bit values across the warp, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

template <int DP>
struct JoinSmem {
    static constexpr int O_LD = DP + 4;                            // fp32 sums [8 heads][DP], over keys and values no longer needed
    static constexpr int BLOCK_BYTES = BLK * DP * 2;
    static constexpr int WARP_BYTES = 4 * BLOCK_BYTES + 256;       // keys and values of two blocks; maximum and sum of 8 heads
    static_assert(8 * O_LD * 4 <= 2 * BLOCK_BYTES, "the sums fit over a block");
};

// The products are taken the other way round, S^T = K Q^T and O^T = V^T P^T: 8 query heads are then the narrow side of
// m16n8k16, where rows of queries would leave 12 of 16 rows empty with 4 heads, and hold twice the registers (101 us that
// way on 4096 rows x 4 key heads).  A warp goes through one or two key heads of its row (the launch says why) and has the
// next block's loads in flight under the present one's products (78 us without).
// EXACT: the head dim is DP itself, and all strides and ends along it are known.
template <typename T, int DP, bool EXACT>
__global__ void __launch_bounds__(JT, 3) attend_join_kernel(const AttendParams p, int heads_per_job) {
    let_later_in();
    wait_for_earlier();
    using S = JoinSmem<DP>;
    constexpr int CH = DP / 8;
    const int D = EXACT ? DP : p.D;
    extern __shared__ __align__(1024) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int jobs_per_row = (p.kv_heads + heads_per_job - 1) / heads_per_job;
    const int64_t job = int64_t(blockIdx.x) * (JT / 32) + warp;
    if (job >= int64_t(p.rows) * jobs_per_row) return;
    const int row = int(job / jobs_per_row), head0 = int(job % jobs_per_row) * heads_per_job;
    const int head1 = min(p.kv_heads, head0 + heads_per_job);
    const PlanShape& sh = p.shape;
    const int G = sh.G;
    const int g = row / sh.group * sh.sub + row % sh.group / sh.per_group, k_row = row % sh.group % sh.per_group;
    const int first_row = row - k_row;
    const int group_rows = min(p.rows, min(first_row + sh.per_group, row / sh.group * sh.group + sh.group)) - first_row;
    const int32_t len = p.len[row];
    const int2 gp = p.plan.group_part[g], rp = p.plan.row_part[row];
    const int begin = p.plan.shared[g] + p.plan.alone[row], left = (len + BLK - 1) / BLK - begin;      // blocks; none without tokens
    const int32_t* table = p.table + int64_t(row) * p.width;
    const int64_t head_bytes = int64_t(p.page_size) * D * 2;
    unsigned char* own = smem + warp * S::WARP_BYTES;
    float* ml_sm = reinterpret_cast<float*>(own + 4 * S::BLOCK_BYTES);     // [8] maxima, [8] sums
    const int eights = (G + 7) / 8;                    // a key head's query heads, eight at a time
    const int steps = (head1 - head0) * eights * left;

    // step: block step % left of the (step / left)-th eight of query heads; a row's pages are the same for all heads, a lane
    // holds the page of one of its blocks (there are at most 9)
    int my_page = lane < left ? table[(begin + lane) / sh.blks_per_page] : 0;
    if (unsigned(my_page) >= unsigned(p.pages)) my_page = 0;      // a plan older than the books: no place outside the pool is read
    static_assert(MAX_TAIL < 32, "a lane per block");
    const int lane_src = lane / CH * (D * 2) + lane % CH * 16;
    const uint32_t lane_dst = chunk_at<DP>(lane / CH, lane % CH);
    int load_unit = 0, load_blk = 0;                   // of the next step to be loaded
    auto load_step = [&](int step) {
        if (step < steps) {
            const int head = head0 + load_unit / eights, blk = begin + load_blk;
            const int page = __shfl_sync(FULL, my_page, load_blk), tokens = min(BLK, len - blk * BLK);
            if (++load_blk == left) { load_blk = 0; ++load_unit; }
            const int64_t off = (int64_t(page) * p.kv_heads + head) * head_bytes + int64_t(blk % sh.blks_per_page) * (BLK * 2) * D + lane_src;
            const unsigned char* k_src = p.k + off;
            const unsigned char* v_src = p.v + off;
            const uint32_t k_at = smem_u32(own) + (step & 1) * 2 * S::BLOCK_BYTES;
#pragma unroll
            for (int j = 0; j < BLK * CH / 32; ++j) {
                const bool some = j * (32 / CH) + lane / CH < tokens && (EXACT || lane % CH * 8 < D);
                // rows j (32 / CH) + lane / CH: what chunk_at() mixes in from the row is the lane's and j's part apart
                const uint32_t dst = k_at + (lane_dst ^ uint32_t(((j * (32 / CH)) & 7) << 4)) + j * 512;
                cp16(dst, some ? k_src + j * (32 / CH) * (D * 2) : p.k, some);
                cp16(dst + S::BLOCK_BYTES, some ? v_src + j * (32 / CH) * (D * 2) : p.v, some);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    load_step(0);

    int step = 0;
    for (int unit = 0; unit < (head1 - head0) * eights; ++unit) {
        const int head = head0 + unit / eights, g0 = unit % eights * 8;
        const int heads = min(8, G - g0);
        const int64_t out_at = (int64_t(row) * p.kv_heads + head) * G;
        float* o_sm = reinterpret_cast<float*>(own);
        if (left > 0) {
            // query fragments: head lane / 4, values 16 kk + 2 (lane % 4) and 8 further
            uint32_t qf[DP / 16][2];
            const bool some_head = (lane >> 2) < heads;
            const unsigned char* q = p.q + row * p.q_row + (head * G + g0 + (lane >> 2)) * p.q_head + (lane & 3) * 4;
#pragma unroll
            for (int kk = 0; kk < DP / 16; ++kk) {
                qf[kk][0] = some_head && kk * 16 < D ? *reinterpret_cast<const uint32_t*>(q + kk * 32) : 0u;
                qf[kk][1] = some_head && kk * 16 + 8 < D ? *reinterpret_cast<const uint32_t*>(q + kk * 32 + 16) : 0u;
            }
            // this thread's two heads: 2 (lane % 4) and the next
            float o[DP / 16][4];
#pragma unroll
            for (int j = 0; j < DP / 16; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
            float m0 = -CUDART_INF_F, m1 = -CUDART_INF_F, l0 = 0.f, l1 = 0.f;
            for (int i = 0; i < left; ++i, ++step) {
                __syncwarp();                          // what the next loads overwrite has been read by all lanes
                load_step(step + 1);
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                __syncwarp();
                const int tokens = min(BLK, len - (begin + i) * BLK);
                const uint32_t k_at = smem_u32(own) + (step & 1) * 2 * S::BLOCK_BYTES, v_at = k_at + S::BLOCK_BYTES;
                float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) {
                    uint32_t kf[4];
                    ldsm4((k_at + chunk_at<DP>(lane & 15, lane >> 4)) ^ uint32_t(kk << 5), kf);
                    mma16<T>(s, kf, qf[kk][0], qf[kk][1]);
                }
                // tokens lane / 4 (s[0], s[1]) and 8 further (s[2], s[3])
                const bool a = (lane >> 2) < tokens, b = (lane >> 2) + 8 < tokens;
                s[0] = a ? s[0] * p.c2 : -CUDART_INF_F;
                s[1] = a ? s[1] * p.c2 : -CUDART_INF_F;
                s[2] = b ? s[2] * p.c2 : -CUDART_INF_F;
                s[3] = b ? s[3] * p.c2 : -CUDART_INF_F;
                float mx0 = fmaxf(s[0], s[2]), mx1 = fmaxf(s[1], s[3]);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    mx0 = fmaxf(mx0, __shfl_xor_sync(FULL, mx0, x));
                    mx1 = fmaxf(mx1, __shfl_xor_sync(FULL, mx1, x));
                }
                const float n0 = fmaxf(m0, mx0), n1 = fmaxf(m1, mx1);
                if (i > 0 && __any_sync(FULL, n0 > m0 || n1 > m1)) {
                    const float f0 = m0 > -CUDART_INF_F ? ex2_approx(m0 - n0) : 0.f, f1 = m1 > -CUDART_INF_F ? ex2_approx(m1 - n1) : 0.f;
                    l0 *= f0;
                    l1 *= f1;
#pragma unroll
                    for (int j = 0; j < DP / 16; ++j) { o[j][0] *= f0; o[j][1] *= f1; o[j][2] *= f0; o[j][3] *= f1; }
                }
                m0 = n0;
                m1 = n1;
                const float ref0 = m0 > -CUDART_INF_F ? m0 : 0.f, ref1 = m1 > -CUDART_INF_F ? m1 : 0.f;
                s[0] = ex2_approx(s[0] - ref0);
                s[1] = ex2_approx(s[1] - ref1);
                s[2] = ex2_approx(s[2] - ref0);
                s[3] = ex2_approx(s[3] - ref1);
                l0 += s[0] + s[2];
                l1 += s[1] + s[3];
                const uint32_t p0 = transposed(pack2<T>(s[0], s[1])), p1 = transposed(pack2<T>(s[2], s[3]));
#pragma unroll
                for (int j = 0; j < DP / 16; ++j) {
                    uint32_t vf[4];
                    ldsm4t((v_at + chunk_at<DP>((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1)) ^ uint32_t(j << 5), vf);
                    mma16<T>(o[j], vf, p0, p1);
                }
            }
            __syncwarp();
            o_sm = reinterpret_cast<float*>(own + ((step - 1) & 1) * 2 * S::BLOCK_BYTES);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) {
                l0 += __shfl_xor_sync(FULL, l0, x);
                l1 += __shfl_xor_sync(FULL, l1, x);
            }
            float* dst = o_sm + (lane & 3) * 2 * S::O_LD + (lane >> 2);
#pragma unroll
            for (int j = 0; j < DP / 16; ++j) {
                dst[16 * j] = o[j][0];
                dst[S::O_LD + 16 * j] = o[j][1];
                dst[16 * j + 8] = o[j][2];
                dst[S::O_LD + 16 * j + 8] = o[j][3];
            }
            if (lane < 4) {
                ml_sm[2 * lane] = m0; ml_sm[2 * lane + 1] = m1;
                ml_sm[8 + 2 * lane] = l0; ml_sm[8 + 2 * lane + 1] = l1;
            }
            __syncwarp();
        }
        // the parts, in order: the group's items, then the row's own, then what was just added up.  A lane takes 4 values of
        // up to four heads at a time, so that their loads are in flight together.
        constexpr int AT_ONCE = 4;
        const int64_t g_at = int64_t(gp.x) + int64_t(head) * group_rows * G + k_row * G + g0, g_step = int64_t(p.kv_heads) * group_rows * G;
        const int64_t r_at = int64_t(rp.x) + int64_t(head) * G + g0, r_step = int64_t(p.kv_heads) * G;
        for (int i0 = lane; i0 < heads * (DP / 4); i0 += 32 * AT_ONCE) {
            float m[AT_ONCE], total[AT_ONCE];
            float4 x[AT_ONCE];
            int h[AT_ONCE];
            bool some[AT_ONCE];
            const int d = i0 % (DP / 4) * 4;           // the same for all of a lane's heads: 32 is a multiple of DP / 4, or the other way round
#pragma unroll
            for (int a = 0; a < AT_ONCE; ++a) {
                h[a] = (i0 + 32 * a) / (DP / 4);
                some[a] = h[a] < heads && d < D;
                m[a] = -CUDART_INF_F;
                total[a] = 0.f;
                x[a] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            auto add = [&](int a, float lse, float weight, const float4& y) {
                const float n = fmaxf(m[a], lse);
                const float f = m[a] > -CUDART_INF_F ? ex2_approx(m[a] - n) : 0.f, w = lse == -CUDART_INF_F ? 0.f : ex2_approx(lse - n);
                m[a] = n;
                total[a] = fmaf(total[a], f, w * weight);
                x[a] = make_float4(fmaf(w, y.x, x[a].x * f), fmaf(w, y.y, x[a].y * f), fmaf(w, y.z, x[a].z * f), fmaf(w, y.w, x[a].w * f));
            };
            auto take = [&](int64_t at) {
                float lse[AT_ONCE];
                float4 y[AT_ONCE];
#pragma unroll
                for (int a = 0; a < AT_ONCE; ++a) {
                    lse[a] = some[a] ? p.plan.part_lse[at + h[a]] : -CUDART_INF_F;
                    y[a] = some[a] ? *reinterpret_cast<const float4*>(p.plan.part + (at + h[a]) * D + d) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
                for (int a = 0; a < AT_ONCE; ++a) add(a, lse[a], 1.f, y[a]);
            };
            for (int s = 0; s < gp.y && len > 0; ++s) take(g_at + s * g_step);
            for (int s = 0; s < rp.y; ++s) take(r_at + s * r_step);
#pragma unroll
            for (int a = 0; a < AT_ONCE; ++a) {
                if (!some[a]) continue;
                if (left > 0) {
                    const float mt = ml_sm[h[a]], lt = ml_sm[8 + h[a]];
                    if (mt > -CUDART_INF_F || lt != lt) add(a, mt > -CUDART_INF_F ? mt : 0.f, lt, *reinterpret_cast<const float4*>(o_sm + h[a] * S::O_LD + d));
                }
                const float inv = total[a] > 0.f ? 1.f / total[a] : (total[a] == 0.f ? 0.f : total[a]);
                *reinterpret_cast<uint2*>(p.out + ((out_at + g0 + h[a]) * D + d) * 2) =
                    make_uint2(pack2<T>(x[a].x * inv, x[a].y * inv), pack2<T>(x[a].z * inv, x[a].w * inv));
                if (d == 0 && p.lse) p.lse[out_at + g0 + h[a]] = total[a] > 0.f ? (m[a] + log2f(total[a])) * LN2_F : (total[a] == 0.f ? -CUDART_INF_F : total[a]);
            }
        }
    }
}

template <typename T, int DP>
int launch_groups(const AttendParams& a, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const GroupParams& p, unsigned grid, cudaStream_t st) {
    static std::atomic<uint64_t> done{0}, done2{0}, done3{0};
    constexpr int join_bytes = JT / 32 * JoinSmem<DP>::WARP_BYTES;
    if (const int rc = allow_smem(attend_group_kernel<T, DP>, Shape<DP>::SMEM, done)) return rc;
    if (const int rc = launch_after(attend_group_kernel<T, DP>, grid, THREADS, Shape<DP>::SMEM, st, q, k, v, p)) return rc;
    if (const int rc = allow_smem(attend_join_kernel<T, DP, true>, join_bytes, done2)) return rc;
    if (const int rc = allow_smem(attend_join_kernel<T, DP, false>, join_bytes, done3)) return rc;
    int sms = 0;
    if (const int rc = device_sms(&sms)) return rc;
    const int64_t places = int64_t(sms) * 3 * (JT / 32), units = int64_t(a.rows) * a.kv_heads;
    // a warp takes two key heads of a row if that leaves a job for every warp that runs at a time: the row's books are read once
    // and the second head's blocks come in under the first's sums (4096 rows of 4 heads: 120.4 us for plan and attention; one
    // head 124.3, all four 123.4, as the warps are then through 2.3 times)
    const int heads_per_job = units >= 2 * places && a.kv_heads > 1 ? 2 : 1;
    const int64_t jobs = int64_t(a.rows) * ((a.kv_heads + heads_per_job - 1) / heads_per_job);
    const unsigned join_grid = unsigned((jobs + JT / 32 - 1) / (JT / 32));
    return launch_after(a.D == DP ? attend_join_kernel<T, DP, true> : attend_join_kernel<T, DP, false>, join_grid, JT, join_bytes, st, a, heads_per_job);
}

int encode(EncodeTiled enc, CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
           const cuuint32_t* box) {
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = enc(map, type, cuuint32_t(rank), const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DISC_OK : DISC_ERR_UNSUPPORTED;
}

}  // namespace

int disc::plan_groups(const PlanParams& p, cudaStream_t st) {
    if (const int rc = launch_after(group_shared_kernel, unsigned(p.shape.groups), 256, 0, st, p)) return rc;
    return launch_after(group_items_kernel, 1, PT, 0, st, p);
}

int disc::attend_groups(const AttendParams& a, int32_t dtype, int32_t n_q_heads, cudaStream_t st) {
    GroupParams p;
    p.plan = a.plan; p.table = a.table; p.width = a.width; p.kv_heads = a.kv_heads; p.G = a.shape.G; p.per_group = a.shape.per_group;
    p.D = a.D; p.page_size = a.page_size; p.blks_per_page = a.shape.blks_per_page; p.c2 = a.c2; p.error = a.error;
    const int DP = a.D <= 64 ? 64 : 128;
    // instruction descriptors: D fp32 (bits 4-5 = 1), A and B f16 = 0 / bf16 = 1 (bits 7-9, 10-12), B of the second
    // product N-major (bit 16), N >> 3 at bit 17, M >> 4 at bit 24
    const uint32_t ty = dtype == DISC_BF16 ? 1u : 0u;
    const uint32_t idesc = (1u << 4) | (ty << 7) | (ty << 10) | (uint32_t(GROUP_M >> 4) << 24);
    p.idesc_qk = idesc | (uint32_t(TN >> 3) << 17);
    p.idesc_pv = idesc | (uint32_t(DP >> 3) << 17) | (1u << 16);
    EncodeTiled enc = nullptr;
    if (const int rc = tensor_map_encoder(&enc)) return rc;
    const CUtensorMapDataType type = dtype == DISC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    alignas(64) CUtensorMap map_q, map_k, map_v;
    if (a.q_row <= 0 || a.q_head <= 0) return DISC_ERR_UNSUPPORTED;
    const cuuint64_t q_dims[3] = {cuuint64_t(a.D), cuuint64_t(n_q_heads), cuuint64_t(a.rows)}, q_strides[2] = {cuuint64_t(a.q_head), cuuint64_t(a.q_row)};
    const cuuint32_t q_box[3] = {cuuint32_t(BOX), cuuint32_t(p.G), cuuint32_t(p.per_group)};
    if (const int rc = encode(enc, &map_q, type, 3, a.q, q_dims, q_strides, q_box)) return rc;
    // a plane as [pages x heads x page size][D]
    const cuuint64_t dims[2] = {cuuint64_t(a.D), cuuint64_t(a.pages) * a.kv_heads * a.page_size}, strides[1] = {cuuint64_t(a.D) * 2};
    const cuuint32_t box[2] = {cuuint32_t(BOX), cuuint32_t(BLK)};
    if (const int rc = encode(enc, &map_k, type, 2, a.k, dims, strides, box)) return rc;
    if (const int rc = encode(enc, &map_v, type, 2, a.v, dims, strides, box)) return rc;
    const unsigned grid = unsigned(a.shape.lanes * a.kv_heads);
    if (dtype == DISC_BF16)
        return DP == 64 ? launch_groups<__nv_bfloat16, 64>(a, map_q, map_k, map_v, p, grid, st) : launch_groups<__nv_bfloat16, 128>(a, map_q, map_k, map_v, p, grid, st);
    return DP == 64 ? launch_groups<__half, 64>(a, map_q, map_k, map_v, p, grid, st) : launch_groups<__half, 128>(a, map_q, map_k, map_v, p, grid, st);
}
