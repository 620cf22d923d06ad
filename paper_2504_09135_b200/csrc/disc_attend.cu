// disc_attend_cached: attention of one new token per row over a key-value cache in pages, and
// disc_attend_plan: how its work is cut.
//
//   out[r] = sum_j p_j v_j,  p = softmax_j(scale q[r] k_j),  lse = log sum_j e^{scale q[r] k_j}
//
// The K candidates of a query hold the pages of its prompt in common.  Read row by row they would
// cross HBM or L2 K times; here the rows of a group and the query heads that read the same key head
// make up one tile of M = rows x heads query vectors, and a page that all its rows hold is read once.  The pages
// that a row has for itself follow in the same stream, each with its owner, and the other rows' scores are
// set to -inf there.  What bounds the kernel is then the bytes of the distinct pages.
//
// Two forms, by the number M of query vectors that read the same pages (rows of the group x query heads per
// key head).  M <= 16, this file: mma.sync m16n8k16 on one tile of 16 rows, far from being the bound.  M > 16,
// disc_attend_group.cu: tcgen05 on tiles of 128 rows.  M <= 16 over a cache held in 8 bits: disc_attend_held.cu, by the plan made here.
//
// Plan (one cluster of 8 blocks): per group the number of leading pages its rows share, and the stream as a
// list of blocks of 16 tokens (page, block in the page, tokens in it, owner); from the lengths of
// the lists the items: every block of threads that runs at a time gets an equal share of all blocks.
//
// Attention: a block of 4 warps per share and key head; blocks of 16 tokens come in through cp.async, three
// tiles of 64 tokens deep.  Every warp takes its own block of 16 tokens of a tile with all the rows, so that the
// warps need no barrier in the loop; their results are joined at the end.
// Running maximum and sum per row in fp32, in units of log2.  An item that is not its group's only one
// writes its rows' normalised sum and log-sum-exp; the block that finishes last joins them in the
// order of the items.
// Measured on 64 rows of 1 to 8191 tokens, 32 / 8 heads of 128, bf16: 160 us for 1.04 GB, the measured copy rate.

#include "disc_attend.cuh"

namespace {

using namespace disc;

constexpr unsigned FULL = 0xffffffffu;
constexpr float LOG2E_F = 1.4426950408889634f;
constexpr int TILE_BLKS = 4;           // blocks of a tile
constexpr int TILE = BLK * TILE_BLKS;
constexpr int STAGES = 3;
constexpr int CLUSTER = 8;
constexpr int PT = 512;                // threads of a plan block

// ---- the plan ---------------------------------------------------------------------------------------

__device__ __forceinline__ int32_t warp_incl_scan(int32_t v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t u = __shfl_up_sync(FULL, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

template <int CL>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(PT) attend_plan_kernel(const PlanParams p) {
    let_later_in();
    wait_for_earlier();
    __shared__ int32_t warp_sums[32][3];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const PlanShape& sh = p.shape;
    const int32_t bpp = sh.blks_per_page;

    // a warp per group: the leading pages that its rows share, and its list of blocks
    for (int32_t g = blockIdx.x * (PT / 32) + warp; g < sh.groups; g += CL * (PT / 32)) {
        const int32_t r0 = g / sh.sub * sh.group + g % sh.sub * sh.per_group;
        const int32_t r1 = min(p.rows, min(r0 + sh.per_group, g / sh.sub * sh.group + sh.group));
        int2* list = p.plan.list + int64_t(g) * sh.list_ld;
        const int32_t n = r1 - r0;
        if (sh.per_group == 1) {
            if (lane == 0) p.plan.count[g] = (p.len[r0] + BLK - 1) / BLK;
            continue;
        }
        int32_t shared = 0;
        if (n > 1) {
            // rows without tokens need no pages: the first that has some is what the others are compared with
            int32_t full = 0x7fffffff, lead = r1;
            for (int32_t r = r0 + lane; r < r1; r += 32) {
                const int32_t len = p.len[r];
                if (len > 0) { full = min(full, len >> p.shift); lead = min(lead, r); }
            }
            full = __reduce_min_sync(FULL, full);
            lead = __reduce_min_sync(FULL, lead);
            if (lead == r1) full = 0;
            const int32_t* first = p.table + int64_t(lead < r1 ? lead : r0) * p.width;
            shared = full;
            for (int32_t j0 = 0; j0 < full && shared == full; j0 += 32) {
                const int32_t j = j0 + lane;
                bool same = true;
                if (j < full) {
                    const int32_t page = first[j];
                    for (int32_t r = lead + 1; r < r1; ++r) same = same && (p.len[r] == 0 || p.table[int64_t(r) * p.width + j] == page);
                }
                const unsigned differ = __ballot_sync(FULL, !same);
                if (differ) shared = j0 + __ffs(differ) - 1;
            }
            for (int32_t i = lane; i < shared * bpp; i += 32) list[i] = make_int2(first[i / bpp], (i % bpp) | (BLK << 8));
        }
        int32_t at = shared * bpp;
        for (int32_t r = r0; r < r1; ++r) {
            const int32_t len = p.len[r];
            const int32_t blks = (len + BLK - 1) / BLK;
            const int32_t* pages = p.table + int64_t(r) * p.width;
            const int32_t owner = n > 1 ? (r - r0 + 1) << 16 : 0;
            for (int32_t i = shared * bpp + lane; i < blks; i += 32)
                list[at + i - shared * bpp] = make_int2(pages[i / bpp], (i % bpp) | (min(BLK, len - i * BLK) << 8) | owner);
            at += max(0, blks - shared * bpp);
        }
        if (lane == 0) p.plan.count[g] = at;
    }
    if (CL == 1) __syncthreads(); else cluster_sync_all();
    if (blockIdx.x != 0) return;

    // one block: how long a lane's share is, and the items
    int32_t sum = 0;
    for (int32_t g = tid; g < sh.groups; g += PT) sum += p.plan.count[g] + START;
    sum = warp_incl_scan(sum, lane);
    if (lane == 31) warp_sums[warp][0] = sum;
    __syncthreads();
    int32_t all = 0;
    for (int w = 0; w < PT / 32; ++w) all += warp_sums[w][0];
    __syncthreads();
    const int32_t share = max(TILE_BLKS, ((all - 1) / sh.lanes + TILE_BLKS) / TILE_BLKS * TILE_BLKS);
    const int32_t lanes = all / share + (all % share > 0);
    int32_t items = 0, slots = 0;
    int32_t blocks = 0;
    for (int32_t g0 = 0; g0 < sh.groups; g0 += PT) {
        const int32_t g = g0 + tid;
        const int32_t n = g < sh.groups ? p.plan.count[g] : 0;
        const int32_t place = g < sh.groups ? n + START : 0;
        const int32_t bs = warp_incl_scan(place, lane);
        __syncthreads();
        if (lane == 31) warp_sums[warp][0] = bs;
        __syncthreads();
        int32_t at = blocks + bs - place;
        for (int w = 0; w < PT / 32; ++w) {
            if (w < warp) at += warp_sums[w][0];
            blocks += warp_sums[w][0];
        }
        const Cut cut = cut_group(at, n, share);
        const int32_t splits = g < sh.groups ? max(1, cut.splits) : 0;         // an empty group is an item too: its rows get zeros
        const int32_t own_slots = splits > 1 ? splits : 0;
        const int32_t is = warp_incl_scan(splits, lane), ss = warp_incl_scan(own_slots, lane);
        if (lane == 31) { warp_sums[warp][1] = is; warp_sums[warp][2] = ss; }
        __syncthreads();
        int32_t i0 = items + is - splits, s0 = slots + ss - own_slots;
        for (int w = 0; w < PT / 32; ++w) {
            if (w < warp) { i0 += warp_sums[w][1]; s0 += warp_sums[w][2]; }
            items += warp_sums[w][1];
            slots += warp_sums[w][2];
        }
        if (g < sh.groups) {
            const int32_t r0 = g / sh.sub * sh.group + g % sh.sub * sh.per_group;
            const int32_t rows = max(0, min(p.rows, min(r0 + sh.per_group, g / sh.sub * sh.group + sh.group)) - r0);
            for (int32_t h = 0; h < p.kv_heads; ++h) p.plan.arrived[int64_t(g) * p.kv_heads + h] = 0;
            for (int32_t i = 0; i < splits; ++i) {
                const int32_t border = (cut.from + i) * share - at;            // from the group's first block
                p.plan.items[i0 + i] = RowItem{g, max(0, border), min(n, border + share), i, r0, rows, splits, splits > 1 ? s0 : -1};
            }
            first_items(p.plan.first, at, n, share, cut, i0, splits);
        }
    }
    for (int32_t i = lanes + tid; i <= sh.lanes; i += PT) p.plan.first[i] = items;
}

// ---- attention --------------------------------------------------------------------------------------
constexpr int AT = 128;                // threads of an attention block

template <int DP>
struct AttendSmem {
    static constexpr int ROW = DP * 2;                             // bytes of a token's vector
    static constexpr int TILE_BYTES = TILE * ROW;                  // keys or values of a tile
    static constexpr int Q_BYTES = 16 * ROW;
    static constexpr int BYTES = STAGES * 2 * TILE_BYTES + Q_BYTES + 256;
};

// The second product takes the probabilities in the inputs' type.  EIGHT: up to 8 query vectors, which leaves rows 8-15 of its
// tile free.  They take what the rounding left out, and V is multiplied with the probabilities to 2^-17 (bf16; f16 2^-22) at no
// cost: a thread's second row holds the remainders of its first.  They have sums of their own until the end, where a sum that is not
// finite is dropped: the remainder of a probability can be 0, and 0 times an infinite value is none of the result.  With 9 to 16
// vectors the probabilities are rounded once; a second product there cost 7 % (64 ragged rows: 182 us against 170).
template <typename T, int DP, bool EIGHT>
__global__ void __launch_bounds__(AT, 2) attend_cached_kernel(const AttendParams p) {
    let_later_in();
    wait_for_earlier();
    using S = AttendSmem<DP>;
    constexpr int CH = DP / 8;                                     // chunks of a row
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char* q_smem = smem + STAGES * 2 * S::TILE_BYTES;
    volatile int32_t* meta = reinterpret_cast<volatile int32_t*>(q_smem + S::Q_BYTES);      // [STAGES][TILE_BLKS]
    __shared__ float w_m[4][16], w_l[4][16];
    __shared__ int s_last;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const PlanShape& sh = p.shape;
    const int G = sh.G;
    // this block's lane and key head
    const int lane_of = blockIdx.x / p.kv_heads, head = blockIdx.x % p.kv_heads;
    const int item_end = p.plan.first[lane_of + 1];
    const int row_lo = lane >> 2;                                  // this thread's two rows of the tile: row_lo, row_lo + 8
    const int own_lo = row_lo / G + 1, own_hi = (row_lo + 8) / G + 1;

    for (int n = p.plan.first[lane_of]; n < item_end; ++n) {
        const int4 item = *reinterpret_cast<const int4*>(p.plan.items + n), more = *(reinterpret_cast<const int4*>(p.plan.items + n) + 1);
        const int g = item.x, r0 = more.x, n_rows = more.y, splits = more.z;
        const int M = n_rows * G;
        const int2* list = p.plan.list + int64_t(g) * sh.list_ld;
        const int32_t* table = p.table + int64_t(r0) * p.width;
        const int32_t len = p.len[r0];
        const int n_tiles = (item.z - item.y + TILE_BLKS - 1) / TILE_BLKS;
        const int64_t head_bytes = int64_t(p.page_size) * p.D * 2;

        __syncthreads();                                           // the unit before is done with the shared memory
        // a warp brings in block `warp` of a tile; which one that is has been read a tile earlier
        auto entry = [&](int t) {
            const int i = item.y + t * TILE_BLKS + warp;
            if (i >= item.z) return make_int2(0, 0);
            if (sh.per_group > 1) return list[i];
            return make_int2(table[i / sh.blks_per_page], i % sh.blks_per_page | max(0, min(BLK, len - i * BLK)) << 8);
        };
        auto load_tile = [&](int t, int2 e) {
            const int stage = t % STAGES;
            // a plan older than the books: rows may have let go of their pages since, and -1 is no place to read from
            if (unsigned(e.x) >= unsigned(p.pages)) e = make_int2(0, 0);
            const int tokens = (e.y >> 8) & 255;
            const int64_t off = (int64_t(e.x) * p.kv_heads + head) * head_bytes + int64_t(e.y & 255) * (BLK * 2) * p.D;
            const uint32_t kd = smem_u32(smem + stage * 2 * S::TILE_BYTES), vd = kd + S::TILE_BYTES;
#pragma unroll
            for (int j = 0; j < BLK * CH / 32; ++j) {
                const int c = j * 32 + lane, row = c / CH, ch = c % CH;
                const bool some = row < tokens && ch * 8 < p.D;
                const int64_t src = some ? off + int64_t(row) * p.D * 2 + ch * 16 : 0;
                const uint32_t dst = chunk_at<DP>(warp * BLK + row, ch);
                cp16(kd + dst, p.k + src, some);
                cp16(vd + dst, p.v + src, some);
            }
            if (lane == 0) meta[stage * TILE_BLKS + warp] = e.y >> 8;
        };
        int2 first[STAGES];
#pragma unroll
        for (int t = 0; t < STAGES; ++t) first[t] = entry(t);
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t) {
            if (t < n_tiles) load_tile(t, first[t]);
            cp_commit();
        }
        int2 next = first[STAGES - 1];
        // query vectors: row m of the tile is row m / G, head m % G of the group's heads
        for (int i = tid; i < 16 * CH; i += AT) {
            const int m = i / CH, ch = i % CH;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (m < M && ch * 8 < p.D)
                x = *reinterpret_cast<const uint4*>(p.q + (r0 + m / G) * p.q_row + (head * G + m % G) * p.q_head + ch * 16);
            *reinterpret_cast<uint4*>(q_smem + chunk_at<DP>(m, ch)) = x;
        }
        __syncthreads();
        uint32_t qf[DP / 16][4];
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk)
            ldsm4(smem_u32(q_smem) + chunk_at<DP>(lane & 15, 2 * kk + (lane >> 4)), qf[kk]);

        float o[DP / 8][4];
#pragma unroll
        for (int j = 0; j < DP / 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
        float m0 = -CUDART_INF_F, m1 = -CUDART_INF_F, l0 = 0.f, l1 = 0.f;

        for (int t = 0; t < n_tiles; ++t) {
            cp_wait<STAGES - 2>();
            __syncwarp();                                          // a warp works on what it has brought in itself
            if (t + STAGES - 1 < n_tiles) load_tile(t + STAGES - 1, next);
            cp_commit();
            next = entry(t + STAGES);
            const int stage = t % STAGES;
            const uint32_t kt = smem_u32(smem + stage * 2 * S::TILE_BYTES), vt = kt + S::TILE_BYTES;
            float s[2][4];
            const int mt = meta[stage * TILE_BLKS + warp], owner = mt >> 8, tokens = mt & 255;
            float mx0 = -CUDART_INF_F, mx1 = -CUDART_INF_F;
            s[0][0] = s[0][1] = s[0][2] = s[0][3] = s[1][0] = s[1][1] = s[1][2] = s[1][3] = 0.f;
            if (tokens) {
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk) {
                    uint32_t kf[4];
                    // matrices: tokens 0-7 and 8-15 of the block, each k 0-7 and 8-15
                    ldsm4(kt + chunk_at<DP>(warp * BLK + (lane & 7) + ((lane >> 4) << 3), 2 * kk + ((lane >> 3) & 1)), kf);
                    mma16<T>(s[0], qf[kk], kf[0], kf[1]);
                    mma16<T>(s[1], qf[kk], kf[2], kf[3]);
                }
            }
            const bool in0 = !owner || owner == own_lo, in1 = !owner || owner == own_hi;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const bool some = h * 8 + (lane & 3) * 2 + e < tokens;
                    s[h][e] = some && in0 ? s[h][e] * p.c2 : -CUDART_INF_F;
                    s[h][2 + e] = !EIGHT && some && in1 ? s[h][2 + e] * p.c2 : -CUDART_INF_F;
                    mx0 = fmaxf(mx0, s[h][e]);
                    if (!EIGHT) mx1 = fmaxf(mx1, s[h][2 + e]);
                }
            mx0 = fmaxf(mx0, __shfl_xor_sync(FULL, mx0, 1));
            if (!EIGHT) mx1 = fmaxf(mx1, __shfl_xor_sync(FULL, mx1, 1));
            mx0 = fmaxf(mx0, __shfl_xor_sync(FULL, mx0, 2));
            if (!EIGHT) mx1 = fmaxf(mx1, __shfl_xor_sync(FULL, mx1, 2));
            if (__any_sync(FULL, mx0 > m0 || (!EIGHT && mx1 > m1))) {
                const float n0 = fmaxf(m0, mx0), n1 = fmaxf(m1, mx1);
                const float f0 = m0 > -CUDART_INF_F ? ex2_approx(m0 - n0) : 0.f, f1 = EIGHT ? f0 : m1 > -CUDART_INF_F ? ex2_approx(m1 - n1) : 0.f;
                m0 = n0;
                m1 = n1;
                l0 *= f0;
                l1 *= f1;
#pragma unroll
                for (int j = 0; j < DP / 8; ++j) { o[j][0] *= f0; o[j][1] *= f0; o[j][2] *= f1; o[j][3] *= f1; }
            }
            const float ref0 = m0 > -CUDART_INF_F ? m0 : 0.f, ref1 = m1 > -CUDART_INF_F ? m1 : 0.f;
            if (!tokens) continue;
            uint32_t pf[4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float* x = s[h];
                x[0] = ex2_approx(x[0] - ref0);
                x[1] = ex2_approx(x[1] - ref0);
                l0 += x[0] + x[1];
                pf[2 * h] = pack2<T>(x[0], x[1]);
                if (EIGHT) {
                    const float2 r = unpack2<T>(pf[2 * h]);
                    x[2] = x[0] - r.x;
                    x[3] = x[1] - r.y;
                } else {
                    x[2] = ex2_approx(x[2] - ref1);
                    x[3] = ex2_approx(x[3] - ref1);
                    l1 += x[2] + x[3];
                }
                pf[2 * h + 1] = pack2<T>(x[2], x[3]);
            }
#pragma unroll
            for (int j = 0; j < DP / 16; ++j) {
                uint32_t vf[4];
                // matrices: tokens 0-7, 8-15 of the block at values 16j..16j+7, then at 16j+8..16j+15
                ldsm4t(vt + chunk_at<DP>(warp * BLK + (lane & 15), 2 * j + (lane >> 4)), vf);
                if (!owner) {
                    mma16<T>(o[2 * j], pf, vf[0], vf[1]);
                    mma16<T>(o[2 * j + 1], pf, vf[2], vf[3]);
                } else {
                    // a row's own tokens: what they add to other rows is 0 * v, which is not 0 for a
                    // non-finite v, so it is left out
                    float t0[4] = {0.f, 0.f, 0.f, 0.f}, t1[4] = {0.f, 0.f, 0.f, 0.f};
                    mma16<T>(t0, pf, vf[0], vf[1]);
                    mma16<T>(t1, pf, vf[2], vf[3]);
                    if (in0) { o[2 * j][0] += t0[0]; o[2 * j][1] += t0[1]; o[2 * j + 1][0] += t1[0]; o[2 * j + 1][1] += t1[1]; }
                    if (EIGHT ? in0 : in1) { o[2 * j][2] += t0[2]; o[2 * j][3] += t0[3]; o[2 * j + 1][2] += t1[2]; o[2 * j + 1][3] += t1[3]; }
                }
            }
        }
        l0 += __shfl_xor_sync(FULL, l0, 1);
        l1 += __shfl_xor_sync(FULL, l1, 1);
        l0 += __shfl_xor_sync(FULL, l0, 2);
        l1 += __shfl_xor_sync(FULL, l1, 2);

        cp_wait<0>();
        __syncthreads();                                           // every warp is done with the tiles
        // sums to shared memory, [warps x 16][DP] fp32
        float* os = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int j = 0; j < DP / 8; ++j) {
            float* a = os + (warp * 16 + (lane >> 2)) * DP + j * 8 + (lane & 3) * 2;
            if (EIGHT) {
                const float r0 = fabsf(o[j][2]) < CUDART_INF_F ? o[j][2] : 0.f, r1 = fabsf(o[j][3]) < CUDART_INF_F ? o[j][3] : 0.f;
                *reinterpret_cast<float2*>(a) = make_float2(o[j][0] + r0, o[j][1] + r1);
                continue;
            }
            *reinterpret_cast<float2*>(a) = make_float2(o[j][0], o[j][1]);
            *reinterpret_cast<float2*>(a + 8 * DP) = make_float2(o[j][2], o[j][3]);
        }
        if ((lane & 3) == 0) {
            w_m[warp][lane >> 2] = m0; w_m[warp][(lane >> 2) + 8] = m1;
            w_l[warp][lane >> 2] = l0; w_l[warp][(lane >> 2) + 8] = l1;
        }
        __syncthreads();

        const int64_t slot = splits > 1 ? (int64_t(more.w + item.w) * p.kv_heads + head) * sh.M : 0;
        constexpr int DV = DP / 4;
        for (int i = tid; i < M * DV; i += AT) {
            const int m = i / DV, d = (i % DV) * 4;
            if (d >= p.D) continue;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            const float mm = fmaxf(fmaxf(w_m[0][m], w_m[1][m]), fmaxf(w_m[2][m], w_m[3][m]));
            float ll = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = w_m[w][m] > -CUDART_INF_F ? ex2_approx(w_m[w][m] - mm) : 0.f;
                const float4 y = *reinterpret_cast<const float4*>(os + (w * 16 + m) * DP + d);
                x.x += f * y.x; x.y += f * y.y; x.z += f * y.z; x.w += f * y.w;
                ll += f * w_l[w][m];
            }
            const float inv = ll > 0.f ? 1.f / ll : (ll == 0.f ? 0.f : ll);
            x.x *= inv; x.y *= inv; x.z *= inv; x.w *= inv;
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
                *reinterpret_cast<uint2*>(p.out + (at * p.D + d) * 2) = make_uint2(pack2<T>(x.x, x.y), pack2<T>(x.z, x.w));
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

int shift_of(int32_t page_size) {
    int s = 0;
    while ((1 << s) < page_size) ++s;
    return s;
}

template <typename T, int DP, bool EIGHT>
int launch_attend(const AttendParams& p, unsigned grid, cudaStream_t st) {
    constexpr int bytes = AttendSmem<DP>::BYTES;
    static std::atomic<uint64_t> done{0};
    if (const int rc = allow_smem(attend_cached_kernel<T, DP, EIGHT>, bytes, done)) return rc;
    return launch_after(attend_cached_kernel<T, DP, EIGHT>, grid, AT, bytes, st, p);
}
template <typename T>
int launch_attend(const AttendParams& p, unsigned grid, cudaStream_t st) {
    if (p.shape.M <= 8) return p.D <= 64 ? launch_attend<T, 64, true>(p, grid, st) : launch_attend<T, 128, true>(p, grid, st);
    return p.D <= 64 ? launch_attend<T, 64, false>(p, grid, st) : launch_attend<T, 128, false>(p, grid, st);
}

}  // namespace

extern "C" {

int64_t disc_attend_plan_bytes(const disc_cache_t* c, int32_t n_q_heads, int32_t group) {
    PlanShape s;
    if (!c) return DISC_ERR_ARG;
    if (const int rc = disc::cache_sizes(c)) return rc;
    if (const int rc = plan_shape(c, n_q_heads, group, &s)) return rc;
    return plan_layout(c, s, nullptr, nullptr);
}

int disc_attend_plan(const disc_cache_t* c, int32_t n_q_heads, int32_t group, void* plan, int64_t plan_bytes, void* stream) {
    if (!c || !c->table || !c->len || !plan) return DISC_ERR_ARG;
    if (const int rc = disc::cache_sizes(c)) return rc;
    PlanParams p;
    if (const int rc = plan_shape(c, n_q_heads, group, &p.shape)) return rc;
    if ((reinterpret_cast<uintptr_t>(plan) & 31u) || plan_bytes < plan_layout(c, p.shape, plan, &p.plan)) return DISC_ERR_ARG;
    p.table = c->table; p.len = c->len; p.rows = c->n_rows; p.width = c->table_width;
    p.page_size = c->page_size; p.shift = shift_of(c->page_size); p.kv_heads = c->n_kv_heads;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p.shape.M > ROWS_M) return disc::plan_groups(p, st);
    // few groups: one block does without the cluster's barrier
    const bool one = p.shape.groups <= PT / 32;
    return launch_after(one ? attend_plan_kernel<1> : attend_plan_kernel<CLUSTER>, one ? 1 : CLUSTER, PT, 0, st, p);
}

int disc_attend_cached(const disc_cache_t* c, int32_t layer, const void* q, int64_t q_row_stride, int64_t q_head_stride,
                       int32_t n_q_heads, int32_t group, float scale, void* plan, int64_t plan_bytes, void* out, float* lse_out,
                       void* stream) {
    if (!c || !c->pool || !c->table || !c->len || !q || !plan || !out) return DISC_ERR_ARG;
    if (const int rc = disc::cache_sizes(c)) return rc;
    if (layer < 0 || layer >= c->n_layers || !(scale > 0.f) || !(scale <= 3.0e38f)) return DISC_ERR_ARG;
    AttendParams p;
    if (const int rc = plan_shape(c, n_q_heads, group, &p.shape)) return rc;
    if ((reinterpret_cast<uintptr_t>(plan) & 31u) || plan_bytes < plan_layout(c, p.shape, plan, &p.plan)) return DISC_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15u) return DISC_ERR_ARG;
    // the stride over an axis of one is never used; any valid one will do
    if (n_q_heads == 1) q_head_stride = (int64_t(c->head_dim) + 7) / 8 * 8;
    if (c->n_rows == 1) q_row_stride = (int64_t(c->head_dim) + 7) / 8 * 8 * n_q_heads;
    if ((q_row_stride | q_head_stride) & 7) return DISC_ERR_UNSUPPORTED;
    const int64_t plane = disc::cache_plane_bytes(c);
    p.k = static_cast<const unsigned char*>(c->pool) + 2 * layer * plane;
    p.v = p.k + plane;
    p.q = static_cast<const unsigned char*>(q); p.q_row = q_row_stride * 2; p.q_head = q_head_stride * 2;
    p.table = c->table; p.len = c->len; p.width = c->table_width; p.pages = c->n_pages;
    p.out = static_cast<unsigned char*>(out); p.lse = lse_out;
    p.rows = c->n_rows; p.kv_heads = c->n_kv_heads; p.D = c->head_dim; p.page_size = c->page_size;
    p.head_bytes = disc::cache_head_bytes(c);
    p.c2 = scale * LOG2E_F;
    p.error = reinterpret_cast<uint32_t*>(p.plan.head);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p.shape.M > ROWS_M) return disc::attend_groups(p, c->dtype, n_q_heads, st);
    if (disc::cache_held(c)) return disc::attend_held(p, c->dtype, st);
    const unsigned grid = unsigned(p.shape.lanes * c->n_kv_heads);
    return c->dtype == DISC_BF16 ? launch_attend<__nv_bfloat16>(p, grid, st) : launch_attend<__half>(p, grid, st);
}

}  // extern "C"
