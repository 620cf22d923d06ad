// What the two forms of the attention over the cache share: the plan's sizes and places (disc_attend.cu, disc_attend_group.cu).
#pragma once

#include "disc_sm100.cuh"

namespace disc {

constexpr int BLK = 16;                // tokens of a block: the smallest page, and the depth of one MMA
constexpr int ROWS_M = 16;             // up to this many query vectors read the same pages: disc_attend.cu, above it disc_attend_group.cu
constexpr int GROUP_M = 128;           // query vectors that a group can have at most
constexpr int G_MAX = 64;              // query heads per key head
constexpr int START = 8;               // what beginning an item costs, in blocks
constexpr int PLACES = 148 * 2;        // blocks that run at a time: two to an SM
constexpr int HELD_BLOCKS = 3;         // rows form over a cache held in 8 bits, up to HELD_FEW query vectors: three
constexpr int HELD_FEW = 8;

struct PlanShape {
    int32_t G;                         // query heads per key head
    int32_t per_group;                 // rows of a group as it is worked on
    int32_t sub;                       // such groups per `group` rows
    int32_t groups;                    // in all
    int32_t M;                         // query vectors of a group
    int32_t group;                     // rows that may share pages, as given
    int32_t blks_per_page;
    int32_t lanes;                     // equal shares that the work of each key head is cut into
    int32_t max_items;
    int64_t list_ld;                   // rows form: blocks a group's list has room for
    int64_t max_part;                  // partial results: query vectors there is room for
};

struct GroupItem {                     // rows [row, row + rows) over the blocks [begin, end) of row `lead`
    int32_t row, rows, begin, end, part, lead, pad[2];
};

struct RowItem {                       // rows [row, row + rows) of group g over the blocks [begin, end) of its list
    int32_t g, begin, end, index;      // index among the group's items
    int32_t row, rows, items, slot;    // the group's items; its first partial result, or -1
};

struct Plan {
    int32_t* head;                     // [0] error word: the caller's to clear, no kernel does
    int32_t* first;                    // [lanes + 1] first item of a lane; lanes without work begin where all items end
    float* part;                       // [max_part][head_dim] normalised sums, fp32
    float* part_lse;                   // [max_part] log-sum-exp in units of log2
    // rows form
    int32_t* count;                    // [groups] blocks
    int32_t* arrived;                  // [groups][kv heads]
    RowItem* items;
    int2* list;                        // [groups][list_ld]: page; block | tokens << 8 | (owner + 1) << 16
    // group form
    GroupItem* group_items;
    int32_t* shared;                   // [groups] leading blocks that its rows share and that are worked on together
    int32_t* lead;                     // [groups] the first row with tokens, whose pages these are
    int32_t* alone;                    // [rows] blocks after those that are worked on as an item of the row's own
    int2* group_part;                  // [groups] first partial result, number of parts
    int2* row_part;                    // [rows]
};

inline int plan_shape(const disc_cache_t* c, int32_t hq, int32_t group, PlanShape* s) {
    if (hq <= 0 || group <= 0 || c->n_kv_heads <= 0 || hq % c->n_kv_heads) return DISC_ERR_ARG;
    s->G = hq / c->n_kv_heads;
    if (s->G > G_MAX) return DISC_ERR_UNSUPPORTED;
    s->group = group = group < c->n_rows ? group : c->n_rows;
    const int64_t vectors = int64_t(group) * s->G;
    s->per_group = vectors <= GROUP_M ? group : GROUP_M / s->G;
    s->sub = (group + s->per_group - 1) / s->per_group;
    const int64_t groups = (int64_t(c->n_rows) + group - 1) / group * s->sub;
    if (groups > (1 << 26)) return DISC_ERR_UNSUPPORTED;
    s->groups = int32_t(groups);
    s->M = s->per_group * s->G;
    s->blks_per_page = c->page_size / BLK;
    // blocks are counted in 32 bits
    if (int64_t(c->n_rows) * (int64_t(c->table_width) * s->blks_per_page + START) >= (int64_t(1) << 30)) return DISC_ERR_UNSUPPORTED;
    const int32_t places = cache_held(c) && s->M <= HELD_FEW ? PLACES / 2 * HELD_BLOCKS : PLACES;
    s->lanes = places / c->n_kv_heads > 1 ? places / c->n_kv_heads : 1;
    // every border between two lanes makes one item two
    if (s->M <= ROWS_M) {
        // a row alone: its blocks are found through the table
        s->list_ld = s->per_group == 1 ? 0 : int64_t(s->per_group) * c->table_width * s->blks_per_page;
        s->max_items = s->groups + s->lanes;
        s->max_part = int64_t(2 * s->lanes) * c->n_kv_heads * s->M;
    } else {
        // the K and V planes as tensor maps: rows of a plane are counted in 32 bits
        if (int64_t(c->n_pages) * c->n_kv_heads * c->page_size >= (int64_t(1) << 31)) return DISC_ERR_UNSUPPORTED;
        s->list_ld = 0;
        s->max_items = s->groups + c->n_rows + s->lanes;
        s->max_part = (int64_t(s->groups) * s->M + int64_t(c->n_rows) * s->G + int64_t(s->lanes) * s->M) * c->n_kv_heads;
        if (s->max_part >= (int64_t(1) << 31)) return DISC_ERR_UNSUPPORTED;
    }
    return DISC_OK;
}

inline int64_t plan_layout(const disc_cache_t* c, const PlanShape& s, void* base_, Plan* p) {
    unsigned char* base = static_cast<unsigned char*>(base_);
    int64_t at = 0;
    auto take = [&](int64_t bytes) { unsigned char* q = base + at; at += (bytes + 31) & ~int64_t(31); return q; };
    Plan t = {};
    t.head = reinterpret_cast<int32_t*>(take(256));
    t.first = reinterpret_cast<int32_t*>(take((int64_t(s.lanes) + 1) * 4));
    t.part = reinterpret_cast<float*>(take(s.max_part * c->head_dim * 4));
    t.part_lse = reinterpret_cast<float*>(take(s.max_part * 4));
    if (s.M <= ROWS_M) {
        t.count = reinterpret_cast<int32_t*>(take(int64_t(s.groups) * 4));
        t.arrived = reinterpret_cast<int32_t*>(take(int64_t(s.groups) * c->n_kv_heads * 4));
        t.items = reinterpret_cast<RowItem*>(take(int64_t(s.max_items) * sizeof(RowItem)));
        t.list = reinterpret_cast<int2*>(take(int64_t(s.groups) * s.list_ld * 8));
    } else {
        t.group_items = reinterpret_cast<GroupItem*>(take(int64_t(s.max_items) * sizeof(GroupItem)));
        t.shared = reinterpret_cast<int32_t*>(take(int64_t(s.groups) * 4));
        t.lead = reinterpret_cast<int32_t*>(take(int64_t(s.groups) * 4));
        t.alone = reinterpret_cast<int32_t*>(take(int64_t(c->n_rows) * 4));
        t.group_part = reinterpret_cast<int2*>(take(int64_t(s.groups) * 8));
        t.row_part = reinterpret_cast<int2*>(take(int64_t(c->n_rows) * 8));
    }
    if (p) *p = t;
    return at;
}

// How the work of a key head is cut, the same way for every key head: all blocks in a row, group after group, in equal
// shares ("lanes") for the blocks of threads that run at a time.  An item is what a lane has of one group.  (Items of equal
// length dealt out in turn left the device waiting for the last ones: 196 us against 185 with 1.5 times as many, 213 with four
// times, 159 with shares, on 64 rows of 1 to 8191 tokens and 8 key heads.)  Behind its blocks a group takes up START more,
// for what beginning an item costs, so that a lane of many short rows is not the last.
struct Cut {
    int32_t from, splits;              // lane of the first item; items
};
__host__ __device__ inline Cut cut_group(int32_t at, int32_t blocks, int32_t share) {
    const int32_t from = at / share;
    return {from, blocks > 0 ? (at + blocks - 1) / share - from + 1 : 0};
}
// The lanes that begin within a group's place [at, at + blocks + START): their first items.  One thread.
__device__ inline void first_items(int32_t* first, int32_t at, int32_t blocks, int32_t share, const Cut& cut, int32_t item0, int32_t items) {
    for (int32_t lane = (at + share - 1) / share; lane * share < at + blocks + START; ++lane)
        first[lane] = item0 + (lane * share < at + blocks ? lane - cut.from : lane * share == at ? 0 : items);
}

// ---- loads and products by mma.sync -------------------------------------------------------------------
// 16 bytes into shared memory; zeros when !some
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool some) {
    const int n = some ? 16 : 0;
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// an 8 x 8 matrix of 16-bit values across the warp, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// d += a b, 16 x 16 by 16 x 8
template <typename T>
__device__ __forceinline__ void mma16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<__nv_bfloat16>(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<__half>(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16-byte chunk `ch` of row `row` of a tile whose rows are DP values long: neighbouring rows' chunks lie in
// different banks, so that ldmatrix reads eight rows at once without conflicts
template <int DP>
__device__ __forceinline__ uint32_t chunk_at(int row, int ch) {
    return uint32_t(row * (DP * 2) + ((ch ^ (row & 7)) << 4));
}

struct PlanParams {
    Plan plan;
    PlanShape shape;
    const int32_t* table;
    const int32_t* len;
    int32_t rows, width, page_size, shift, kv_heads;
};

struct AttendParams {
    Plan plan;
    PlanShape shape;
    const unsigned char* k;            // this layer's planes
    const unsigned char* v;
    const unsigned char* q;
    int64_t q_row, q_head;             // bytes
    const int32_t* table;
    const int32_t* len;
    unsigned char* out;
    float* lse;
    int32_t rows, width, pages, kv_heads, D, page_size;
    int32_t head_bytes;                // of a page and key head
    float c2;                          // scale log2(e)
    uint32_t* error;
};

constexpr float LN2_F = 0.6931471805599453f;

// Two outputs.  In f16 a value held in 8 bits can exceed the type's largest one by the rounding of its code; reading it gives the largest, and so
// does a mean of such values, which would else be infinite.  Infinities themselves, which 16 bits can hold, stay.
template <typename T>
__device__ __forceinline__ uint32_t pack_out(float a, float b) { return pack2<T>(a, b); }
template <>
__device__ __forceinline__ uint32_t pack_out<__half>(float a, float b) {
    auto within = [](float x) { return fabsf(x) < CUDART_INF_F ? fminf(fmaxf(x, -65504.f), 65504.f) : x; };
    return pack2<__half>(within(a), within(b));
}

// The items of a group, joined in their order by the block of threads that finished last: one pass, eight parts on their way at
// a time.  slot: the group's first part; M query vectors of the rows from r0 on, DP >= D values.
template <typename T, int DP, int THREADS>
__device__ __forceinline__ void join_items(const AttendParams& p, int32_t slot, int splits, int head, int M, int r0) {
    const PlanShape& sh = p.shape;
    const int G = sh.G;
    constexpr int DV = DP / 4;
    const int64_t slot0 = (int64_t(slot) * p.kv_heads + head) * sh.M, step = int64_t(p.kv_heads) * sh.M;
    for (int i = threadIdx.x; i < M * DV; i += THREADS) {
        const int m = i / DV, d = (i % DV) * 4;
        if (d >= p.D) continue;
        float top = -CUDART_INF_F, total = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int j0 = 0; j0 < splits; j0 += 8) {
            float lse[8];
            float4 y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j0 + j < splits) {
                    const int64_t part = slot0 + (j0 + j) * step + m;
                    lse[j] = __ldcg(p.plan.part_lse + part);
                    y[j] = __ldcg(reinterpret_cast<const float4*>(p.plan.part + part * p.D + d));
                }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j0 + j < splits) {
                    const float n = fmaxf(top, lse[j]);
                    const float f = top > -CUDART_INF_F ? ex2_approx(top - n) : 0.f, w = lse[j] == -CUDART_INF_F ? 0.f : ex2_approx(lse[j] - n);
                    top = n;
                    total = fmaf(total, f, w);
                    x = make_float4(fmaf(w, y[j].x, x.x * f), fmaf(w, y[j].y, x.y * f), fmaf(w, y[j].z, x.z * f), fmaf(w, y[j].w, x.w * f));
                }
        }
        const float inv = total > 0.f ? 1.f / total : (total == 0.f ? 0.f : total);
        const int64_t at = int64_t(r0 + m / G) * p.kv_heads * G + head * G + m % G;
        *reinterpret_cast<uint2*>(p.out + (at * p.D + d) * 2) = make_uint2(pack_out<T>(x.x * inv, x.y * inv), pack_out<T>(x.z * inv, x.w * inv));
        if (d == 0 && p.lse) p.lse[at] = total > 0.f ? (top + log2f(total)) * LN2_F : (total == 0.f ? -CUDART_INF_F : total);
    }
}

// disc_attend_group.cu: more than ROWS_M query vectors read the same pages; dtype as in disc_cache_t
int plan_groups(const PlanParams& p, cudaStream_t st);
int attend_groups(const AttendParams& p, int32_t dtype, int32_t n_q_heads, cudaStream_t st);
// disc_attend_held.cu: up to ROWS_M, over a cache held in 8 bits
int attend_held(const AttendParams& p, int32_t dtype, cudaStream_t st);

}  // namespace disc
