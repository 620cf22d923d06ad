// The pages of the key-value cache: rows that share, copy, release and move pages.
//
//   disc_cache_fork     row r becomes what row parent[r] was, sharing its pages
//   disc_cache_free     rows let go of their pages
//   disc_cache_extend   room for new tokens: free pages, and private copies of shared last pages
//   disc_cache_write    keys and values of new tokens into the pages
//   disc_cache_compact  the live pages move to the front of the pool
//
// The books are whole numbers on the device (page table, lengths, reference counts) and nothing is
// read by the host, so that a decode can be enqueued, or captured as a graph, without a wait.  A page is
// free when its reference count is 0; new pages are the free ones of lowest id, rows served in ascending
// order.  The counts are changed by atomic additions (their sum does not depend on the order) and
// everything that depends on an order goes by prefix sums, so the same calls give the same table every time.
//
// What these calls cost is latency, a few dependent reads of small arrays (4096 rows: fork 7 us, extend 13), except for
// the copies of page contents, which are bound by the bytes: 48 us for the 0.26 GB of 4096 candidates' last pages
// (5.3 TB/s), 102 us for a compaction's 0.58 GB (5.7 TB/s; the measured copy rate is 6.5).

#include "disc_internal.cuh"

namespace {

using namespace disc;

constexpr unsigned FULL = 0xffffffffu;

// scratch: counters, the table on its way, marks per page, lists
struct Scratch {
    int32_t* head;        // [0] copies to make, [1] live pages, [2] pages to move
    int32_t* len;         // [rows]
    int32_t* table;       // [rows][width]
    int32_t* sharers;     // [pages]
    unsigned long long* keeper;   // [pages]
    int32_t* list;        // [pages] free pages in order / [pages] where a page goes
    int4* copy;           // [rows] source page, copy, tokens
    int2* move;           // [pages] from, to
};
constexpr int HEAD_BYTES = 256;

inline int64_t up16(int64_t b) { return (b + 15) & ~int64_t(15); }
inline int64_t scratch_layout(const disc_cache_t* c, Scratch* s) {
    unsigned char* base = static_cast<unsigned char*>(c->scratch);
    int64_t at = 0;
    auto take = [&](int64_t bytes) { unsigned char* p = base + at; at += up16(bytes); return p; };
    const int64_t rows = c->n_rows, pages = c->n_pages;
    Scratch t;
    t.head = reinterpret_cast<int32_t*>(take(HEAD_BYTES));
    t.copy = reinterpret_cast<int4*>(take(rows * 16));
    t.move = reinterpret_cast<int2*>(take(pages * 8));
    t.len = reinterpret_cast<int32_t*>(take(rows * 4));
    t.table = reinterpret_cast<int32_t*>(take(rows * c->table_width * 4));
    t.sharers = reinterpret_cast<int32_t*>(take(pages * 4));
    t.keeper = reinterpret_cast<unsigned long long*>(take(pages * 8));
    t.list = reinterpret_cast<int32_t*>(take(pages * 4));
    if (s) *s = t;
    return at;
}

struct Books {
    int32_t* table;
    int32_t* len;
    int32_t* ref;
    int32_t rows, width, pages, page_size;
    int32_t shift;                     // log2 of the page size
};

// ---- fork / free ------------------------------------------------------------------------------------
// One warp per row, two steps.  The first notes every changing row's new pages and moves the reference counts;
// the second writes the table.  All rows take the first before any takes the second, because a row that changes may be another
// row's parent: two launches, or, for up to 32 rows, one block with a barrier.
__device__ __forceinline__ int32_t parent_of(int32_t row, const int32_t* parent, const uint8_t* freed) {
    return parent ? parent[row] : (freed[row] ? -1 : row);
}
__device__ __forceinline__ void take_row(const Books& b, const Scratch& s, int32_t row, int32_t p, int lane) {
    const bool some = p >= 0 && p < b.rows;
    const int32_t len = some ? b.len[p] : 0;
    const int32_t used = (len + b.page_size - 1) >> b.shift, old = (b.len[row] + b.page_size - 1) >> b.shift;
    const int32_t* from = b.table + size_t(some ? p : 0) * b.width;
    const int32_t* was = b.table + size_t(row) * b.width;
    int32_t* to = s.table + size_t(row) * b.width;
    for (int32_t j = lane; j < max(used, old); j += 32) {
        if (j < used) {
            const int32_t page = from[j];
            to[j] = page;
            atomicAdd(b.ref + page, 1);
        }
        if (j < old) atomicAdd(b.ref + was[j], -1);
    }
    if (lane == 0) s.len[row] = len;
}
__device__ __forceinline__ void settle_row(const Books& b, const Scratch& s, int32_t row, int lane) {
    const int32_t len = s.len[row];
    const int32_t used = (len + b.page_size - 1) >> b.shift, old = (b.len[row] + b.page_size - 1) >> b.shift;
    const int32_t* from = s.table + size_t(row) * b.width;
    int32_t* to = b.table + size_t(row) * b.width;
    for (int32_t j = lane; j < max(used, old); j += 32) to[j] = j < used ? from[j] : -1;
    __syncwarp();
    if (lane == 0) b.len[row] = len;
}
// step 0: the first, 1: the second, 2: both, in one block
template <int STEP>
__global__ void __launch_bounds__(STEP == 2 ? 1024 : 256) cache_fork_kernel(Books b, const int32_t* parent,
                                                                           const uint8_t* freed, Scratch s) {
    let_later_in();
    wait_for_earlier();
    const int32_t row = int32_t((blockIdx.x * blockDim.x + threadIdx.x) >> 5);
    const int lane = threadIdx.x & 31;
    const int32_t p = row < b.rows ? parent_of(row, parent, freed) : row;
    if (STEP != 1 && p != row) take_row(b, s, row, p, lane);
    if (STEP == 2) __syncthreads();
    if (STEP != 0 && p != row) settle_row(b, s, row, lane);
}

// ---- extend ------------------------------------------------------------------------------------------
// The calls that decide by order, extend and compact, run as one cluster of 8 blocks: their steps hang on one another, and a
// cluster's barrier costs less than a launch.  One block alone takes 38 us to extend 4096 rows over 27,000 pages, the
// cluster 13, most of it waiting for one load after the other; but 16 rows over some hundred pages take 10 us in the
// cluster and 6 in one block, which is what small caches get.
constexpr int XT = 1024;
constexpr int CLUSTER = 8;
constexpr int ONE_BLOCK = 8192;        // up to this many pages (and XT rows): one block

__device__ __forceinline__ int32_t remote_int(const int32_t* p, uint32_t rank) {
    uint32_t a;
    int32_t v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(uint32_t(__cvta_generic_to_shared(p))), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// the barrier of CL blocks
template <int CL>
__device__ __forceinline__ void sync_blocks() {
    if (CL == 1) __syncthreads(); else cluster_sync_all();
}

// exclusive sum over the block of v; *total gets the whole sum.  Called by the whole block.
__device__ __forceinline__ int32_t block_scan(int32_t v, int32_t* warp_sums, int32_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t u = __shfl_up_sync(FULL, incl, o);
        if (lane >= o) incl += u;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    int32_t w = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t u = __shfl_up_sync(FULL, w, o);
        if (lane >= o) w += u;
    }
    *total = __shfl_sync(FULL, w, 31);
    const int32_t before = __shfl_sync(FULL, w, max(warp - 1, 0));
    return incl - v + (warp ? before : 0);
}

// The blocks' own numbers, one each, exchanged: the sum over the blocks before this one, and over all.  `mine` is shared
// memory that stays as it is until the next barrier of the cluster.  Begins with a barrier of the cluster.
template <int CL>
__device__ __forceinline__ void cluster_sums(const int32_t* mine, uint32_t rank, int32_t* before, int32_t* all) {
    sync_blocks<CL>();
    int32_t b = 0, t = 0;
#pragma unroll
    for (uint32_t c = 0; c < CL; ++c) {
        const int32_t v = CL == 1 ? *mine : remote_int(mine, c);
        if (c < rank) b += v;
        t += v;
    }
    *before = b;
    *all = t;
}

// this block's share [a, b) of n things, in runs of 4
template <int CL>
__device__ __forceinline__ void share_of(int32_t n, uint32_t rank, int32_t* a, int32_t* b) {
    const int32_t per = ((n + CL - 1) / CL + 3) & ~3;
    *a = min(n, int32_t(rank) * per);
    *b = min(n, *a + per);
}
// four consecutive reference counts from p (a multiple of 4); 1 beyond the last
__device__ __forceinline__ int4 four_refs(const int32_t* ref, int32_t p, int32_t end) {
    if (p + 4 <= end && (reinterpret_cast<uintptr_t>(ref) & 15) == 0) return *reinterpret_cast<const int4*>(ref + p);
    return make_int4(p < end ? ref[p] : 1, p + 1 < end ? ref[p + 1] : 1, p + 2 < end ? ref[p + 2] : 1, p + 3 < end ? ref[p + 3] : 1);
}

struct Pool {
    unsigned char* base;
    int32_t planes, heads;
    int64_t plane_bytes;
    int32_t head_bytes, token_bytes;
};
// Copies of the tokens in partly filled pages: a warp per copy, plane and head, which is one run of tokens x head dim.
// This warp's units: first, first + step, ... below n.
__device__ __forceinline__ void copy_units(const Pool& o, const Scratch& s, int64_t first, int64_t step, int64_t n) {
    const int lane = threadIdx.x & 31;
    for (int64_t i = first; i < n; i += step) {
        const int32_t h = int32_t(i % o.heads);
        const int64_t j = i / o.heads;
        const int32_t pl = int32_t(j % o.planes);
        const int4 c = s.copy[j / o.planes];
        const uint4* from = reinterpret_cast<const uint4*>(o.base + pl * o.plane_bytes + (int64_t(c.x) * o.heads + h) * o.head_bytes);
        uint4* to = reinterpret_cast<uint4*>(o.base + pl * o.plane_bytes + (int64_t(c.y) * o.heads + h) * o.head_bytes);
        const int32_t vecs = c.z * o.token_bytes / 16;
        for (int32_t v0 = lane; v0 < vecs; v0 += 32 * 4) {         // four loads in flight
            uint4 x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (v0 + u * 32 < vecs) x[u] = from[v0 + u * 32];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (v0 + u * 32 < vecs) __stcs(to + v0 + u * 32, x[u]);
        }
    }
}
__global__ void __launch_bounds__(256) cache_copy_kernel(Pool o, Scratch s) {
    let_later_in();
    wait_for_earlier();
    copy_units(o, s, (int64_t(blockIdx.x) * blockDim.x + threadIdx.x) >> 5, int64_t(gridDim.x) * (blockDim.x >> 5),
               int64_t(s.head[0]) * o.planes * o.heads);
}

struct Need {
    int32_t add, len, first, last, page;                   // table positions [first, last) are new; page: the partial last one or -1
    bool too_long;                                         // the table has no room for the row's pages
};
__device__ __forceinline__ Need row_need(const Books& b, const int32_t* add, int32_t row) {
    Need n;
    n.add = add ? add[row] : 1;
    n.len = b.len[row];
    n.first = (n.len + b.page_size - 1) >> b.shift;
    n.page = -1;
    n.last = n.first;
    n.too_long = n.add > 0 && int64_t(n.len) + n.add > (int64_t(b.width) << b.shift);
    if (n.add > 0 && !n.too_long) {
        n.last = (n.len + n.add + b.page_size - 1) >> b.shift;
        if (n.len & (b.page_size - 1)) n.page = b.table[size_t(row) * b.width + n.first - 1];
    }
    return n;
}

// the longer row has the smaller key, of equally long ones the lower
__device__ __forceinline__ unsigned long long keeper_key(const Books& b, const Need& n, int32_t row) {
    return static_cast<unsigned long long>(b.page_size - (n.len & (b.page_size - 1))) << 32 | uint32_t(row);
}

//  1. Rows that go on writing into a partly filled page mark it: how many rows do (sharers), and the lowest of the longest of
//     them (keeper).  If they are all the rows that hold the page, the keeper writes on in place; the others, and
//     all of them where a row that stays behind holds the page too, get a copy.  The longest, because the rows of a page can differ in
//     length (one that found no page stays behind the others), and one that finds no page for its copy now keeps its tokens
//     only if nobody writes before its end.
//  2. Prefix sums over the rows of the pages they need; rows beyond the number of free pages get nothing.
//  3. The free pages of lowest id, in order, as many as are needed, and from them each row's share.
// A thread has ROWS consecutive rows, in registers from the first step to the last, or, where there are more of them, reads
// them again in every step.
template <int CL, int ROWS>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(XT) cache_extend_kernel(Books b, const int32_t* add, Scratch s,
                                                                                  uint8_t* status, Pool o, bool copy_here) {
    let_later_in();
    wait_for_earlier();
    __shared__ int32_t warp_sums[32];
    __shared__ int32_t own_need, own_free;
    const int tid = threadIdx.x, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    int32_t a0, a1;
    share_of<CL>(b.rows, rank, &a0, &a1);
    const int32_t per = ROWS ? ROWS : (a1 - a0 + XT - 1) / XT;
    const int32_t r0 = min(a1, a0 + tid * per), n_rows = min(a1, r0 + per) - r0;
    constexpr int HELD = ROWS ? ROWS : 1;
    Need held[HELD] = {};
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (i < n_rows) held[i] = row_need(b, add, r0 + i);
    // f(row's number, what it needs) for the thread's rows
    auto each = [&](auto f) {
        if (ROWS) {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i < n_rows) f(r0 + i, held[i]);
        } else {
            for (int32_t i = 0; i < n_rows; ++i) f(r0 + i, row_need(b, add, r0 + i));
        }
    };
    each([&](int32_t, const Need& n) { if (n.page >= 0) { s.sharers[n.page] = 0; s.keeper[n.page] = ~0ull; } });
    if (rank == 0 && tid == 0) s.head[0] = 0;

    // the free pages of this block's share
    int32_t p0, p1, n_free = 0;
    share_of<CL>(b.pages, rank, &p0, &p1);
    int32_t mine = 0;
    for (int32_t p = p0 + tid * 4; p < p1; p += XT * 4) {
        const int4 r = four_refs(b.ref, p, p1);
        mine += (r.x == 0) + (r.y == 0) + (r.z == 0) + (r.w == 0);
    }
    block_scan(mine, warp_sums, &n_free);
    if (tid == 0) own_free = n_free;

    sync_blocks<CL>();
    each([&](int32_t row, const Need& n) { if (n.page >= 0) { atomicAdd(s.sharers + n.page, 1); atomicMin(s.keeper + n.page, keeper_key(b, n, row)); } });
    sync_blocks<CL>();

    auto copies = [&](const Need& n, int32_t row) {
        if (n.page < 0) return 0;
        const int32_t ref = b.ref[n.page];
        if (ref <= 1) return 0;
        return s.sharers[n.page] == ref && s.keeper[n.page] == keeper_key(b, n, row) ? 0 : 1;
    };
    int32_t held_copy[HELD];
    mine = 0;
    if (ROWS) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) held_copy[i] = i < n_rows ? copies(held[i], r0 + i) : 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i < n_rows) mine += held[i].last - held[i].first + held_copy[i];
    } else {
        each([&](int32_t row, const Need& n) {
            const int32_t cp = copies(n, row);
            s.len[row] = cp;
            mine += n.last - n.first + cp;
        });
    }
    int32_t total = 0;
    int32_t at = block_scan(mine, warp_sums, &total);
    if (tid == 0) own_need = total;
    int32_t before, needed, free_before, free_all;
    cluster_sums<CL>(&own_need, rank, &before, &needed);
    at += before;
    free_before = 0;
    free_all = 0;
#pragma unroll
    for (uint32_t c = 0; c < CL; ++c) {
        const int32_t v = CL == 1 ? own_free : remote_int(&own_free, c);
        if (c < rank) free_before += v;
        free_all += v;
    }

    // the free pages, lowest first, as far as they are needed
    for (int32_t q = p0; q < p1 && free_before < needed; q += XT * 4) {
        const int32_t p = q + tid * 4;
        const int4 r = p < p1 ? four_refs(b.ref, p, p1) : make_int4(1, 1, 1, 1);
        const int32_t mask = (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
        int32_t got = 0;
        int32_t x = free_before + block_scan(__popc(mask), warp_sums, &got);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if ((mask >> j) & 1) {
                if (x < needed) s.list[x] = p + j;
                ++x;
            }
        free_before += got;
    }
    // every decision has been made on the counts as they were, the list is complete; then the counts change
    sync_blocks<CL>();
    // by whole warps, also for lanes without a row
    auto settle = [&](bool some, int32_t row, const Need& n, int32_t cp) {
        uint8_t st = 0;
        bool copy = false;
        int32_t to = 0;
        if (some && n.add > 0) {
            const int32_t pages = n.last - n.first + cp;
            if (n.too_long || (pages > 0 && at + pages > free_all)) st = DISC_ROW_NOPAGE;
            else {
                int32_t from = at;
                int32_t* t = b.table + size_t(row) * b.width;
                if (cp) {
                    copy = true;
                    to = s.list[from++];
                    t[n.first - 1] = to;
                    b.ref[to] = 1;
                    atomicAdd(b.ref + n.page, -1);
                }
                for (int32_t j = n.first; j < n.last; ++j) {
                    const int32_t page = s.list[from++];
                    t[j] = page;
                    b.ref[page] = 1;
                }
                b.len[row] = n.len + n.add;
            }
            if (!n.too_long) at += pages;
        }
        if (some) status[row] = st;
        // a place in the list of copies, whose order does not matter
        const unsigned copying = __ballot_sync(FULL, copy);
        if (copying) {
            const int first = __ffs(copying) - 1;
            int32_t base = 0;
            if (lane == first) base = atomicAdd(s.head, __popc(copying));
            base = __shfl_sync(FULL, base, first);
            if (copy) s.copy[base + __popc(copying & ((1u << lane) - 1u))] = make_int4(n.page, to, n.len & (b.page_size - 1), 0);
        }
    };
    if (ROWS) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) settle(i < n_rows, r0 + i, held[i], held_copy[i]);
    } else {
        // the copies are decided by counts that other rows are changing: they were noted with the decision
        for (int32_t i = 0; i < per; ++i) {
            const bool some = i < n_rows;
            Need n = {};
            if (some) n = row_need(b, add, r0 + i);
            settle(some, r0 + i, n, some ? s.len[r0 + i] : 0);
        }
    }
    sync_blocks<CL>();                                    // no block leaves while another may still read its shared memory
    if (CL == 1 && copy_here) copy_units(o, s, tid >> 5, XT / 32, int64_t(s.head[0]) * o.planes * o.heads);
}

// ---- write -------------------------------------------------------------------------------------------
struct WriteParams {
    const unsigned char* k;
    const unsigned char* v;
    int64_t k_token, k_head, v_token, v_head;   // strides in bytes
    const int32_t* cu;                          // [n+1] nullable: one token per sequence
    const int32_t* rows;                        // [n] nullable: sequence i is row i
    const uint8_t* status;                      // [rows] nullable: rows with a status are left alone
    int32_t n, tokens;
    unsigned char* k_plane;
    unsigned char* v_plane;
    int32_t heads, head_bytes, token_bytes;
};
// one warp per new token: its keys and values of all heads
__global__ void __launch_bounds__(256) cache_write_kernel(Books b, WriteParams w) {
    let_later_in();
    wait_for_earlier();
    const int32_t t = int32_t((int64_t(blockIdx.x) * blockDim.x + threadIdx.x) >> 5);       // up to 2^30 tokens: 2^35 threads
    const int lane = threadIdx.x & 31;
    if (t >= w.tokens) return;
    int32_t seq = t, back = 1;                  // the token is the back-th from the end of its sequence
    if (w.cu) {
        int32_t lo = 0, hi = w.n;               // cu[lo] <= t < cu[hi]
        if (t < w.cu[0] || t >= w.cu[w.n]) return;
        while (hi - lo > 1) {
            const int32_t m = (lo + hi) >> 1;
            if (w.cu[m] <= t) lo = m; else hi = m;
        }
        seq = lo;
        back = w.cu[lo + 1] - t;
    }
    const int32_t row = w.rows ? w.rows[seq] : seq;
    if (row < 0 || row >= b.rows || (w.status && w.status[row])) return;
    const int32_t pos = b.len[row] - back;
    if (pos < 0) return;
    const int32_t page = b.table[size_t(row) * b.width + (pos >> b.shift)], off = pos & (b.page_size - 1);
    if (page < 0 || page >= b.pages) return;
    const int32_t vecs = w.token_bytes / 16, all = vecs * w.heads;
    for (int32_t i = lane; i < 2 * all; i += 32) {
        const bool val = i >= all;
        const int32_t j = val ? i - all : i, h = j / vecs, x = j - h * vecs;
        const unsigned char* from = (val ? w.v + t * w.v_token + h * w.v_head : w.k + t * w.k_token + h * w.k_head) + x * 16;
        unsigned char* to = (val ? w.v_plane : w.k_plane) + (int64_t(page) * w.heads + h) * w.head_bytes + int64_t(off) * w.token_bytes + x * 16;
        *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
    }
}

// ---- compact -----------------------------------------------------------------------------------------
// One cluster: the number n of live pages; the live pages at n and above, in order, are to go to the free pages below
// n, in order; their reference counts go along.
template <int CL>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(XT) cache_plan_compact_kernel(Books b, Scratch s, int32_t* live_out) {
    let_later_in();
    wait_for_earlier();
    __shared__ int32_t warp_sums[32];
    __shared__ int32_t own_live, own_holes, own_movers;
    const int tid = threadIdx.x;
    const uint32_t rank = cluster_rank();
    int32_t p0, p1;
    share_of<CL>(b.pages, rank, &p0, &p1);
    int32_t mine = 0, total = 0;
    for (int32_t p = p0 + tid * 4; p < p1; p += XT * 4) {
        const int4 r = four_refs(b.ref, p, p1);
        const int32_t here = min(4, p1 - p);
        mine += (r.x > 0) + (here > 1 && r.y > 0) + (here > 2 && r.z > 0) + (here > 3 && r.w > 0);
    }
    block_scan(mine, warp_sums, &total);
    if (tid == 0) own_live = total;
    int32_t before, live;
    cluster_sums<CL>(&own_live, rank, &before, &live);
    // holes of this share: its places below n that no live page has; movers: its live pages from n on
    const int32_t below = max(0, min(p1, live) - p0);
    int32_t live_below = 0;
    mine = 0;
    for (int32_t p = p0 + tid * 4; p < min(p1, live); p += XT * 4) {
        const int4 r = four_refs(b.ref, p, p1);
        const int32_t here = min(4, min(p1, live) - p);
        mine += (r.x > 0) + (here > 1 && r.y > 0) + (here > 2 && r.z > 0) + (here > 3 && r.w > 0);
    }
    block_scan(mine, warp_sums, &live_below);
    if (tid == 0) { own_holes = below - live_below; own_movers = total - live_below; }
    int32_t holes, movers, n_holes, n_movers;
    cluster_sums<CL>(&own_holes, rank, &holes, &n_holes);
    movers = 0;
    n_movers = 0;
#pragma unroll
    for (uint32_t c = 0; c < CL; ++c) {
        const int32_t v = CL == 1 ? own_movers : remote_int(&own_movers, c);
        if (c < rank) movers += v;
        n_movers += v;
    }
    for (int32_t q = p0; q < p1; q += XT * 4) {
        const int32_t p = q + tid * 4;
        const int4 r4 = p < p1 ? four_refs(b.ref, p, p1) : make_int4(1, 1, 1, 1);
        const int32_t r[4] = {r4.x, r4.y, r4.z, r4.w};
        int32_t h = 0, m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = p + j < p1;
            h |= int32_t(in && p + j < live && r[j] <= 0) << j;
            m |= int32_t(in && p + j >= live && r[j] > 0) << j;
        }
        int32_t n = 0;
        const int32_t at = block_scan(__popc(h) | (__popc(m) << 16), warp_sums, &n);
        int32_t ih = holes + (at & 0xffff), im = movers + (at >> 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if ((h >> j) & 1) s.move[ih++].y = p + j;
            if ((m >> j) & 1) s.move[im++].x = p + j;
            if (p + j < p1) s.list[p + j] = p + j;
        }
        holes += n & 0xffff;
        movers += n >> 16;
    }
    sync_blocks<CL>();
    for (int32_t i = int32_t(rank) * XT + tid; i < n_movers; i += CL * XT) {
        const int2 m = s.move[i];
        s.list[m.x] = m.y;
        b.ref[m.y] = b.ref[m.x];
        b.ref[m.x] = 0;
    }
    if (rank == 0 && tid == 0) { s.head[1] = live; s.head[2] = n_movers; *live_out = live; }
}
// The moves, a block per page and plane, and the new page numbers in the table.
__global__ void __launch_bounds__(256) cache_move_kernel(Books b, unsigned char* pool, Scratch s, int32_t planes,
                                                         int64_t plane_bytes, int32_t page_bytes) {
    let_later_in();
    wait_for_earlier();
    const int64_t entries = int64_t(b.rows) * b.width;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < entries; i += int64_t(gridDim.x) * blockDim.x) {
        const int32_t p = b.table[i];
        if (p >= 0 && p < b.pages) b.table[i] = s.list[p];
    }
    const int64_t n = int64_t(s.head[2]) * planes;
    const int32_t vecs = page_bytes / 16;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int2 m = s.move[i / planes];
        unsigned char* plane = pool + (i % planes) * plane_bytes;
        const uint4* from = reinterpret_cast<const uint4*>(plane + int64_t(m.x) * page_bytes);
        uint4* to = reinterpret_cast<uint4*>(plane + int64_t(m.y) * page_bytes);
        for (int32_t v0 = threadIdx.x; v0 < vecs; v0 += 256 * 4) {
            uint4 x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (v0 + u * 256 < vecs) x[u] = __ldcs(from + v0 + u * 256);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (v0 + u * 256 < vecs) __stcs(to + v0 + u * 256, x[u]);
        }
    }
}

int check_cache(const disc_cache_t* c) {
    if (!c || !c->pool || !c->table || !c->len || !c->ref || !c->scratch) return DISC_ERR_ARG;
    if (const int rc = disc::cache_sizes(c)) return rc;
    if (c->scratch_bytes < scratch_layout(c, nullptr)) return DISC_ERR_ARG;
    return DISC_OK;
}

Books books(const disc_cache_t* c) {
    Books b;
    b.table = c->table; b.len = c->len; b.ref = c->ref;
    b.rows = c->n_rows; b.width = c->table_width; b.pages = c->n_pages; b.page_size = c->page_size;
    b.shift = 0;
    while ((1 << b.shift) < c->page_size) ++b.shift;
    return b;
}

int take(const disc_cache_t* c, const int32_t* parent, const uint8_t* freed, cudaStream_t st) {
    Scratch s;
    scratch_layout(c, &s);
    if (c->n_rows <= 32) return launch_after(cache_fork_kernel<2>, 1, unsigned(c->n_rows) * 32, 0, st, books(c), parent, freed, s);
    const unsigned grid = unsigned((int64_t(c->n_rows) * 32 + 255) / 256);
    if (const int rc = launch_after(cache_fork_kernel<0>, grid, 256, 0, st, books(c), parent, freed, s)) return rc;
    return launch_after(cache_fork_kernel<1>, grid, 256, 0, st, books(c), parent, freed, s);
}

}  // namespace

// the sizes of a cache alone
int disc::cache_sizes(const disc_cache_t* c) {
    if (c->n_layers <= 0 || c->n_pages <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 || c->n_rows <= 0 || c->table_width <= 0) return DISC_ERR_ARG;
    if (c->dtype != DISC_BF16 && c->dtype != DISC_F16) return DISC_ERR_UNSUPPORTED;
    if (c->head_dim % 8 || c->head_dim > DISC_MAX_HEAD_DIM) return DISC_ERR_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 128 || (c->page_size & (c->page_size - 1))) return DISC_ERR_UNSUPPORTED;
    // a row's tokens are counted in 32 bits, pages and rows in 2^26 at most
    if (c->n_pages > (1 << 26) || c->n_rows > (1 << 26) || int64_t(c->table_width) * c->page_size >= (int64_t(1) << 31) ||
        int64_t(c->n_rows) * c->table_width > (int64_t(1) << 30)) return DISC_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(c->pool) | reinterpret_cast<uintptr_t>(c->scratch)) & 15u) return DISC_ERR_ARG;
    return DISC_OK;
}

extern "C" {

int64_t disc_cache_scratch_bytes(const disc_cache_t* c) {
    if (!c || c->n_rows <= 0 || c->n_pages <= 0 || c->table_width <= 0) return DISC_ERR_ARG;
    return scratch_layout(c, nullptr);
}

int disc_cache_fork(const disc_cache_t* c, const int32_t* parent, void* stream) {
    if (const int rc = check_cache(c)) return rc;
    if (!parent) return DISC_ERR_ARG;
    return take(c, parent, nullptr, static_cast<cudaStream_t>(stream));
}

int disc_cache_free(const disc_cache_t* c, const uint8_t* freed, void* stream) {
    if (const int rc = check_cache(c)) return rc;
    if (!freed) return DISC_ERR_ARG;
    return take(c, nullptr, freed, static_cast<cudaStream_t>(stream));
}

int disc_cache_extend(const disc_cache_t* c, const int32_t* add, uint8_t* status_out, void* stream) {
    if (const int rc = check_cache(c)) return rc;
    if (!status_out) return DISC_ERR_ARG;
    Scratch s;
    scratch_layout(c, &s);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if (const int rc = device_sms(&sms)) return rc;
    // rows of a thread: up to 4 are held in registers
    const int64_t share = ((int64_t(c->n_rows) + CLUSTER - 1) / CLUSTER + 3) & ~int64_t(3), per = (share + XT - 1) / XT;
    const bool one = c->n_rows <= XT && c->n_pages <= ONE_BLOCK;
    Pool o;
    o.base = static_cast<unsigned char*>(c->pool); o.planes = c->n_layers * 2; o.heads = c->n_kv_heads;
    o.token_bytes = c->head_dim * 2; o.head_bytes = c->page_size * o.token_bytes;
    o.plane_bytes = int64_t(c->n_pages) * c->n_kv_heads * o.head_bytes;
    // copies that the one block can make itself, up to 8 a warp, are not worth a launch
    const int64_t units = int64_t(c->n_rows) * o.planes * o.heads;
    const bool copy_here = one && units <= XT / 32 * 8;
    auto extend = one ? cache_extend_kernel<1, 1> : per <= 1 ? cache_extend_kernel<CLUSTER, 1> : per <= 4 ? cache_extend_kernel<CLUSTER, 4> : cache_extend_kernel<CLUSTER, 0>;
    if (const int rc = launch_after(extend, one ? 1 : CLUSTER, XT, 0, st, books(c), add, s, status_out, o, copy_here)) return rc;
    if (copy_here) return DISC_OK;
    const int64_t most = (units + 7) / 8;
    return launch_after(cache_copy_kernel, unsigned(most < sms * 8 ? most : sms * 8), 256, 0, st, o, s);
}

int disc_cache_write(const disc_cache_t* c, int32_t layer, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                     int64_t v_token_stride, int64_t v_head_stride, int64_t n_tokens, const int32_t* cu, int32_t n_seqs,
                     const int32_t* rows, const uint8_t* status, void* stream) {
    if (const int rc = check_cache(c)) return rc;
    if (layer < 0 || layer >= c->n_layers || n_tokens < 0 || n_seqs < 0 || n_tokens > (int64_t(1) << 30)) return DISC_ERR_ARG;
    if (!cu && n_tokens != n_seqs) return DISC_ERR_ARG;
    if (!rows && n_seqs > c->n_rows) return DISC_ERR_ARG;
    if (n_tokens == 0 || n_seqs == 0) return DISC_OK;
    if (!k || !v) return DISC_ERR_ARG;
    // the stride over an axis of one is never used
    if (n_tokens == 1) k_token_stride = v_token_stride = 0;
    if (c->n_kv_heads == 1) k_head_stride = v_head_stride = 0;
    // 16-byte reads: the bases on 16-byte boundaries, the strides multiples of 8 values
    if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u) return DISC_ERR_ARG;
    if ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) & 7) return DISC_ERR_UNSUPPORTED;
    WriteParams w;
    w.k = static_cast<const unsigned char*>(k); w.v = static_cast<const unsigned char*>(v);
    w.k_token = k_token_stride * 2; w.k_head = k_head_stride * 2; w.v_token = v_token_stride * 2; w.v_head = v_head_stride * 2;
    w.cu = cu; w.rows = rows; w.status = status; w.n = n_seqs; w.tokens = int32_t(n_tokens);
    w.heads = c->n_kv_heads; w.token_bytes = c->head_dim * 2; w.head_bytes = c->page_size * w.token_bytes;
    const int64_t plane = int64_t(c->n_pages) * w.heads * w.head_bytes;
    w.k_plane = static_cast<unsigned char*>(c->pool) + 2 * int64_t(layer) * plane;
    w.v_plane = w.k_plane + plane;
    return launch_after(cache_write_kernel, unsigned((n_tokens * 32 + 255) / 256), 256, 0, static_cast<cudaStream_t>(stream), books(c), w);
}

int disc_cache_compact(const disc_cache_t* c, int32_t* live_out, void* stream) {
    if (const int rc = check_cache(c)) return rc;
    if (!live_out) return DISC_ERR_ARG;
    Scratch s;
    scratch_layout(c, &s);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if (const int rc = device_sms(&sms)) return rc;
    const bool one = c->n_pages <= ONE_BLOCK;
    auto plan = one ? cache_plan_compact_kernel<1> : cache_plan_compact_kernel<CLUSTER>;
    if (const int rc = launch_after(plan, one ? 1 : CLUSTER, XT, 0, st, books(c), s, live_out)) return rc;
    const int32_t page_bytes = c->n_kv_heads * c->page_size * c->head_dim * 2;
    return launch_after(cache_move_kernel, unsigned(sms * 8), 256, 0, st, books(c), static_cast<unsigned char*>(c->pool), s, c->n_layers * 2,
                        int64_t(c->n_pages) * page_bytes, page_bytes);
}

}  // extern "C"
