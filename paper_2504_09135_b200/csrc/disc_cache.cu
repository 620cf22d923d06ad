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
// What these calls cost is latency, a few dependent reads of small arrays, except for the copies of page
// contents, which are bound by the bytes.

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
    int32_t* keeper;      // [pages]
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
    t.keeper = reinterpret_cast<int32_t*>(take(pages * 4));
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
// One warp per row.  The first kernel notes every changing row's new pages and moves the reference counts;
// the second writes the table.  Two launches, because a row that changes may be another row's parent.
__global__ void __launch_bounds__(256) cache_take_kernel(Books b, const int32_t* __restrict__ parent, const uint8_t* __restrict__ freed,
                                                         Scratch s) {
    const int32_t row = int32_t((blockIdx.x * blockDim.x + threadIdx.x) >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= b.rows) return;
    const int32_t p = parent ? parent[row] : (freed[row] ? -1 : row);
    if (p == row) return;
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
__global__ void __launch_bounds__(256) cache_settle_kernel(Books b, const int32_t* __restrict__ parent, const uint8_t* __restrict__ freed,
                                                           Scratch s) {
    const int32_t row = int32_t((blockIdx.x * blockDim.x + threadIdx.x) >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= b.rows) return;
    const int32_t p = parent ? parent[row] : (freed[row] ? -1 : row);
    if (p == row) return;
    const int32_t used = (s.len[row] + b.page_size - 1) >> b.shift, old = (b.len[row] + b.page_size - 1) >> b.shift;
    const int32_t* from = s.table + size_t(row) * b.width;
    int32_t* to = b.table + size_t(row) * b.width;
    for (int32_t j = lane; j < max(used, old); j += 32) to[j] = j < used ? from[j] : -1;
    __syncwarp();
    if (lane == 0) b.len[row] = s.len[row];
}

// ---- extend ------------------------------------------------------------------------------------------
constexpr int XT = 1024;

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
    if (warp == 0) {
        int32_t w = warp_sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t u = __shfl_up_sync(FULL, w, o);
            if (lane >= o) w += u;
        }
        warp_sums[lane] = w;
    }
    __syncthreads();
    *total = warp_sums[31];
    return incl - v + (warp ? warp_sums[warp - 1] : 0);
}

struct Need {
    int32_t add, len, first, last, page, copy, pages;      // table positions [first, last) are new; page: the partial last one or -1
};
__device__ __forceinline__ Need row_need(const Books& b, const int32_t* add, int32_t row) {
    Need n;
    n.add = add ? add[row] : 1;
    n.len = b.len[row];
    n.first = (n.len + b.page_size - 1) >> b.shift;
    n.page = -1;
    n.copy = 0;
    n.last = n.first;
    if (n.add > 0) {
        n.last = int32_t((int64_t(n.len) + n.add + b.page_size - 1) >> b.shift);
        if (n.len & (b.page_size - 1)) n.page = b.table[size_t(row) * b.width + n.first - 1];
    }
    n.pages = n.last - n.first;
    return n;
}
// no room in the table for the row's pages
__device__ __forceinline__ bool too_long(const Books& b, const Need& n) {
    return int64_t(n.len) + n.add > (int64_t(b.width) << b.shift);
}

// One block: the arrays are small and every step hangs on the one before.
//  1. Rows that go on writing into a partly filled page mark it: how many rows do (sharers), and the lowest of
//     them (keeper).  If they are all the rows that hold the page, the keeper writes on in place; the others, and
//     all of them where a row that stays behind holds the page too, get a copy.
//  2. Prefix sums over the rows of the pages they need; rows beyond the number of free pages get nothing.
//  3. The free pages of lowest id, in order, as many as are needed, and from them each row's share.
__global__ void __launch_bounds__(XT) cache_extend_kernel(Books b, const int32_t* __restrict__ add, Scratch s, uint8_t* __restrict__ status) {
    __shared__ int32_t warp_sums[32];
    const int tid = threadIdx.x;
    for (int32_t row = tid; row < b.rows; row += XT) {
        const Need n = row_need(b, add, row);
        if (n.page >= 0 && !too_long(b, n)) { s.sharers[n.page] = 0; s.keeper[n.page] = 0x7fffffff; }
    }
    __syncthreads();
    for (int32_t row = tid; row < b.rows; row += XT) {
        const Need n = row_need(b, add, row);
        if (n.page >= 0 && !too_long(b, n)) { atomicAdd(s.sharers + n.page, 1); atomicMin(s.keeper + n.page, row); }
    }
    __syncthreads();

    // pages needed in all
    int32_t mine = 0;
    const int32_t per = (b.rows + XT - 1) / XT;            // rows of a thread: consecutive
    const int32_t r0 = min(b.rows, tid * per), r1 = min(b.rows, r0 + per);
    auto copies = [&](const Need& n, int32_t row) {
        if (n.page < 0) return 0;
        const int32_t ref = b.ref[n.page];
        if (ref <= 1) return 0;
        return s.sharers[n.page] == ref && s.keeper[n.page] == row ? 0 : 1;
    };
    for (int32_t row = r0; row < r1; ++row) {
        const Need n = row_need(b, add, row);
        if (n.add > 0 && !too_long(b, n)) mine += n.pages + copies(n, row);
    }
    int32_t needed = 0;
    const int32_t before = block_scan(mine, warp_sums, &needed);

    // the free pages, lowest first, as far as they are needed
    int32_t n_free = 0;
    if (needed > 0) {
        for (int32_t p0 = 0; p0 < b.pages && n_free < needed; p0 += XT * 4) {
            int32_t mask = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t p = p0 + tid * 4 + j;
                if (p < b.pages && b.ref[p] == 0) mask |= 1 << j;
            }
            int32_t got = 0;
            int32_t at = n_free + block_scan(__popc(mask), warp_sums, &got);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if ((mask >> j) & 1) s.list[at++] = p0 + tid * 4 + j;
            n_free += got;
        }
    }
    if (tid == 0) s.head[0] = 0;
    __syncthreads();

    int32_t at = before, n_copy = 0;
    // two rounds over the thread's rows: the decisions read the reference counts and marks, then the counts change
    for (int32_t row = r0; row < r1; ++row) {
        const Need n = row_need(b, add, row);
        uint8_t st = 0;
        int32_t share = -1;                                // where the row's pages start in the list, + copy bit
        if (n.add > 0) {
            if (too_long(b, n)) st = DISC_ROW_NOPAGE;
            else {
                const int32_t cp = copies(n, row), pages = n.pages + cp;
                if (pages > 0 && at + pages > n_free) st = DISC_ROW_NOPAGE;
                else { share = at * 2 + cp; n_copy += cp; }
                at += pages;
            }
        }
        s.len[row] = share;
        status[row] = st;
    }
    int32_t all = 0;
    int32_t slot = block_scan(n_copy, warp_sums, &all);
    for (int32_t row = r0; row < r1; ++row) {
        const int32_t share = s.len[row];
        if (share < 0) continue;
        const Need n = row_need(b, add, row);
        int32_t from = share >> 1;
        int32_t* t = b.table + size_t(row) * b.width;
        if (share & 1) {
            const int32_t to = s.list[from++];
            s.copy[slot++] = make_int4(n.page, to, n.len & (b.page_size - 1), 0);
            t[n.first - 1] = to;
            b.ref[to] = 1;
            atomicAdd(b.ref + n.page, -1);
        }
        for (int32_t j = n.first; j < n.last; ++j) {
            const int32_t to = s.list[from++];
            t[j] = to;
            b.ref[to] = 1;
        }
        b.len[row] = n.len + n.add;
    }
    if (tid == 0) s.head[0] = all;
}

// The copies of the partly filled pages: a warp per copy, plane and head, which is one run of tokens x head dim.
__global__ void __launch_bounds__(256) cache_copy_kernel(unsigned char* __restrict__ pool, Scratch s, int32_t planes, int32_t heads,
                                                         int64_t plane_bytes, int32_t head_bytes, int32_t token_bytes) {
    const int lane = threadIdx.x & 31;
    const int64_t n = int64_t(s.head[0]) * planes * heads;
    const int64_t step = int64_t(gridDim.x) * (blockDim.x >> 5);
    for (int64_t i = (int64_t(blockIdx.x) * blockDim.x + threadIdx.x) >> 5; i < n; i += step) {
        const int32_t h = int32_t(i % heads);
        const int64_t j = i / heads;
        const int32_t pl = int32_t(j % planes);
        const int4 c = s.copy[j / planes];
        const uint4* from = reinterpret_cast<const uint4*>(pool + pl * plane_bytes + (int64_t(c.x) * heads + h) * head_bytes);
        uint4* to = reinterpret_cast<uint4*>(pool + pl * plane_bytes + (int64_t(c.y) * heads + h) * head_bytes);
        const int32_t vecs = c.z * token_bytes / 16;
        for (int32_t v = lane; v < vecs; v += 32) to[v] = from[v];
    }
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
    const int32_t t = int32_t((blockIdx.x * blockDim.x + threadIdx.x) >> 5);
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
// One block: the number n of live pages; the live pages at n and above, in order, are to go to the free pages below
// n, in order; their reference counts go along.
__global__ void __launch_bounds__(XT) cache_plan_compact_kernel(Books b, Scratch s, int32_t* __restrict__ live_out) {
    __shared__ int32_t warp_sums[32];
    const int tid = threadIdx.x;
    int32_t mine = 0;
    for (int32_t p = tid; p < b.pages; p += XT) mine += b.ref[p] > 0;
    int32_t live = 0;
    block_scan(mine, warp_sums, &live);
    int32_t holes = 0, movers = 0;
    for (int32_t p0 = 0; p0 < b.pages; p0 += XT) {
        const int32_t p = p0 + tid;
        const int32_t ref = p < b.pages ? b.ref[p] : 0;
        const bool hole = p < live && ref <= 0, mover = p >= live && p < b.pages && ref > 0;
        int32_t n = 0;
        const int32_t at = block_scan(hole | (mover << 16), warp_sums, &n);
        if (hole) s.move[holes + (at & 0xffff)].y = p;
        if (mover) s.move[movers + (at >> 16)].x = p;
        if (p < b.pages) s.list[p] = p;
        holes += n & 0xffff;
        movers += n >> 16;
    }
    __syncthreads();
    for (int32_t i = tid; i < movers; i += XT) {
        const int2 m = s.move[i];
        s.list[m.x] = m.y;
        b.ref[m.y] = b.ref[m.x];
        b.ref[m.x] = 0;
    }
    if (tid == 0) { s.head[1] = live; s.head[2] = movers; *live_out = live; }
}
// The moves, a block per page and plane, and the new page numbers in the table.
__global__ void __launch_bounds__(256) cache_move_kernel(Books b, unsigned char* __restrict__ pool, Scratch s, int32_t planes,
                                                         int64_t plane_bytes, int32_t page_bytes) {
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
        for (int32_t v = threadIdx.x; v < vecs; v += blockDim.x) to[v] = from[v];
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
    const unsigned grid = unsigned((int64_t(c->n_rows) * 32 + 255) / 256);
    cache_take_kernel<<<grid, 256, 0, st>>>(books(c), parent, freed, s);
    cache_settle_kernel<<<grid, 256, 0, st>>>(books(c), parent, freed, s);
    DISC_CUDA(cudaGetLastError());
    return DISC_OK;
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
    cache_extend_kernel<<<1, XT, 0, st>>>(books(c), add, s, status_out);
    const int32_t planes = c->n_layers * 2, token_bytes = c->head_dim * 2, head_bytes = c->page_size * token_bytes;
    const int64_t most = (int64_t(c->n_rows) * planes * c->n_kv_heads + 7) / 8;
    const unsigned grid = unsigned(most < sms * 8 ? most : sms * 8);
    cache_copy_kernel<<<grid, 256, 0, st>>>(static_cast<unsigned char*>(c->pool), s, planes, c->n_kv_heads,
                                            int64_t(c->n_pages) * c->n_kv_heads * head_bytes, head_bytes, token_bytes);
    DISC_CUDA(cudaGetLastError());
    return DISC_OK;
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
    cache_write_kernel<<<unsigned((n_tokens * 32 + 255) / 256), 256, 0, static_cast<cudaStream_t>(stream)>>>(books(c), w);
    DISC_CUDA(cudaGetLastError());
    return DISC_OK;
}

int disc_cache_compact(const disc_cache_t* c, int32_t* live_out, void* stream) {
    if (const int rc = check_cache(c)) return rc;
    if (!live_out) return DISC_ERR_ARG;
    Scratch s;
    scratch_layout(c, &s);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if (const int rc = device_sms(&sms)) return rc;
    cache_plan_compact_kernel<<<1, XT, 0, st>>>(books(c), s, live_out);
    const int32_t page_bytes = c->n_kv_heads * c->page_size * c->head_dim * 2;
    cache_move_kernel<<<unsigned(sms * 8), 256, 0, st>>>(books(c), static_cast<unsigned char*>(c->pool), s, c->n_layers * 2,
                                                         int64_t(c->n_pages) * page_bytes, page_bytes);
    DISC_CUDA(cudaGetLastError());
    return DISC_OK;
}

}  // extern "C"
