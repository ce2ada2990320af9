// Paged cache: forking, keeping the accepted path of a draft, compacting.  A call reads one page book and writes
// another, so that a call that finds too few pages leaves the caller with the book it had.
//
// Each call is two launches: a small one that decides (one block walks the rows and the pages' counts in order, since
// a fresh page's number depends on every row and page before it) and one that moves pages and writes the new
// book with the whole GPU.  Bound by HBM where pages move (every byte read once and written once, 16 bytes a thread and
// access), else by the two launches; the second is chained to the first.  A call that has little to do is one launch instead, a cluster of eight blocks
// with the cluster's barrier between the two parts.
#include "plc_pages.cuh"

namespace plc {
namespace {

constexpr int kPlanThreads = 1024, kMoveThreads = 256;
constexpr int kFewBlocks = 8, kFewThreads = kPlanThreads;
constexpr int kPartBytes = 32768;                 // of a page's plane (one layer's keys or values): a block's share at a time

struct Workspace {
    int32_t* head;      // [4]: page moves, shortage
    int32_t* first;     // [rows_in] lowest row that continues the row
    int32_t* count;     // [rows_in] rows that continue it
    int32_t* base;      // [rows_out] index of the row's first fresh page in `list`
    int32_t* src;       // [moves] page to copy, index in `list` of where to, slots
    int32_t* at;
    int32_t* used;
    int32_t* list;      // [n_pages] fresh pages in order
};
uint64_t workspace_words(int64_t n_pages, int64_t rows_in, int64_t rows_out) {
    const int64_t moves = rows_out > n_pages ? rows_out : n_pages;
    return (uint64_t)(4 + 2 * rows_in + rows_out + 3 * moves + n_pages);
}
Workspace workspace_at(void* p, int64_t n_pages, int64_t rows_in, int64_t rows_out) {
    const int64_t moves = rows_out > n_pages ? rows_out : n_pages;
    Workspace w;
    w.head = static_cast<int32_t*>(p);
    w.first = w.head + 4;
    w.count = w.first + rows_in;
    w.base = w.count + rows_in;
    w.src = w.base + rows_out;
    w.at = w.src + moves;
    w.used = w.at + moves;
    w.list = w.used + moves;
    return w;
}

// Exclusive sum over the block's threads; *total receives the whole sum.  Every thread calls it.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* total) {
    __shared__ unsigned long long part[kPlanThreads / 32];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    unsigned long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(kFull, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                              // the previous call's sums have been read
    if (lane == 31) part[wid] = x;
    __syncthreads();
    unsigned long long ahead = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w) {
        const unsigned long long p = part[w];
        if (w < wid) ahead += p;
        all += p;
    }
    *total = all;
    return ahead + x - v;
}

// All of a cluster's blocks have come here, and see what the others have written.
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// What row s of the new book continues.
struct ForkRow {
    int from;             // row of the old book, -1: none
    int len, full, has, wants;   // positions; full pages; pages that hold positions; pages that the row shall have
    bool bad, wide;       // something out of range; more pages than a row has room for
};
__device__ __forceinline__ ForkRow fork_row(const PoolDev& p, const BookDev& in, const int32_t* parent, const int32_t* room, int s) {
    ForkRow r{-1, 0, 0, 0, 0, false, false};
    const int from = parent[s];
    if (from == -1) return r;
    if (from < 0 || from >= in.rows) { r.bad = true; return r; }
    const int len = in.len[from], more = room ? room[s] : 0;
    if (len < 0 || len > most_positions(in, p) || more < 0) { r.bad = true; return r; }
    r.from = from;
    r.len = len;
    r.full = len / p.page_pos;
    r.has = r.full + (len % p.page_pos != 0);
    const long long wants = ((long long)len + more + p.page_pos - 1) / p.page_pos;
    r.wide = wants > in.max_pages;
    r.wants = r.wide ? r.has : (int)wants;
    return r;
}
__device__ __forceinline__ bool page_ok(const PoolDev& p, int page) { return page >= 0 && page < p.n_pages; }

// Whether row s copies the partly filled page of the row that it continues (*last): it is not the first to continue
// it, or somebody else holds the page too.
__device__ __forceinline__ bool fork_copies(const PoolDev& p, const BookDev& in, const ForkRow& r, int s, int first, int* last) {
    if (r.from < 0 || r.has == r.full) return false;
    *last = in.table[(long long)r.from * in.max_pages + r.full];
    return page_ok(p, *last) && (first != s || in.ref[*last] != 1);
}

// Block 0 plans; the others copy the counts, which the second launch then changes.
__device__ __forceinline__ void fork_plan(const PoolDev& p, const BookDev& in, const BookDev& out, const int32_t* parent, const int32_t* room, const Workspace& w,
                                          uint32_t* status) {
    const int tid = threadIdx.x;
    if (blockIdx.x > 0) {
        for (long long i = (long long)(blockIdx.x - 1) * kPlanThreads + tid; i < p.n_pages; i += (long long)(gridDim.x - 1) * kPlanThreads)
            out.ref[i] = in.ref[i];
        return;
    }
    for (int r = tid; r < in.rows; r += kPlanThreads) { w.first[r] = 0x7fffffff; w.count[r] = 0; }
    __syncthreads();
    uint32_t bits = 0;
    for (int s = tid; s < out.rows; s += kPlanThreads) {
        const ForkRow r = fork_row(p, in, parent, room, s);
        if (r.bad) bits |= kStRange;
        if (r.wide) bits |= kStCapacity;
        if (r.from >= 0) { atomicMin(&w.first[r.from], s); atomicAdd(&w.count[r.from], 1); }
    }
    __syncthreads();
    unsigned long long need = 0;                   // fresh pages in the low half, copies in the high half
    for (int s0 = 0; s0 < out.rows; s0 += kPlanThreads) {
        const int s = s0 + tid;
        unsigned long long mine = 0;
        int last = -1, used = 0;
        if (s < out.rows) {
            const ForkRow r = fork_row(p, in, parent, room, s);
            const bool copies = r.from >= 0 && fork_copies(p, in, r, s, w.first[r.from], &last);
            used = r.len - r.full * p.page_pos;
            mine = (unsigned long long)(r.wants - r.has + (copies ? 1 : 0)) + (copies ? 1ull << 40 : 0ull);
        }
        unsigned long long total;
        const unsigned long long at = need + block_scan(mine, &total);
        if (s < out.rows) {
            w.base[s] = (int)min(at & ((1ull << 40) - 1), 0x7fffffffull);
            if (mine >> 40) {
                const int c = (int)(at >> 40);
                w.src[c] = last;
                w.at[c] = w.base[s];
                w.used[c] = used;
            }
        }
        need += total;
    }
    const unsigned long long pages = need & ((1ull << 40) - 1);
    unsigned long long found = 0;
    for (long long i0 = 0; i0 < p.n_pages && found < pages; i0 += kPlanThreads) {
        const long long i = i0 + tid;
        const bool free = i < p.n_pages && in.ref[i] == 0;
        unsigned long long total;
        const unsigned long long at = found + block_scan(free ? 1 : 0, &total);
        if (free && at < pages) w.list[at] = (int)i;
        found += total;
    }
    if (found < pages) bits |= kStCapacity;
    const bool short_of = __syncthreads_or(bits & kStCapacity);
    if (bits) atomicOr(status, bits);
    if (tid == 0) { w.head[0] = short_of ? 0 : (int)(need >> 40); w.head[1] = short_of; }
}
__global__ void __launch_bounds__(kPlanThreads)
fork_plan_kernel(PoolDev p, BookDev in, BookDev out, const int32_t* parent, const int32_t* room, Workspace w, uint32_t* status) {
    chain_next();
    fork_plan(p, in, out, parent, room, w, status);
}

// Copies `used` slots of one plane of a page, the vectors [v0, v0 + n) of them in the plane's own order.
struct Mover {
    int lanes_log2;       // 16-byte pieces of a vector
    bool slots_inner;     // neighbouring slots are nearer than neighbouring heads
};
template <int THREADS>
__device__ __forceinline__ void move_vectors(const PoolDev& p, const Mover& m, const uint8_t* src, uint8_t* dst, int used, int v0, int n) {
    const int inner = m.slots_inner ? used : p.H;
    const int64_t si = m.slots_inner ? p.sp : p.sh, so = m.slots_inner ? p.sh : p.sp;
    const int units = n << m.lanes_log2;
    for (int u0 = threadIdx.x; u0 < units; u0 += 4 * THREADS) {
        uint4 x[4];
        int64_t off[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int u = u0 + k * THREADS;
            if (u < units) {
                const int v = v0 + (u >> m.lanes_log2), o = v / inner, i = v - o * inner;
                off[k] = o * so + i * si + (int64_t)(u & ((1 << m.lanes_log2) - 1)) * 16;
                x[k] = *reinterpret_cast<const uint4*>(src + off[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (u0 + k * THREADS < units) *reinterpret_cast<uint4*>(dst + off[k]) = x[k];
    }
}
__device__ __forceinline__ int64_t plane_offset(const PoolDev& p, int plane) { return (int64_t)(plane >> 1) * p.sl + (int64_t)(plane & 1) * p.skv; }

// Every page move of the list, one (move, plane, part) a block at a time; `used` null: whole pages.
template <int THREADS>
__device__ __forceinline__ void move_pages(const PoolDev& p, const Mover& m, int moves, const int32_t* src, const int32_t* at, const int32_t* used,
                                           const int32_t* list) {
    const int per_part = max(1, kPartBytes >> (m.lanes_log2 + 4));
    const int parts = (p.page_pos * p.H + per_part - 1) / per_part, planes = 2 * p.L;
    const long long items = (long long)moves * planes * parts;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int part = (int)(item % parts), plane = (int)(item / parts % planes), c = (int)(item / parts / planes);
        const int u = used ? used[c] : p.page_pos, v0 = part * per_part, n = min(per_part, u * p.H - v0);
        if (n <= 0) continue;
        uint8_t* base = p.base + plane_offset(p, plane);
        move_vectors<THREADS>(p, m, base + (int64_t)src[c] * p.spage, base + (int64_t)list[at ? at[c] : c] * p.spage, u, v0, n);
    }
}

template <int THREADS>
__device__ __forceinline__ void fork_move(const PoolDev& p, const Mover& m, const BookDev& in, const BookDev& out, const int32_t* parent, const int32_t* room,
                                          const Workspace& w, uint32_t* status) {
    const bool short_of = w.head[1] != 0;
    const long long step = (long long)gridDim.x * THREADS, t0 = (long long)blockIdx.x * THREADS + threadIdx.x;
    const int cols = out.max_pages;
    uint32_t bits = 0;
    for (long long i = t0; i < (long long)out.rows * cols; i += step) {
        const int s = (int)(i / cols), j = (int)(i - (long long)s * cols);
        int page = -1, len = 0;
        if (!short_of) {
            const ForkRow r = fork_row(p, in, parent, room, s);
            len = r.len;
            if (j < r.wants) {
                int last = -1;
                const bool copies = j >= r.full && fork_copies(p, in, r, s, w.first[r.from], &last);
                if (j < r.has && !(copies && j == r.full)) {
                    page = in.table[(long long)r.from * cols + j];
                    if (!page_ok(p, page)) { bits |= kStRange; page = -1; }
                } else {
                    page = w.list[w.base[s] + (j < r.has ? 0 : j - r.has + (copies ? 1 : 0))];
                    out.ref[page] = 1;             // it was free, and this row alone has it
                }
            }
        }
        out.table[i] = page;
        if (j == 0) out.len[s] = len;
    }
    if (!short_of)
        for (long long i = t0; i < (long long)in.rows * cols; i += step) {
            const int r = (int)(i / cols), j = (int)(i - (long long)r * cols), page = in.table[i];
            if (!page_ok(p, page)) { if (page != -1) bits |= kStRange; continue; }
            const int n = w.count[r];
            int held = 0;                          // new rows that name the page in this one's stead
            if (n > 0) {
                const int len = in.len[r], full = len / p.page_pos;
                held = j < full ? n : j == full && len % p.page_pos != 0 && in.ref[page] == 1 ? 1 : 0;
            }
            if (held != 1) atomicAdd(&out.ref[page], held - 1);
        }
    if (bits) atomicOr(status, bits);
    move_pages<THREADS>(p, m, w.head[0], w.src, w.at, w.used, w.list);
}
__global__ void __launch_bounds__(kMoveThreads)
fork_move_kernel(PoolDev p, Mover m, BookDev in, BookDev out, const int32_t* parent, const int32_t* room, Workspace w, uint32_t* status) {
    chain_wait();
    fork_move<kMoveThreads>(p, m, in, out, parent, room, w, status);
}
__global__ void __launch_bounds__(kFewThreads)
fork_few_kernel(PoolDev p, Mover m, BookDev in, BookDev out, const int32_t* parent, const int32_t* room, Workspace w, uint32_t* status) {
    fork_plan(p, in, out, parent, room, w, status);
    cluster_meet();
    fork_move<kFewThreads>(p, m, in, out, parent, room, w, status);
}

// Whether row s's path can be kept as it is asked for; every thread of the block calls it.
__device__ __forceinline__ bool path_ok(const PoolDev& p, const BookDev& in, const int32_t* path, int n, int stride, int s, int len) {
    bool ok = n >= 0 && n <= stride && len >= 0 && len <= most_positions(in, p);
    if (ok)
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int at = path[i];
            const long long from = (long long)len + at, to = (long long)len + i, most = most_positions(in, p);
            bool good = at >= i && (i == 0 || path[i - 1] < at) && from < most;
            if (good) {
                const int32_t* row = in.table + (long long)s * in.max_pages;
                const int a = row[from / p.page_pos], b = row[to / p.page_pos];
                good = page_ok(p, a) && page_ok(p, b) && (at == i || in.ref[b] == 1);
            }
            ok = ok && good;
        }
    return __syncthreads_and(ok);
}

// Slot len + path[i] -> len + i, i rising: a thread has one 16-byte column of a plane to itself and path[i] >= i, so no
// slot is written before it has been read.  Eight positions' loads are in flight a thread.  Also copies the counts.
constexpr int kKeepThreads = 128, kKeepBatch = 64;
template <int THREADS>
__device__ __forceinline__ void copy_counts(const PoolDev& p, const BookDev& in, const BookDev& out, unsigned block, unsigned blocks) {
    for (long long i = (long long)block * THREADS + threadIdx.x; i < p.n_pages; i += (long long)blocks * THREADS) out.ref[i] = in.ref[i];
}
// `share` of `shares` blocks that move row s.
template <int THREADS>
__device__ __forceinline__ void keep_move(const PoolDev& p, int lanes_log2, const BookDev& in, const int32_t* paths, const int32_t* n_path, int stride, int s, int share,
                                          int shares) {
    __shared__ int64_t from[kKeepBatch], to[kKeepBatch];
    const int n = n_path[s], len = in.len[s];
    const int32_t* path = paths + (long long)s * stride;
    const int32_t* row = in.table + (long long)s * in.max_pages;
    if (n == 0 || !path_ok(p, in, path, n, stride, s, len)) return;
    const int columns = p.H << lanes_log2, blocks = (columns + THREADS - 1) / THREADS, items = 2 * p.L * blocks;
    for (int i0 = 0; i0 < n; i0 += kKeepBatch) {
        const int m = min(kKeepBatch, n - i0);
        __syncthreads();
        for (int i = threadIdx.x; i < m; i += THREADS) {
            const int a = len + path[i0 + i], b = len + i0 + i;
            from[i] = a == b ? -1 : (int64_t)row[a / p.page_pos] * p.spage + (int64_t)(a % p.page_pos) * p.sp;
            to[i] = (int64_t)row[b / p.page_pos] * p.spage + (int64_t)(b % p.page_pos) * p.sp;
        }
        __syncthreads();
        for (int item = share; item < items; item += shares) {
            const int plane = item / blocks, column = (item - plane * blocks) * THREADS + threadIdx.x;
            if (column >= columns) continue;
            uint8_t* base = p.base + plane_offset(p, plane) + (int64_t)(column >> lanes_log2) * p.sh + (int64_t)(column & ((1 << lanes_log2) - 1)) * 16;
            for (int i = 0; i < m; i += 8) {
                uint4 x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (i + k < m && from[i + k] >= 0) x[k] = *reinterpret_cast<const uint4*>(base + from[i + k]);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (i + k < m && from[i + k] >= 0) *reinterpret_cast<uint4*>(base + to[i + k]) = x[k];
            }
        }
    }
}
__global__ void __launch_bounds__(kKeepThreads)
keep_move_kernel(PoolDev p, int lanes_log2, BookDev in, BookDev out, const int32_t* paths, const int32_t* n_path, int stride) {
    chain_next();
    copy_counts<kKeepThreads>(p, in, out, blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y);
    keep_move<kKeepThreads>(p, lanes_log2, in, paths, n_path, stride, blockIdx.x, blockIdx.y, gridDim.y);
}

// The new book: a block a row.
template <int THREADS>
__device__ __forceinline__ void keep_book(const PoolDev& p, const BookDev& in, const BookDev& out, const int32_t* paths, const int32_t* n_path, int stride, int s,
                                          uint32_t* status) {
    const int n = n_path[s], len = in.len[s];
    const bool ok = path_ok(p, in, paths + (long long)s * stride, n, stride, s, len);
    // a row that stays as it is keeps what it holds behind its length, too
    const long long now = (long long)len + n, keep = ok ? (now + p.page_pos - 1) / p.page_pos : in.max_pages;
    uint32_t bits = ok ? 0u : kStRange;
    for (int j = threadIdx.x; j < in.max_pages; j += THREADS) {
        const long long i = (long long)s * in.max_pages + j;
        const int page = in.table[i];
        if (page != -1 && !page_ok(p, page)) bits |= kStRange;
        out.table[i] = j < keep ? page : -1;
        if (j >= keep && page_ok(p, page)) atomicAdd(&out.ref[page], -1);
    }
    if (threadIdx.x == 0) out.len[s] = ok ? (int)now : len;
    if (bits) atomicOr(status, bits);
}
__global__ void __launch_bounds__(kKeepThreads)
keep_book_kernel(PoolDev p, BookDev in, BookDev out, const int32_t* paths, const int32_t* n_path, int stride, uint32_t* status) {
    chain_wait();
    keep_book<kKeepThreads>(p, in, out, paths, n_path, stride, blockIdx.x, status);
}
// One row.
constexpr int kKeepFewThreads = 512;
__global__ void __launch_bounds__(kKeepFewThreads)
keep_few_kernel(PoolDev p, int lanes_log2, BookDev in, BookDev out, const int32_t* paths, const int32_t* n_path, int stride, uint32_t* status) {
    copy_counts<kKeepFewThreads>(p, in, out, blockIdx.x, gridDim.x);
    keep_move<kKeepFewThreads>(p, lanes_log2, in, paths, n_path, stride, 0, blockIdx.x, gridDim.x);
    cluster_meet();
    if (blockIdx.x == 0) keep_book<kKeepFewThreads>(p, in, out, paths, n_path, stride, 0, status);
}

__device__ __forceinline__ void compact_plan(const PoolDev& p, const BookDev& in, const BookDev& out, int32_t* moved, const Workspace& w) {
    const int tid = threadIdx.x;
    unsigned long long live = 0, total;
    for (long long i = tid; i < p.n_pages; i += kPlanThreads) live += in.ref[i] > 0;
    block_scan(live, &live);
    unsigned long long done = 0;                   // holes in the low half, moves in the high half
    for (long long i0 = 0; i0 < p.n_pages; i0 += kPlanThreads) {
        const long long i = i0 + tid;
        const int ref = i < p.n_pages ? in.ref[i] : 0;
        const bool used = ref > 0, low = i < (long long)live, hole = low && !used, goes = used && !low;
        const unsigned long long at = done + block_scan((hole ? 1ull : 0ull) + (goes ? 1ull << 32 : 0ull), &total);
        if (hole) w.list[at & 0xffffffffu] = (int)i;
        if (goes) w.src[at >> 32] = (int)i;
        if (i < p.n_pages) {
            if (!goes) moved[i] = used ? (int)i : -1;
            out.ref[i] = low ? ref : 0;            // a hole's count is set below
        }
        done += total;
    }
    const int moves = (int)(done >> 32);
    __syncthreads();
    for (int c = tid; c < moves; c += kPlanThreads) {
        moved[w.src[c]] = w.list[c];
        out.ref[w.list[c]] = in.ref[w.src[c]];
    }
    if (tid == 0) w.head[0] = moves;
}
__global__ void __launch_bounds__(kPlanThreads)
compact_plan_kernel(PoolDev p, BookDev in, BookDev out, int32_t* moved, Workspace w) {
    chain_next();
    compact_plan(p, in, out, moved, w);
}

template <int THREADS>
__device__ __forceinline__ void compact_move(const PoolDev& p, const Mover& m, const BookDev& in, const BookDev& out, const int32_t* moved, const Workspace& w,
                                             uint32_t* status) {
    const long long step = (long long)gridDim.x * THREADS, t0 = (long long)blockIdx.x * THREADS + threadIdx.x;
    uint32_t bits = 0;
    for (long long i = t0; i < (long long)in.rows * in.max_pages; i += step) {
        const int page = in.table[i];
        if (page != -1 && !page_ok(p, page)) bits |= kStRange;
        out.table[i] = page_ok(p, page) ? moved[page] : -1;
    }
    for (long long i = t0; i < in.rows; i += step) out.len[i] = in.len[i];
    if (bits) atomicOr(status, bits);
    move_pages<THREADS>(p, m, w.head[0], w.src, nullptr, nullptr, w.list);
}
__global__ void __launch_bounds__(kMoveThreads)
compact_move_kernel(PoolDev p, Mover m, BookDev in, BookDev out, const int32_t* moved, Workspace w, uint32_t* status) {
    chain_wait();
    compact_move<kMoveThreads>(p, m, in, out, moved, w, status);
}
__global__ void __launch_bounds__(kFewThreads)
compact_few_kernel(PoolDev p, Mover m, BookDev in, BookDev out, int32_t* moved, Workspace w, uint32_t* status) {
    if (blockIdx.x == 0) compact_plan(p, in, out, moved, w);
    cluster_meet();
    compact_move<kFewThreads>(p, m, in, out, moved, w, status);
}

// One step, so that no bit that a call on another stream sets meanwhile is lost.
__global__ void take_status_kernel(uint32_t* status, uint32_t* bits) { *bits = atomicExch(status, 0u); }

Mover mover_of(const PoolDev& p) {
    Mover m;
    const int pieces = p.d * p.esz / 16;
    m.lanes_log2 = 0;
    while ((1 << m.lanes_log2) < pieces) ++m.lanes_log2;
    const int64_t a = p.sp < 0 ? -p.sp : p.sp, b = p.sh < 0 ? -p.sh : p.sh;
    m.slots_inner = a < b;
    return m;
}

// Blocks of the moving launch: enough for `moves` page moves and `words` table entries, at most eight an SM.
unsigned move_blocks(const PoolDev& p, long long moves, long long words) {
    const long long bytes = (long long)p.page_pos * p.H * p.d * p.esz;
    const long long parts = moves * 2 * p.L * ((bytes + kPartBytes - 1) / kPartBytes), tables = (words + kMoveThreads - 1) / kMoveThreads;
    const long long want = parts > tables ? parts : tables, most = 8LL * sm_count();
    return (unsigned)(want < 1 ? 1 : want > most ? most : want);
}

// Whether one cluster does a call, by the bytes that it may move at most and the words that it goes through.  A launch less saves the caller 1.7 us (fork of
// four beams, 16 KB: 15.3 -> 13.6 us a call; a path of 13 positions, 400 KB: 15.4 -> 13.7 us); eight SMs move whole pages slowly (compaction
// of 400 KB: 7.1 -> 14.8 us), paths, whose loads are all in flight at once, as fast as more.  Paths in this form are of one row: its blocks share a path's
// planes, and one of them writes the row's book.
constexpr long long kFewPageBytes = 1 << 17, kFewPathBytes = 1 << 20, kFewWords = 1 << 14;
long long plane_bytes(const PoolDev& p, long long positions) { return positions * p.H * p.d * p.esz * 2 * p.L; }

bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}
plc_status check_books(const plc_page_pool* pool, const plc_page_book* in, const plc_page_book* out, bool same_rows, PoolDev* p, BookDev* i,
                       BookDev* o) {
    plc_status rc = check_pool(pool, p);
    if (rc || (rc = check_book(in, i)) || (rc = check_book(out, o))) return rc;
    if (i->max_pages != o->max_pages || (same_rows && i->rows != o->rows)) return PLC_E_SHAPE;
    const uint64_t ti = 4ull * i->rows * i->max_pages, to = 4ull * o->rows * o->max_pages, n = 4ull * p->n_pages;
    if (overlap(i->table, ti, o->table, to) || overlap(i->len, 4ull * i->rows, o->len, 4ull * o->rows) || overlap(i->ref, n, o->ref, n))
        return PLC_E_INVALID;
    return PLC_OK;
}
plc_status check_workspace(const PoolDev& p, int rows_in, int rows_out, void* ws, uint64_t bytes) {
    if (!ws) return PLC_E_INVALID;
    if (!plc_aligned16(ws)) return PLC_E_ALIGN;
    return bytes < 4 * workspace_words(p.n_pages, rows_in, rows_out) ? PLC_E_CAPACITY : PLC_OK;
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" {

plc_status plc_take_status(uint32_t* status_dev, uint32_t* bits_dev, void* stream) {
    if (!status_dev || !bits_dev || status_dev == bits_dev) return PLC_E_INVALID;
    if ((reinterpret_cast<uintptr_t>(status_dev) | reinterpret_cast<uintptr_t>(bits_dev)) & 3) return PLC_E_ALIGN;
    if (launch_kernel(take_status_kernel, 1, 1, 0, static_cast<cudaStream_t>(stream), false, 1, status_dev, bits_dev) != cudaSuccess) return PLC_E_CUDA;
    count_launch(1);
    return PLC_OK;
}

plc_status plc_pages_workspace(int32_t n_pages, int32_t rows_in, int32_t rows_out, uint64_t* bytes) {
    if (n_pages < 1 || rows_in < 1 || rows_out < 1 || !bytes) return PLC_E_INVALID;
    *bytes = 4 * workspace_words(n_pages, rows_in, rows_out);
    return PLC_OK;
}

plc_status plc_pages_fork(const plc_page_pool* pool, const plc_page_book* in, const int32_t* parent_dev, const int32_t* room_dev,
                          const plc_page_book* out, void* workspace_dev, uint64_t workspace_bytes, uint32_t* status_dev, void* stream) {
    PoolDev p;
    BookDev i, o;
    plc_status rc = check_books(pool, in, out, false, &p, &i, &o);
    if (rc) return rc;
    if (!parent_dev || !status_dev) return PLC_E_INVALID;
    if ((rc = check_workspace(p, i.rows, o.rows, workspace_dev, workspace_bytes))) return rc;
    const Workspace w = workspace_at(workspace_dev, p.n_pages, i.rows, o.rows);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const long long words = (long long)(i.rows > o.rows ? i.rows : o.rows) * i.max_pages;
    if (plane_bytes(p, (long long)o.rows * p.page_pos) <= kFewPageBytes && words + p.n_pages <= kFewWords) {
        if (launch_kernel(fork_few_kernel, kFewBlocks, kFewThreads, 0, st, false, kFewBlocks, p, mover_of(p), i, o, parent_dev, room_dev, w, status_dev) != cudaSuccess)
            return PLC_E_CUDA;
        count_launch(1);
        return PLC_OK;
    }
    const unsigned counters = (unsigned)((p.n_pages + 4 * kPlanThreads - 1) / (4 * kPlanThreads));
    if (launch_kernel(fork_plan_kernel, 1 + (counters > 64 ? 64 : counters), kPlanThreads, 0, st, false, 1, p, i, o, parent_dev, room_dev, w, status_dev) !=
        cudaSuccess)
        return PLC_E_CUDA;
    if (launch_kernel(fork_move_kernel, move_blocks(p, o.rows, words), kMoveThreads, 0, st, true, 1, p, mover_of(p), i, o, parent_dev, room_dev, w,
                      status_dev) != cudaSuccess)
        return PLC_E_CUDA;
    count_launch(2);
    return PLC_OK;
}

plc_status plc_pages_keep(const plc_page_pool* pool, const plc_page_book* in, const int32_t* path_dev, const int32_t* n_path_dev, int32_t path_stride,
                          const plc_page_book* out, uint32_t* status_dev, void* stream) {
    PoolDev p;
    BookDev i, o;
    plc_status rc = check_books(pool, in, out, true, &p, &i, &o);
    if (rc) return rc;
    if (!path_dev || !n_path_dev || !status_dev || path_stride < 1) return PLC_E_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Mover m = mover_of(p);
    if (i.rows == 1 && plane_bytes(p, path_stride) <= kFewPathBytes && (long long)i.max_pages + p.n_pages <= kFewWords) {
        if (launch_kernel(keep_few_kernel, kFewBlocks, kKeepFewThreads, 0, st, false, kFewBlocks, p, m.lanes_log2, i, o, path_dev, n_path_dev, (int)path_stride,
                          status_dev) != cudaSuccess)
            return PLC_E_CUDA;
        count_launch(1);
        return PLC_OK;
    }
    const long long items = 2LL * p.L * (((p.H << m.lanes_log2) + kKeepThreads - 1) / kKeepThreads);
    long long split = (16LL * sm_count() + i.rows - 1) / i.rows;
    split = split > items ? items : split;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)i.rows, (unsigned)(split > 65535 ? 65535 : split));
    cfg.blockDim = dim3(kKeepThreads);
    cfg.stream = st;
    if (cudaLaunchKernelEx(&cfg, keep_move_kernel, p, m.lanes_log2, i, o, path_dev, n_path_dev, (int)path_stride) != cudaSuccess) return PLC_E_CUDA;
    if (launch_kernel(keep_book_kernel, (unsigned)i.rows, kKeepThreads, 0, st, true, 1, p, i, o, path_dev, n_path_dev, (int)path_stride, status_dev) !=
        cudaSuccess)
        return PLC_E_CUDA;
    count_launch(2);
    return PLC_OK;
}

plc_status plc_pages_compact(const plc_page_pool* pool, const plc_page_book* in, const plc_page_book* out, int32_t* moved_dev, void* workspace_dev,
                             uint64_t workspace_bytes, uint32_t* status_dev, void* stream) {
    PoolDev p;
    BookDev i, o;
    plc_status rc = check_books(pool, in, out, true, &p, &i, &o);
    if (rc) return rc;
    if (!moved_dev || !status_dev) return PLC_E_INVALID;
    if ((rc = check_workspace(p, i.rows, o.rows, workspace_dev, workspace_bytes))) return rc;
    const Workspace w = workspace_at(workspace_dev, p.n_pages, i.rows, o.rows);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (plane_bytes(p, (long long)p.n_pages / 2 * p.page_pos) <= kFewPageBytes && (long long)i.rows * i.max_pages + p.n_pages <= kFewWords) {
        if (launch_kernel(compact_few_kernel, kFewBlocks, kFewThreads, 0, st, false, kFewBlocks, p, mover_of(p), i, o, moved_dev, w, status_dev) != cudaSuccess)
            return PLC_E_CUDA;
        count_launch(1);
        return PLC_OK;
    }
    if (launch_kernel(compact_plan_kernel, 1, kPlanThreads, 0, st, false, 1, p, i, o, moved_dev, w) != cudaSuccess) return PLC_E_CUDA;
    if (launch_kernel(compact_move_kernel, move_blocks(p, p.n_pages, (long long)i.rows * i.max_pages), kMoveThreads, 0, st, true, 1, p, mover_of(p), i, o,
                      static_cast<const int32_t*>(moved_dev), w, status_dev) != cudaSuccess)
        return PLC_E_CUDA;
    count_launch(2);
    return PLC_OK;
}

}  // extern "C"
