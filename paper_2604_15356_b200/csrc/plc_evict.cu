// Eviction from the paged cache by accumulated attention weight (plc_pages_evict).
//
// A row that holds more than its budget keeps, in every layer and head by itself, the positions of the largest weights and its last ones; what is kept moves
// together in order, keys, values and weights alike, and the pages behind the new length are released.
//
// Two launches, three where books are large.  The first selects: a block a (row, layer, head) finds the weight of the last position that is kept by its bits, eight at a time from the
// top, and writes a bit for each position that is kept, and the kept weights; one block more decides, like the plan of a fork, which pages are fresh ones
// (a launch of its own where books are large).  The last moves the vectors in pieces and writes the new book.  A position never moves up, so that a row can stay in its pages: a piece's places hold one or two
// earlier pieces of the same row, and it is written once those have been read.
//
// HBM bound where much moves: 16 rows of up to 2048 positions, 8 layers of 8 heads of 128 in bf16, 1024 kept: 129 us on the device, 18 of them the selection (0.5 GB moved, 4.5 TB/s).
// One row of 1000 positions in 4 layers 18 us, both launches: chains of dependent loads.  What counted: nothing that every thread does once a piece (64-bit
// divisions by all: 170 us), a piece's word set before the wait for others and without a fence (123, 145), loops small enough that the selection's code is not what it
// waits for (29 us of selection unrolled, 18 rolled).
#include "plc_pages.cuh"

namespace plc {
namespace {

constexpr int kSelectThreads = 256, kSelectWarps = kSelectThreads / 32;
constexpr int kCopyThreads = 256, kMoveThreads = kCopyThreads + 64;      // that copy; and two warps that find out what comes next
constexpr int kPlanThreads = 1024;                // of a plan in a launch of its own
constexpr uint32_t kSpin = 1u << 22;

// Positions of a piece: as many vectors as 32 KB of shared memory hold, at most 128.
constexpr int piece_log2(int vector_bytes) { return vector_bytes <= 256 ? 7 : vector_bytes <= 512 ? 6 : 5; }

struct EvictHead {
    int32_t short_of;                             // the free pages do not suffice
    int32_t pad;
    unsigned long long ticket;                    // pieces that blocks have taken
};
struct EvictArgs {
    const float* weight; int64_t ws_row, ws_layer, ws_head; int n_pos;
    float* out;                                   // [rows][L][H][n_pos]
    const int32_t* budgets; int budget, recent;
    int piece_log2, pieces;                       // positions of a piece; pieces that n_pos has
    int held;                                     // positions of a row whose weights stay in shared memory while they are selected
    int planned;                                  // 1: a block of the selection makes the plan
    // workspace
    EvictHead* head;
    long long* first;                             // [rows + 1] pieces of the rows before
    int32_t* base;                                // [rows] index of the row's first fresh page in `list`; -1: the row stays as it is
    int32_t* count;                               // [rows] its fresh pages
    int32_t* list;                                // [n_pages]
    int32_t* rank;                                // [rows][row_pages] the how-manieth fresh page of its row a new page is, -1: the row's own
    int row_pages;                                // pages that n_pos positions fill
    uint32_t* kept;                               // [rows][L][H][pieces][positions of a piece / 32] a bit a position
    int32_t* ahead;                               // [rows][L][H][pieces] positions kept before the piece
    uint32_t* read;                               // [rows][L][H][pieces][2] a piece's keys, values have been read
};

// What becomes of a row.
struct EvictRow { int len, now; bool goes, bad; };
__device__ __forceinline__ EvictRow evict_row(const PoolDev& p, const BookDev& in, const EvictArgs& a, int s) {
    EvictRow r;
    const int budget = a.budgets ? a.budgets[s] : a.budget;
    r.len = in.len[s];
    r.bad = r.len < 0 || r.len > most_positions(in, p) || (budget >= 0 && r.len > budget && r.len > a.n_pos);
    r.goes = !r.bad && budget >= 0 && r.len > budget;
    r.now = r.goes ? budget : r.len;
    return r;
}
__device__ __forceinline__ bool page_ok(const PoolDev& p, int page) { return page >= 0 && page < p.n_pages; }
__device__ __forceinline__ int pages_for(const PoolDev& p, int n) { return (int)(((long long)n + p.page_pos - 1) / p.page_pos); }

// Order of the weights as unsigned numbers; NaN is lightest, -0 is +0.
__device__ __forceinline__ uint32_t weight_order(float w) {
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// Sum over the block's threads before this one; *total: over all.
template <int THREADS> __device__ __forceinline__ long long sum_before(long long v, long long* total) {
    __shared__ long long part[THREADS / 32];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(kFull, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                              // the sums before have been read
    if (lane == 31) part[wid] = x;
    __syncthreads();
    long long before = x - v, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < wid) before += part[w];
        all += part[w];
    }
    *total = all;
    return before;
}

// How many of row s's new pages others hold, which makes them fresh ones: -1 where the row stays, kOutOfRange where a page of its does not exist.  A block calls it, which also
// writes down which they are.
constexpr int kOutOfRange = 1 << 30;
__device__ __forceinline__ void count_fresh(const PoolDev& p, const BookDev& in, const EvictArgs& a, int s, const EvictRow& r, bool good) {
    const int keep = good ? pages_for(p, r.now) : 0;
    long long before = 0, some;
    for (int j0 = 0; j0 < keep; j0 += kSelectThreads) {
        const int j = j0 + threadIdx.x;
        const bool shared = j < keep && in.ref[in.table[(int64_t)s * in.max_pages + j]] != 1;
        const long long at = before + sum_before<kSelectThreads>(shared, &some);
        if (j < keep) a.rank[(int64_t)s * a.row_pages + j] = shared ? (int)at : -1;
        before += some;
    }
    if (!a.planned && threadIdx.x == 0) a.count[s] = !r.goes ? -1 : good ? (int)before : kOutOfRange;
}

// One block: how many fresh pages each row needs (where the rows' own blocks have not counted them) and which, and how many pieces there are to move.
template <int THREADS>
__device__ __forceinline__ void evict_plan(const PoolDev& p, const BookDev& in, const EvictArgs& a, uint32_t* status) {
    const int tid = threadIdx.x;
    uint32_t bits = 0;
    if (a.planned) {
        for (int s = tid; s < in.rows; s += THREADS) {
            const EvictRow r = evict_row(p, in, a, s);
            a.base[s] = r.goes ? pages_for(p, r.len) : -1;               // pages that the row holds, for now
            a.count[s] = r.goes ? 0 : -1;
        }
        __syncthreads();
        const int entries = in.rows * in.max_pages;
#pragma unroll 2
        for (int e = tid; e < entries; e += THREADS) {
            const int row = e / in.max_pages, at = e - row * in.max_pages, page = in.table[e], holds = a.base[row];
            if (at >= holds) continue;
            if (!page_ok(p, page)) atomicOr(&a.count[row], kOutOfRange);
            else if (in.ref[page] != 1 && at < pages_for(p, evict_row(p, in, a, row).now)) atomicAdd(&a.count[row], 1);
        }
        __syncthreads();
    }
    long long need = 0, moves = 0;
    for (int s0 = 0; s0 < in.rows; s0 += THREADS) {
        const int s = s0 + tid;
        int count = s < in.rows ? __ldcg(&a.count[s]) : -1;
        const EvictRow r = s < in.rows ? evict_row(p, in, a, s) : EvictRow{};
        if (r.bad || count >= kOutOfRange) { bits |= kStRange; count = -1; }
        const long long pieces = count >= 0 ? (long long)((r.len + (1 << a.piece_log2) - 1) >> a.piece_log2) * p.L * p.H * 2 : 0;
        long long total;
        const long long at = need + sum_before<THREADS>(count >= 0 ? count : 0, &total);
        need += total;
        const long long first = moves + sum_before<THREADS>(pieces, &total);
        moves += total;
        if (s < in.rows) {
            a.base[s] = count >= 0 ? (int)min(at, 0x7fffffffll) : -1;
            a.count[s] = count;
            a.first[s] = first;
        }
    }
    constexpr int EACH = 8;                       // pages of a thread at a time
    long long found = 0;
    for (long long i0 = 0; i0 < p.n_pages && found < need; i0 += EACH * THREADS) {
        const long long i = i0 + EACH * tid;
        uint32_t free = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (i + k < p.n_pages && in.ref[i + k] == 0) free |= 1u << k;
        long long total;
        long long at = found + sum_before<THREADS>(__popc(free), &total);
        for (; free && at < need; free &= free - 1) a.list[at++] = (int)i + __ffs(free) - 1;
        found += total;
    }
    const bool short_of = found < need;
    if (short_of) bits |= kStCapacity;
    if (bits) atomicOr(status, bits);
    if (tid == 0) {
        a.head->short_of = short_of;
        a.head->ticket = 0;
        a.first[in.rows] = short_of ? 0 : moves;
    }
}
__global__ void __launch_bounds__(kPlanThreads) evict_plan_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev in, const __grid_constant__ EvictArgs a,
                                                                  uint32_t* status) {
    chain_next();
    chain_wait();
    evict_plan<kPlanThreads>(p, in, a, status);
}

__device__ __forceinline__ void copy_weights(const float* w, float* out, int n, int n_pos) {
    for (int t = threadIdx.x; t < n_pos; t += blockDim.x) out[t] = t < n ? w[t] : 0.f;
}

struct SelectShared {
    alignas(16) int bins[256];                    // counted by ints, read by int4
    int above[kSelectWarps], equal[kSelectWarps];
    uint32_t prefix;
    int want;
};

// The loops are kept small: a block goes through each of them few times, and code that comes from memory for the first time costs more than it does.
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev in, const __grid_constant__ BookDev out,
                                                                      const __grid_constant__ EvictArgs a, uint32_t* status) {
    extern __shared__ uint32_t key_s[];           // of a short row's weights
    __shared__ SelectShared sh;
    chain_next();
    if ((int)blockIdx.x < a.planned) { evict_plan<kSelectThreads>(p, in, a, status); return; }
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int lane_at = blockIdx.x - a.planned, h = lane_at % p.H, l = lane_at / p.H % p.L, s = lane_at / p.H / p.L;
    const float* w = a.weight + (int64_t)s * a.ws_row + (int64_t)l * a.ws_layer + (int64_t)h * a.ws_head;
    float* to = a.out + (int64_t)lane_at * a.n_pos;
    // the weights are on their way before the row's length is known
#pragma unroll 4
    for (int t = tid; t < a.held; t += kSelectThreads) key_s[t] = weight_order(w[t]);
    for (long long i = (long long)lane_at * kSelectThreads + tid; i < p.n_pages; i += (long long)(gridDim.x - a.planned) * kSelectThreads) out.ref[i] = in.ref[i];
    const EvictRow r = evict_row(p, in, a, s);
    bool good = r.goes;
    if (good)
        for (int j = tid; j < pages_for(p, r.len); j += kSelectThreads) good = good && page_ok(p, in.table[(int64_t)s * in.max_pages + j]);
    good = __syncthreads_and(good);
    if (l == 0 && h == 0) count_fresh(p, in, a, s, r, good);              // a block of the row
    if (!good) {
        copy_weights(w, to, min(max(r.len, 0), a.n_pos), a.n_pos);
        return;
    }
    const int n = r.len - min(a.recent, r.now);                          // candidates; what stands behind them is kept
    int want = r.now - (r.len - n);                                      // of the candidates
    const bool held = r.len <= a.held;
    const int pieces = (r.len + (1 << a.piece_log2) - 1) >> a.piece_log2;
    uint32_t* read = a.read + (int64_t)lane_at * a.pieces * 2;
    for (int c = tid; c < 2 * pieces; c += kSelectThreads) read[c] = 0;
    auto key = [&](int t) { return held ? key_s[t] : weight_order(w[t]); };
    // the want-th largest key among the candidates, eight bits at a time from the top
    uint32_t last = 0;
#pragma unroll 1
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        sh.bins[tid] = 0;
        __syncthreads();
        const uint32_t above = shift == 24 ? 0u : ~0u << (shift + 8);
#pragma unroll 2
        for (int t = tid; t < n; t += kSelectThreads) {
            const uint32_t k = key(t);
            if ((k & above) == last) atomicAdd(&sh.bins[k >> shift & 255], 1);
        }
        __syncthreads();
        if (wid == 0) {                                                  // the bin that the want-th falls into
            const int4 b0 = *reinterpret_cast<const int4*>(sh.bins + 8 * (31 - lane)), b1 = *reinterpret_cast<const int4*>(sh.bins + 8 * (31 - lane) + 4);
            const int sum = b0.x + b0.y + b0.z + b0.w + b1.x + b1.y + b1.z + b1.w;
            int upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(kFull, upto, o);
                if (lane >= o) upto += v;
            }
            if (upto >= want && upto - sum < want) {
                int left = want - (upto - sum), i = 8 * (31 - lane) + 7;
                while (left > sh.bins[i]) left -= sh.bins[i--];
                sh.prefix = last | (uint32_t)i << shift;
                sh.want = left;
            }
        }
        __syncthreads();
        last = sh.prefix;
        want = sh.want;
    }
    const bool nothing = want == 0;
    // kept: what is above `last`, the first `want` that equal it, and what stands behind the candidates.  A warp takes a run of groups of 32 positions; first
    // how many it keeps, then where they go.
    auto is_above = [&](uint32_t k, int t) { return __ballot_sync(kFull, t < n ? !nothing && k > last : t < r.len); };
    auto is_equal = [&](uint32_t k, int t) { return __ballot_sync(kFull, t < n && !nothing && k == last); };
    const int groups = (r.len + 31) / 32, each = (groups + kSelectWarps - 1) / kSelectWarps, g0 = wid * each, g1 = min(g0 + each, groups);
    int above = 0, equal = 0;
#pragma unroll 2
    for (int g = g0; g < g1; ++g) {
        const int t = g * 32 + lane;
        const uint32_t k = t < n ? key(t) : 0u;
        above += __popc(is_above(k, t));
        equal += __popc(is_equal(k, t));
    }
    if (lane == 0) { sh.above[wid] = above; sh.equal[wid] = equal; }
    __syncthreads();
    int at = 0, ties = 0;
    for (int v = 0; v < wid; ++v) { at += sh.above[v]; ties += sh.equal[v]; }
    const int words_log2 = a.piece_log2 - 5, words = 1 << words_log2;
    uint32_t* kept = a.kept + ((int64_t)lane_at * a.pieces << words_log2);
    int32_t* ahead = a.ahead + (int64_t)lane_at * a.pieces;
    const uint32_t lt = lanemask_lt();
#pragma unroll 2
    for (int g = g0; g < g1; ++g) {
        const int t = g * 32 + lane;
        const float x = t < r.len ? w[t] : 0.f;
        const uint32_t k = t < n ? key(t) : 0u, up = is_above(k, t), eq = is_equal(k, t);
        const uint32_t m = up | __ballot_sync(kFull, (eq >> lane & 1u) && ties + __popc(eq & lt) < want);
        const int here = at + min(ties, want);
        if (m >> lane & 1u) to[here + __popc(m & lt)] = x;
        if (lane == 0) {
            kept[g] = m;
            if ((g & (words - 1)) == 0) ahead[g >> words_log2] = here;
        }
        at += __popc(up);
        ties += __popc(eq);
    }
    // words of the last piece that no position reaches
    for (int c = groups + tid; c < pieces << words_log2; c += kSelectThreads) kept[c] = 0;
    for (int t = r.now + tid; t < a.n_pos; t += kSelectThreads) to[t] = 0.f;
}

// The row's new pages: its own where nobody else holds them, else fresh ones.
__device__ __forceinline__ void evict_book(const PoolDev& p, const BookDev& in, const BookDev& out, const EvictArgs& a, int s, uint32_t* status) {
    const int lane = threadIdx.x & 31;                                   // a warp calls it
    const bool goes = a.base[s] >= 0 && !a.head->short_of;
    const int len = in.len[s], now = goes ? evict_row(p, in, a, s).now : len, keep = goes ? pages_for(p, now) : in.max_pages;
    uint32_t bits = 0;
    for (int j = lane; j < in.max_pages; j += 32) {
        const int64_t i = (int64_t)s * in.max_pages + j;
        const int page = in.table[i], rank = goes && j < keep ? a.rank[(int64_t)s * a.row_pages + j] : -1;
        if (page != -1 && !page_ok(p, page)) bits |= kStRange;
        if (goes && page_ok(p, page) && (rank >= 0 || j >= keep)) atomicAdd(&out.ref[page], -1);
        const int now_at = rank >= 0 ? a.list[a.base[s] + rank] : page;
        if (rank >= 0) out.ref[now_at] = 1;                              // it was free, and this row alone has it
        out.table[i] = j < keep ? now_at : -1;
    }
    if (lane == 0) out.len[s] = now;
    if (bits) atomicOr(status, bits);
}

// The row that a piece belongs to: the last one that begins at or before it.  A warp calls it.
__device__ __forceinline__ int row_of(const long long* first, int rows, long long item) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = rows;
    for (;;) {
        const int step = (hi - lo + 31) / 32, most = (hi - lo - 1) / step, at = lo + min(lane, most) * step;
        const int j = min(31 - __clz(__ballot_sync(kFull, first[at] <= item)), most);
        lo += j * step;
        hi = min(hi, lo + step);
        if (step == 1) return lo;
    }
}

// A piece that a block has taken: its row (-1: there are no more) and its number in it.
struct Taken { long long rest; int s; };
// A piece of a row's keys or values of one head, with which of its positions are kept.
struct Piece {
    uint8_t* plane;
    uint32_t* read;                               // its row's first piece's word
    int s, c, first, n;                           // row (-1: there are no more), piece; where the first that is kept goes; how many are
    uint32_t kept[4];
    int before[4];
};

// Moves the pieces.  A block takes them in order, a row's piece of all layers and heads before its next: it reads what is kept of a piece into shared memory, says so, and writes
// once the one or two pieces whose places it writes over have been read; those are earlier ones, taken by blocks that run.
__global__ void __launch_bounds__(kMoveThreads, 6) evict_move_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev in, const __grid_constant__ BookDev out,
                                                                  const __grid_constant__ EvictArgs a, int lanes_log2, uint32_t* status) {
    extern __shared__ uint4 held[];
    __shared__ int64_t src_s[2][128], dst_s[2][128];
    __shared__ Piece piece_s[2];
    __shared__ Taken taken_s[2];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    chain_wait();
    const long long total = a.first[in.rows], lanes = (long long)p.L * p.H;
    if (a.head->short_of)                                                // the weights stay as they are, too
        for (long long at = blockIdx.x; at < lanes * in.rows; at += gridDim.x) {
            const int h = (int)(at % p.H), l = (int)(at / p.H % p.L), s = (int)(at / p.H / p.L);
            if (a.base[s] >= 0)
                copy_weights(a.weight + (int64_t)s * a.ws_row + (int64_t)l * a.ws_layer + (int64_t)h * a.ws_head, a.out + at * a.n_pos, in.len[s], a.n_pos);
        }
    const uint32_t held_at = (uint32_t)__cvta_generic_to_shared(held);
    const int mask = (1 << lanes_log2) - 1, words = 1 << (a.piece_log2 - 5);
    // What comes next is found in two steps, each by a warp of its own and a piece ahead of the other: its number and row, then what is kept of it.
    auto tickets = [&](int n) { return (long long)__shfl_sync(kFull, lane == 0 ? atomicAdd(&a.head->ticket, (unsigned long long)n) : 0ull, 0); };
    auto take = [&](Taken& x, long long item) {
        const int s = item < total ? row_of(a.first, in.rows, item) : -1;
        if (lane == 0) { x.s = s; x.rest = s < 0 ? 0 : item - a.first[s]; }
    };
    auto enter = [&](const Taken& t, Piece& x) {
        if (t.s < 0) {
            if (lane == 0) x.s = -1;
            return;
        }
        long long c;
        int of_row;                               // layer and head
        if (t.rest <= 0x7fffffffll && lanes <= 0x3fffffffll) {
            c = (int)t.rest / (int)(2 * lanes);
            of_row = ((int)t.rest - (int)(2 * lanes) * (int)c) >> 1;
        } else {
            c = t.rest / (2 * lanes);
            of_row = (int)((t.rest - 2 * lanes * c) / 2);
        }
        const long long at = (long long)t.s * lanes + of_row;
        const uint32_t kept = lane < words ? a.kept[(at * a.pieces + c) * words + lane] : 0u;
        const int first = a.ahead[at * a.pieces + c], l = of_row / p.H, h = of_row - l * p.H, kv = (int)(t.rest & 1), mine = __popc(kept);
        int before = 0, n = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int m = __shfl_sync(kFull, mine, v);
            before += v < lane ? m : 0;
            n += m;
        }
        if (lane < 4) { x.kept[lane] = kept; x.before[lane] = before; }
        if (lane == 0) {
            x.s = t.s;
            x.c = (int)c;
            x.first = first;
            x.n = n;
            x.plane = p.base + (int64_t)l * p.sl + (int64_t)kv * p.skv + (int64_t)h * p.sh;
            x.read = a.read + at * a.pieces * 2 + kv;
        }
    };
    constexpr int taker = kCopyThreads / 32, enterer = taker + 1;
    if (wid == taker) {
        const long long item = tickets(2);
        take(taken_s[0], item);
        take(taken_s[1], item + 1);
    } else                                        // the others write the book meanwhile
        for (int s = blockIdx.x * (kCopyThreads / 32) + wid; s < in.rows && wid < taker; s += gridDim.x * (kCopyThreads / 32)) evict_book(p, in, out, a, s, status);
    __syncthreads();
    if (wid == enterer) enter(taken_s[0], piece_s[0]);
    __syncthreads();
    for (int turn = 0; piece_s[turn].s >= 0; turn ^= 1) {
        const Piece& x = piece_s[turn];
        const int32_t* table = in.table + (int64_t)x.s * in.max_pages;
        int64_t *src = src_s[turn], *dst = dst_s[turn];
        const bool fresh = a.count[x.s] > 0;
        if (wid < words) {
            const uint32_t m = x.kept[wid];
            if (m >> lane & 1u) {
                const int i = x.before[wid] + __popc(m & lanemask_lt()), t = (x.c << a.piece_log2) + tid, to = x.first + i, from_page = t / p.page_pos, j = to / p.page_pos;
                const int rank = fresh ? a.rank[(int64_t)x.s * a.row_pages + j] : -1, mine = rank >= 0 ? a.list[a.base[x.s] + rank] : table[j];
                src[i] = (int64_t)table[from_page] * p.spage + (int64_t)(t - from_page * p.page_pos) * p.sp;
                dst[i] = (int64_t)mine * p.spage + (int64_t)(to - j * p.page_pos) * p.sp;
            }
        }
        __syncthreads();
        const int units = wid < taker ? x.n << lanes_log2 : 0;
        uint8_t* plane = x.plane;
#pragma unroll 2
        for (int u = tid; u < units; u += kCopyThreads) {
            const int64_t from = src[u >> lanes_log2];
            if (from != dst[u >> lanes_log2])
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(held_at + u * 16), "l"(plane + from + (u & mask) * 16) : "memory");
        }
        if (wid == taker) take(taken_s[turn], tickets(1));
        if (wid == enterer) enter(taken_s[turn ^ 1], piece_s[turn ^ 1]);
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        // The copies have arrived, so that nothing can change what they brought: the word needs no fence before it (which, behind the block's writes, took 4500
        // clocks), and who sees it writes behind a barrier.
        if (tid == enterer * 32) asm volatile("st.relaxed.gpu.global.u32 [%0], %1;" ::"l"(x.read + 2 * x.c), "r"(1u) : "memory");
        // have the pieces been read that this one is written over?
        bool ok = true;
        if (wid < 2 && lane == 0 && x.n > 0) {
            const int other = (wid == 0 ? x.first : x.first + x.n - 1) >> a.piece_log2;
            if (other < x.c) {
                uint32_t done = 0;
                for (uint32_t k = 0; k < kSpin && !done; ++k) asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(done) : "l"(x.read + 2 * other) : "memory");
                ok = done != 0;
                if (!ok) atomicOr(status, kStTimeout);
            }
        }
        if (!__syncthreads_and(ok)) continue;
#pragma unroll 2
        for (int u = tid; u < units; u += kCopyThreads) {
            const int64_t to = dst[u >> lanes_log2];
            if (src[u >> lanes_log2] != to) *reinterpret_cast<uint4*>(plane + to + (u & mask) * 16) = held[u];
        }
    }
}

struct EvictLayout { uint64_t first, base, count, list, rank, kept, ahead, read, bytes; };
uint64_t row_pages(const PoolDev& p, int n_pos) { return ((uint64_t)n_pos + p.page_pos - 1) / p.page_pos; }
EvictLayout layout_of(const PoolDev& p, long long rows, int n_pos) {
    const uint64_t piece = 1u << piece_log2(p.d * p.esz), pieces = ((uint64_t)n_pos + piece - 1) / piece, lanes = (uint64_t)rows * p.L * p.H;
    EvictLayout x;
    x.first = sizeof(EvictHead);
    x.base = x.first + 8 * (rows + 1);
    x.count = x.base + 4 * rows;
    x.list = x.count + 4 * rows;
    x.rank = x.list + 4ull * p.n_pages;
    x.kept = x.rank + 4 * rows * row_pages(p, n_pos);
    x.ahead = x.kept + lanes * pieces * (piece / 32) * 4;
    x.read = x.ahead + lanes * pieces * 4;
    x.bytes = x.read + lanes * pieces * 8;
    return x;
}
plc_status check_lanes(const PoolDev& p, long long rows, int n_pos) {
    if (n_pos < 1) return PLC_E_INVALID;
    return rows * p.L * p.H > 0x3fffffffll || n_pos > kMostPositions ? PLC_E_SHAPE : PLC_OK;
}
bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}
// Whether the kept weights lie between the first and the last of the old ones, or across either end: other blocks still read those while they are written.
bool among(const PoolDev& p, int rows, const plc_weights& w, const float* out) {
    __int128 lo = 0, hi = w.n_pos;                // elements from the base
    const __int128 reach[3] = {(__int128)(rows - 1) * w.stride_row, (__int128)(p.L - 1) * w.stride_layer, (__int128)(p.H - 1) * w.stride_head};
    for (const __int128 r : reach) (r < 0 ? lo : hi) += r;
    const __int128 base = (__int128)reinterpret_cast<uintptr_t>(w.base_dev), to = (__int128)reinterpret_cast<uintptr_t>(out);
    return to < base + 4 * hi && base + 4 * lo < to + (__int128)4 * rows * p.L * p.H * w.n_pos;
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" {

plc_status plc_pages_evict_workspace(const plc_page_pool* pool, int32_t rows, int32_t n_pos, uint64_t* bytes) {
    PoolDev p;
    plc_status rc = check_pool(pool, &p);
    if (rc) return rc;
    if (rows < 1 || !bytes) return PLC_E_INVALID;
    if (rows > (1 << 20)) return PLC_E_SHAPE;
    if ((rc = check_lanes(p, rows, n_pos))) return rc;
    *bytes = layout_of(p, rows, n_pos).bytes;
    return PLC_OK;
}

plc_status plc_pages_evict(const plc_page_pool* pool, const plc_page_book* in, const plc_weights* weights, const int32_t* budget_dev, int32_t budget, int32_t recent,
                           const plc_page_book* out, float* out_weights_dev, void* workspace_dev, uint64_t workspace_bytes, uint32_t* status_dev, void* stream) {
    PoolDev p;
    BookDev i, o;
    plc_status rc = check_pool(pool, &p);
    if (rc || (rc = check_book(in, &i)) || (rc = check_book(out, &o))) return rc;
    if (i.max_pages != o.max_pages || i.rows != o.rows) return PLC_E_SHAPE;
    if (!weights || !weights->base_dev || !out_weights_dev || !workspace_dev || !status_dev || recent < 0 || (!budget_dev && budget < 0)) return PLC_E_INVALID;
    if ((rc = check_lanes(p, i.rows, weights->n_pos))) return rc;
    if (!plc_aligned16(workspace_dev) || ((reinterpret_cast<uintptr_t>(weights->base_dev) | reinterpret_cast<uintptr_t>(out_weights_dev)) & 3)) return PLC_E_ALIGN;
    const uint64_t t = 4ull * i.rows * i.max_pages, n = 4ull * p.n_pages;
    if (overlap(i.table, t, o.table, t) || overlap(i.len, 4ull * i.rows, o.len, 4ull * i.rows) || overlap(i.ref, n, o.ref, n)) return PLC_E_INVALID;
    if (among(p, i.rows, *weights, out_weights_dev)) return PLC_E_INVALID;
    const EvictLayout x = layout_of(p, i.rows, weights->n_pos);
    if (workspace_bytes < x.bytes) return PLC_E_CAPACITY;
    const long long lanes = (long long)i.rows * p.L * p.H;
    uint8_t* ws = static_cast<uint8_t*>(workspace_dev);
    const int log2 = piece_log2(p.d * p.esz), piece = 1 << log2;
    // Weights in shared memory: rows of up to 8192, as long as there is room for (49152) where few blocks run anyway (five rows of up to 13423 positions in 4 heads: 68 us without, 59 with).
    const int most_held = lanes <= 4 * sm_count() ? 49152 : 8192, held = weights->n_pos < most_held ? weights->n_pos : most_held;
    // The plan is a block of the selection where it has little to look at, else a launch of its own, and the rows' blocks count their pages (31 rows of 4176 pages of one
    // position: 308 us in the selection, 116 so; where 16 rows have 65 pages each a launch more costs 2 us).
    const bool apart = (long long)i.rows * i.max_pages > 16384;
    const EvictArgs a{weights->base_dev, weights->stride_row, weights->stride_layer, weights->stride_head, weights->n_pos, out_weights_dev, budget_dev, budget, recent,
                      log2, (int)(((long long)weights->n_pos + piece - 1) / piece), held, apart ? 0 : 1, reinterpret_cast<EvictHead*>(ws),
                      reinterpret_cast<long long*>(ws + x.first), reinterpret_cast<int32_t*>(ws + x.base), reinterpret_cast<int32_t*>(ws + x.count),
                      reinterpret_cast<int32_t*>(ws + x.list), reinterpret_cast<int32_t*>(ws + x.rank), (int)row_pages(p, weights->n_pos),
                      reinterpret_cast<uint32_t*>(ws + x.kept), reinterpret_cast<int32_t*>(ws + x.ahead), reinterpret_cast<uint32_t*>(ws + x.read)};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int lanes_log2 = 0;
    while ((16 << lanes_log2) < p.d * p.esz) ++lanes_log2;
    if (held * 4 > 40 * 1024 && cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 49152 * 4) != cudaSuccess) return PLC_E_CUDA;
    if (launch_kernel(evict_select_kernel, (unsigned)(a.planned + lanes), kSelectThreads, (size_t)held * 4, st, false, 1, p, i, o, a, status_dev) != cudaSuccess) return PLC_E_CUDA;
    if (apart && launch_kernel(evict_plan_kernel, 1, kPlanThreads, 0, st, true, 1, p, i, a, status_dev) != cudaSuccess) return PLC_E_CUDA;
    // as many blocks as run at once (six of 32 KB an SM), or as the pieces that full rows would have
    const long long most = 6ll * sm_count(), want = 2 * lanes * a.pieces;
    if (launch_kernel(evict_move_kernel, (unsigned)(want < most ? want : most), kMoveThreads, (size_t)piece * p.d * p.esz, st, true, 1, p, i, o, a, lanes_log2, status_dev) != cudaSuccess)
        return PLC_E_CUDA;
    count_launch(apart ? 3 : 2);
    return PLC_OK;
}

}  // extern "C"
