// Eviction from the paged cache by accumulated attention weight (plc_pages_evict).
//
// A row that holds more than its budget keeps, in every layer and head by itself, the positions of the largest weights and its last ones; what is kept moves
// together in order, keys, values and weights alike, and the pages behind the new length are released.
//
// Two launches.  The first selects: a block a (row, layer, head) finds the weight of the last position that is kept by its bits, eight at a time from the
// top, writes a bit for each position that is kept, and the kept weights; one block more decides, like the plan of a fork, which pages are fresh ones.  The
// second moves the vectors and writes the new book.  A position never moves up, and a block that takes a (row, layer, head, keys or values) reads each
// piece of it before it writes, so it can stay in its pages.
#include <math.h>

#include "plc_pages.cuh"

namespace plc {
namespace {

constexpr int kSelectThreads = 256, kMoveThreads = 256;
constexpr int kPiecePos = 128;                    // positions of a piece, four words of kept bits

struct EvictArgs {
    const float* weight; int64_t ws_row, ws_layer, ws_head; int n_pos;
    float* out;                                   // [rows][L][H][n_pos]
    const int32_t* budgets; int budget, recent;
    // workspace
    int32_t* head;                                // [4]: 1 where the free pages do not suffice
    int32_t* base;                                // [rows] index of the row's first fresh page in `list`; -1: the row stays as it is
    int32_t* list;                                // [n_pages]
    uint32_t* kept;                               // [rows][L][H][pieces][4] a bit a position
    int32_t* ahead;                               // [rows][L][H][pieces] positions kept before the piece
    int pieces;
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

// Order of the weights as unsigned numbers; NaN is lightest, -0 is +0.
__device__ __forceinline__ uint32_t weight_order(float w) {
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// One block: which rows go, how many fresh pages they need and which.
__device__ __forceinline__ void evict_plan(const PoolDev& p, const BookDev& in, const EvictArgs& a, uint32_t* status) {
    __shared__ long long sums[kSelectThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    long long need = 0;
    uint32_t bits = 0;
    for (int s0 = 0; s0 < in.rows; s0 += kSelectThreads / 32) {       // a warp a row
        const int s = s0 + wid;
        int mine = 0;
        bool ok = false;
        if (s < in.rows) {
            const EvictRow r = evict_row(p, in, a, s);
            if (r.bad) bits |= kStRange;
            ok = r.goes;
            if (ok) {
                const int held = (r.len + p.page_pos - 1) / p.page_pos, keep = (r.now + p.page_pos - 1) / p.page_pos;
                bool good = true;
                for (int j = lane; j < held; j += 32) {
                    const int page = in.table[(int64_t)s * in.max_pages + j];
                    if (!page_ok(p, page)) good = false;
                    else if (j < keep && in.ref[page] != 1) ++mine;
                }
                ok = __all_sync(kFull, good);
                if (!ok) bits |= kStRange;
                mine = ok ? __reduce_add_sync(kFull, mine) : 0;
            }
        }
        __syncthreads();
        if (lane == 0) sums[wid] = mine;
        __syncthreads();
        long long at = need;
        for (int w = 0; w < kSelectThreads / 32; ++w) {
            if (w < wid) at += sums[w];
            need += sums[w];
        }
        if (s < in.rows && lane == 0) a.base[s] = ok ? (int)min(at, 0x7fffffffll) : -1;
    }
    __syncthreads();
    long long found = 0;
    for (long long i0 = 0; i0 < p.n_pages && found < need; i0 += kSelectThreads) {
        const long long i = i0 + tid;
        const bool free = i < p.n_pages && in.ref[i] == 0;
        const uint32_t m = __ballot_sync(kFull, free);
        __syncthreads();
        if (lane == 0) sums[wid] = __popc(m);
        __syncthreads();
        long long at = found + __popc(m & lanemask_lt());
        for (int w = 0; w < kSelectThreads / 32; ++w) {
            if (w < wid) at += sums[w];
            found += sums[w];
        }
        if (free && at < need) a.list[at] = (int)i;
    }
    if (found < need) bits |= kStCapacity;
    if (bits) atomicOr(status, bits);
    if (tid == 0) a.head[0] = found < need;
}

__device__ __forceinline__ void copy_weights(const float* w, float* out, int n, int n_pos) {
    for (int t = threadIdx.x; t < n_pos; t += blockDim.x) out[t] = t < n ? w[t] : 0.f;
}

__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev in, const __grid_constant__ BookDev out,
                                                                      const __grid_constant__ EvictArgs a, uint32_t* status) {
    chain_next();
    if (blockIdx.x == 0) { evict_plan(p, in, a, status); return; }
    __shared__ int bins[256];
    __shared__ int warp_above[8], warp_equal[8], warp_recent[8];
    __shared__ uint32_t prefix_s;
    __shared__ int want_s;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const long long lane_at = blockIdx.x - 1;
    for (long long i = lane_at * kSelectThreads + tid; i < p.n_pages; i += (long long)(gridDim.x - 1) * kSelectThreads) out.ref[i] = in.ref[i];
    const int h = (int)(lane_at % p.H), l = (int)(lane_at / p.H % p.L), s = (int)(lane_at / p.H / p.L);
    const EvictRow r = evict_row(p, in, a, s);
    const float* w = a.weight + (int64_t)s * a.ws_row + (int64_t)l * a.ws_layer + (int64_t)h * a.ws_head;
    float* to = a.out + lane_at * a.n_pos;
    bool good = r.goes;
    if (good)
        for (int j = tid; j < (r.len + p.page_pos - 1) / p.page_pos; j += kSelectThreads) good = good && page_ok(p, in.table[(int64_t)s * in.max_pages + j]);
    if (!__syncthreads_and(good)) {
        copy_weights(w, to, min(max(r.len, 0), a.n_pos), a.n_pos);
        return;
    }
    const int n = r.len - min(a.recent, r.now);                          // candidates; what stands behind them is kept
    int want = r.now - (r.len - n);
    // the want-th largest key among the candidates, eight bits at a time
    uint32_t prefix = 0;
    bool all = want == 0;                                                // nothing of them is kept
    for (int shift = 24; shift >= 0 && !all; shift -= 8) {
        bins[tid] = 0;
        __syncthreads();
        for (int t = tid; t < n; t += kSelectThreads) {
            const uint32_t k = weight_order(w[t]);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&bins[k >> shift & 255], 1);
        }
        __syncthreads();
        if (wid == 0) {                                                  // from the top: the bin that the want-th falls into
            int mine = 0;
            for (int i = 0; i < 8; ++i) mine += bins[255 - (lane * 8 + i)];
            int upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(kFull, upto, o);
                if (lane >= o) upto += v;
            }
            if (upto >= want && upto - mine < want) {
                int left = want - (upto - mine), i = 0;
                while (left > bins[255 - (lane * 8 + i)]) left -= bins[255 - (lane * 8 + i++)];
                prefix_s = prefix | (uint32_t)(255 - (lane * 8 + i)) << shift;
                want_s = left;
            }
        }
        __syncthreads();
        prefix = prefix_s;
        want = want_s;
        __syncthreads();
    }
    const uint32_t last = all ? ~0u : prefix;                            // kept: above it, and the first `want` that equal it
    // a warp takes a run of pieces; first what it keeps, then where that goes
    const int pieces = (r.len + kPiecePos - 1) / kPiecePos, each = (pieces + 7) / 8, p0 = min(pieces, wid * each), p1 = min(pieces, p0 + each);
    int above = 0, equal = 0, recent = 0;
    for (int t0 = p0 * kPiecePos; t0 < min(p1 * kPiecePos, r.len); t0 += 32) {
        const int t = t0 + lane;
        const uint32_t k = t < n ? weight_order(w[t]) : 0u;
        above += __popc(__ballot_sync(kFull, t < n && k > last && !all));
        equal += __popc(__ballot_sync(kFull, t < n && k == last && !all));
        recent += __popc(__ballot_sync(kFull, t >= n && t < r.len));
    }
    if (lane == 0) { warp_above[wid] = above; warp_equal[wid] = equal; warp_recent[wid] = recent; }
    __syncthreads();
    int at = 0, ties = 0;                                                // kept, and equal ones seen, before this warp's run
    for (int v = 0; v < wid; ++v) {
        at += warp_above[v] + warp_recent[v] + max(0, min(warp_equal[v], want - ties));
        ties += warp_equal[v];
    }
    const uint32_t lt = lanemask_lt();
    for (int t0 = p0 * kPiecePos; t0 < p1 * kPiecePos; t0 += 32) {
        if (t0 % kPiecePos == 0 && lane == 0) a.ahead[lane_at * a.pieces + t0 / kPiecePos] = at;
        const int t = t0 + lane;
        const float x = t < r.len ? w[t] : 0.f;
        const uint32_t k = weight_order(x);
        const uint32_t eq = __ballot_sync(kFull, t < n && k == last && !all);
        const bool take = t < n ? !all && (k > last || (k == last && ties + __popc(eq & lt) < want)) : t < r.len;
        const uint32_t m = __ballot_sync(kFull, take);
        if (take) to[at + __popc(m & lt)] = x;
        if (lane == 0) a.kept[(lane_at * a.pieces + t0 / kPiecePos) * 4 + t0 % kPiecePos / 32] = m;
        at += __popc(m);
        ties += __popc(eq);
    }
    for (int t = r.now + tid; t < a.n_pos; t += kSelectThreads) to[t] = 0.f;
}

// Page j of row s's new positions: its own where nobody else holds it, else a fresh one.  `fresh` of them come before.
__device__ __forceinline__ void evict_book(const PoolDev& p, const BookDev& in, const BookDev& out, const EvictArgs& a, int s, uint32_t* status) {
    const int lane = threadIdx.x & 31;                                   // a warp calls it
    const bool goes = a.base[s] >= 0 && !a.head[0];
    const int len = in.len[s], now = goes ? evict_row(p, in, a, s).now : len, keep = goes ? (now + p.page_pos - 1) / p.page_pos : in.max_pages;
    int at = a.base[s];
    uint32_t bits = 0;
    for (int j0 = 0; j0 < in.max_pages; j0 += 32) {
        const int j = j0 + lane;
        const int64_t i = (int64_t)s * in.max_pages + j;
        int page = j < in.max_pages ? in.table[i] : -1;
        if (page != -1 && !page_ok(p, page)) bits |= kStRange;
        const bool fresh = goes && j < keep && j < in.max_pages && in.ref[page] != 1;
        const uint32_t m = __ballot_sync(kFull, fresh);
        if (goes && page_ok(p, page) && (fresh || j >= keep)) atomicAdd(&out.ref[page], -1);
        if (fresh) {
            page = a.list[at + __popc(m & lanemask_lt())];
            out.ref[page] = 1;                                           // it was free, and this row alone has it
        }
        at += __popc(m);
        if (j < in.max_pages) out.table[i] = j < keep ? page : -1;
    }
    if (lane == 0) out.len[s] = now;
    if (bits) atomicOr(status, bits);
}

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev in, const __grid_constant__ BookDev out,
                                                                  const __grid_constant__ EvictArgs a, int lanes_log2, uint32_t* status) {
    __shared__ int64_t src_s[kPiecePos], dst_s[kPiecePos];
    __shared__ int n_s;
    chain_wait();
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const bool short_of = a.head[0] != 0;
    for (int s = blockIdx.x * (kMoveThreads / 32) + wid; s < in.rows; s += gridDim.x * (kMoveThreads / 32)) evict_book(p, in, out, a, s, status);
    const long long items = 2ll * in.rows * p.L * p.H;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long at_lane = item >> 1;
        const int kv = (int)(item & 1), h = (int)(at_lane % p.H), l = (int)(at_lane / p.H % p.L), s = (int)(at_lane / p.H / p.L);
        if (a.base[s] < 0) continue;
        const EvictRow r = evict_row(p, in, a, s);
        if (short_of) {                                                  // the weights stay as they are, too
            if (kv == 0) copy_weights(a.weight + (int64_t)s * a.ws_row + (int64_t)l * a.ws_layer + (int64_t)h * a.ws_head, a.out + at_lane * a.n_pos, min(r.len, a.n_pos), a.n_pos);
            continue;
        }
        uint8_t* plane = p.base + (int64_t)l * p.sl + (int64_t)kv * p.skv + (int64_t)h * p.sh;
        const int32_t* table = in.table + (int64_t)s * in.max_pages;
        const int pieces = (r.len + kPiecePos - 1) / kPiecePos;
        for (int c = 0; c < pieces; ++c) {
            __syncthreads();
            const int first = a.ahead[at_lane * a.pieces + c];
            if (tid < kPiecePos) {
                const uint32_t m = a.kept[(at_lane * a.pieces + c) * 4 + wid];
                int before = 0, n = 0;
                for (int v = 0; v < 4; ++v) {
                    const int cnt = __popc(a.kept[(at_lane * a.pieces + c) * 4 + v]);
                    if (v < wid) before += cnt;
                    n += cnt;
                }
                if (tid == 0) n_s = n;
                if (m >> lane & 1u) {
                    const int i = before + __popc(m & lanemask_lt()), t = c * kPiecePos + tid, to = first + i, j = to / p.page_pos;
                    const int page = table[t / p.page_pos];
                    int mine = table[j];
                    if (in.ref[mine] != 1) {                             // the row's how-manieth fresh page it is
                        int k = 0;
                        for (int e = 0; e < j; ++e) k += in.ref[table[e]] != 1;
                        mine = a.list[a.base[s] + k];
                    }
                    src_s[i] = (int64_t)page * p.spage + (int64_t)(t % p.page_pos) * p.sp;
                    dst_s[i] = (int64_t)mine * p.spage + (int64_t)(to % p.page_pos) * p.sp;
                }
            }
            __syncthreads();
            const int n = n_s, units = n << lanes_log2;
            for (int u0 = 0; u0 < units; u0 += 8 * kMoveThreads) {
                uint4 x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int u = u0 + k * kMoveThreads + tid;
                    if (u < units) x[k] = *reinterpret_cast<const uint4*>(plane + src_s[u >> lanes_log2] + (u & ((1 << lanes_log2) - 1)) * 16);
                }
                __syncthreads();                                         // all of the piece has been read that lies before what is written
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int u = u0 + k * kMoveThreads + tid;
                    if (u < units && src_s[u >> lanes_log2] != dst_s[u >> lanes_log2])
                        *reinterpret_cast<uint4*>(plane + dst_s[u >> lanes_log2] + (u & ((1 << lanes_log2) - 1)) * 16) = x[k];
                }
            }
        }
    }
}

int pieces_of(int n_pos) { return (n_pos + kPiecePos - 1) / kPiecePos; }
uint64_t evict_bytes(const PoolDev& p, long long rows, int n_pos) {
    const uint64_t words = 4 + (((uint64_t)rows + p.n_pages + 3) & ~3ull), lanes = (uint64_t)rows * p.L * p.H;
    return 4 * (words + lanes * pieces_of(n_pos) * 5);
}
plc_status check_lanes(const PoolDev& p, long long rows, int n_pos) {
    if (n_pos < 1) return PLC_E_INVALID;
    return rows * p.L * p.H > 0x3fffffffll || n_pos > kMostPositions ? PLC_E_SHAPE : PLC_OK;
}
bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
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
    *bytes = evict_bytes(p, rows, n_pos);
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
    if (weights->base_dev == out_weights_dev) return PLC_E_INVALID;
    if (workspace_bytes < evict_bytes(p, i.rows, weights->n_pos)) return PLC_E_CAPACITY;
    const long long lanes = (long long)i.rows * p.L * p.H;
    EvictArgs a{weights->base_dev, weights->stride_row, weights->stride_layer, weights->stride_head, weights->n_pos, out_weights_dev, budget_dev, budget, recent,
                nullptr, nullptr, nullptr, nullptr, nullptr, pieces_of(weights->n_pos)};
    a.head = static_cast<int32_t*>(workspace_dev);
    a.base = a.head + 4;
    a.list = a.base + i.rows;
    a.kept = reinterpret_cast<uint32_t*>(a.head + 4 + (((uint64_t)i.rows + p.n_pages + 3) & ~3ull));
    a.ahead = reinterpret_cast<int32_t*>(a.kept + (uint64_t)lanes * a.pieces * 4);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int lanes_log2 = 0;
    while ((16 << lanes_log2) < p.d * p.esz) ++lanes_log2;
    if (launch_kernel(evict_select_kernel, (unsigned)(1 + lanes), kSelectThreads, 0, st, false, 1, p, i, o, a, status_dev) != cudaSuccess) return PLC_E_CUDA;
    const long long most = 8ll * sm_count();
    if (launch_kernel(evict_move_kernel, (unsigned)(2 * lanes < most ? 2 * lanes : most), kMoveThreads, 0, st, true, 1, p, i, o, a, lanes_log2, status_dev) != cudaSuccess)
        return PLC_E_CUDA;
    count_launch(2);
    return PLC_OK;
}

}  // extern "C"
