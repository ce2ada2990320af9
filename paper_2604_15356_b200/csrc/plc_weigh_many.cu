// Attention weights where the sessions have many rows (entries times the query heads of a group): chunks of prompts, drafts of many heads.
//
// As in the other kernel positions are the rows of S = K Q^T, here the 128 lanes of tensor memory: a thread has a position, and the exponentials of the
// tile's columns are summed in its register, from row tile to row tile.  A CTA holds a tile of positions in shared memory (two of them, so that the next one arrives meanwhile)
// and goes through the row tiles that see any of it; Q and S have two buffers each, Q four where there are many row tiles of up to 128 components.  Boxes of pages and of queries where their layouts allow it,
// else pieces of 16 bytes.
//
// Bound by the exponentials (16 a clock and SM; the products need half as long) and by what is serial with them: 2048 tokens of 8 x 4 heads of 128 behind 8192 positions 243 us on the
// device (156 GFLOP, 640 TFLOP/s; the exponentials' unit is busy 0.67 of the time, the tensor pipe 0.33).  A step, 128 rows by 256 positions, takes 3160 clocks: 2300 to 2700 in the sums, of
// which the unit needs 2048, 170 to 580 waiting, 150 to 200 between steps; 8000 clocks pass before the first.  The power is not what bounds it: by the SMs' own counters calls in a row run at
// 1.83 GHz, where the unit alone would need 141 us (one call after a second's pause at 1.64 GHz).  Two threads a position were slower (297 us against 263 then), a quarter of the exponentials
// by a polynomial hardly faster (241 against 249).
// Or, where there is one row tile, by HBM: 32 sessions of up to 4096 positions, 5 tokens of 8 x 4 heads of 128: 44 us (177 MB, 4.1 TB/s).  Tiles of 128 positions with four
// buffers of keys took 76 with one warp for all copies against 54.
//
// Work: all (session, head, position tile, row tile) form one sequence, cut into equal ranges, one a CTA.  The first and the last piece of a range may be parts of an
// item (session, head, position tile); those leave their sums in the workspace, and a second launch adds them in a fixed order.
#include "plc_boxes.cuh"
#include "plc_tensor.cuh"
#include "plc_weigh.cuh"

namespace plc {
namespace {

constexpr float kLog2e = 1.44269504088896f;
// Row tiles whose normalisers, and items whose positions, are kept: the copies run up to six of them ahead of the exponentials.
constexpr int kRing = 8;

// DEEP: many row tiles an item, so that the queries' ring is what counts; else keys of the next item arrive while this one's are used.
template <int D, bool DEEP> struct Many {
    static constexpr int k_slots = DEEP ? 1 : 2, q_slots = DEEP && D != 256 ? 4 : 2;
    static constexpr int blocks = (D + 63) / 64;                       // 128-byte wide column blocks (32 components: half of one)
    static constexpr int groups = D == 256 ? 1 : 2, pos = 128 * groups;  // positions of a tile; four warps for each 128
    static constexpr int rows = D == 256 && !DEEP ? 64 : 128;          // of a row tile
    static constexpr int k_bytes = blocks * pos * 128, q_bytes = blocks * rows * 128;
    static constexpr int soft = 128 * groups, copy = 128, threads = soft + copy + 64;           // exponentials; copies; boxes of keys, products
    static constexpr int tmem = 2 * groups * rows;                     // S twice
    static constexpr int words = pos / 32;
    static constexpr size_t used = k_slots * (size_t)k_bytes + q_slots * q_bytes + kRing * (rows + words + 4) * 4 + 256 + 1024;
    static constexpr size_t smem = used > 120 * 1024 ? used : 120 * 1024;                    // one CTA an SM: it takes the tensor memory
};

// Where a CTA's range stands: item (session, head, position tile) and row tile in it.
template <int D, bool DEEP> struct Walk {
    using M = Many<D, DEEP>;
    int s, h, pt, rt, tiles, row_tiles;
    Newest x;
    // the first row tile that sees any of position tile pt
    __device__ __forceinline__ int begin_of(const WeighArgs& a, int tile) const {
        const long long behind = (long long)tile * M::pos - (x.len - x.n);
        return behind > 0 ? (int)(behind * a.group / M::rows) : 0;
    }
    __device__ __forceinline__ void enter(const PoolDev& p, const BookDev& b, const WeighArgs& a, int session) {
        bool bad;
        s = session;
        x = newest_of(p, b, a, s, &bad);
        tiles = (x.len + M::pos - 1) / M::pos;
        row_tiles = (int)(((long long)x.n * a.group + M::rows - 1) / M::rows);
    }
    // steps of one head
    __device__ __forceinline__ long long steps(const WeighArgs& a) const {
        long long n = (long long)tiles * row_tiles;
        for (int t = max(0, (x.len - x.n) / M::pos); t < tiles; ++t) n -= begin_of(a, t);
        return n;
    }
    __device__ __forceinline__ void start(const PoolDev& p, const BookDev& b, const WeighArgs& a, int session, long long rest) {
        enter(p, b, a, session);
        const long long n = steps(a);
        h = (int)(rest / n);
        rest -= h * n;
        const int full = min((int)min(rest / row_tiles, 0x7fffffffll), max(0, (x.len - x.n) / M::pos));        // tiles that all rows see
        pt = full;
        rest -= (long long)full * row_tiles;
        for (;; ++pt) {
            const int each = row_tiles - begin_of(a, pt);
            if (rest < each) break;
            rest -= each;
        }
        rt = begin_of(a, pt) + (int)rest;
    }
    // the next row tile; true where it is another item's
    __device__ __forceinline__ bool next(const PoolDev& p, const BookDev& b, const WeighArgs& a) {
        if (++rt < row_tiles) return false;
        if (++pt == tiles) {
            pt = 0;
            if (++h == p.H) {
                h = 0;
                do
                    if (++s >= b.rows) return true;
                    else enter(p, b, a, s);
                while (x.len == 0);
            }
        }
        rt = begin_of(a, pt);
        return true;
    }
    __device__ __forceinline__ int cols(const WeighArgs& a) const { return min(M::rows, x.n * a.group - rt * M::rows); }
};

// Waits, for so long at most, until a barrier's phase is complete.
__device__ __noinline__ void land(uint32_t bar, uint32_t parity) {
    for (uint32_t k = 0; k < kSpin; ++k)
        if (mbar_done(bar, parity)) break;
}

// Adds the exponentials of 32 columns' scores.  PLAIN: all of them count; else columns before `first_row` do not, nor those whose row counts for nothing, so
// that a key of infinities or NaN shows in the rows that see it alone.
template <bool PLAIN>
__device__ __forceinline__ void add_up(const uint32_t (&r)[32], const float* neg, unsigned long long c2, int first_row, unsigned long long (&acc)[4]) {
#pragma unroll
    for (int k = 0; k < 32; k += 4) {
        const float4 n = *reinterpret_cast<const float4*>(neg + k);
        float e[4];
        unpack2(fma2(pack2(__uint_as_float(r[k]), __uint_as_float(r[k + 1])), c2, pack2(n.x, n.y)), e[0], e[1]);
        unpack2(fma2(pack2(__uint_as_float(r[k + 2]), __uint_as_float(r[k + 3])), c2, pack2(n.z, n.w)), e[2], e[3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = exp2_approx(e[j]);
        if (!PLAIN) {
            const float nn[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k + j < first_row || isinf(nn[j])) e[j] = 0.f;
        }
        acc[k >> 1 & 2] = add2(acc[k >> 1 & 2], pack2(e[0], e[1]));
        acc[(k >> 1 & 2) + 1] = add2(acc[(k >> 1 & 2) + 1], pack2(e[2], e[3]));
    }
}

template <class T, int D, bool DEEP>
__global__ void __launch_bounds__(Many<D, DEEP>::threads, 1) weigh_many_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b, const __grid_constant__ WeighArgs a,
                                                                         const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap q_map, uint32_t* status) {
    using M = Many<D, DEEP>;
    constexpr int QS = M::q_slots, KS = M::k_slots, pieces = D / 8, copy_warp = M::soft / 32, box_warp = copy_warp + M::copy / 32, mma_warp = box_warp + 1;
    extern __shared__ uint8_t smem_raw[];
    __shared__ long long sums[M::threads / 32];
    __shared__ long long range_at[2];
    uint8_t* ks = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* qs = ks + KS * M::k_bytes;
    float* neg = reinterpret_cast<float*>(qs + QS * M::q_bytes);                // [kRing][rows] - lse log2 e; -inf: no row
    uint32_t* there = reinterpret_cast<uint32_t*>(neg + kRing * M::rows);          // [kRing][words] positions that have a page
    uint32_t* none = there + kRing * M::words;                                     // [kRing][4] row tiles with rows that count for nothing
    uint64_t* bars = reinterpret_cast<uint64_t*>(none + kRing * 4);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 12 + 2 * QS);
    volatile uint32_t* failed = tmem_slot + 1;
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const uint32_t k_full = smem_u32(bars), k_empty = k_full + 16, s_full = k_full + 32, s_empty = k_full + 64, q_full = k_full + 96,
                   q_empty = q_full + 8 * QS;
    chain_next();
    if (tid == 0) {
        for (int i = 0; i < QS; ++i) {
            mbar_init(q_full + 8 * i, M::copy / 32 + (a.q_boxes ? 1 : M::copy));
            mbar_init(q_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(k_full + 8 * i, a.box_pos ? 1 : M::copy + M::copy / 32);
            mbar_init(k_empty + 8 * i, 1);
            for (int m = 0; m < M::groups; ++m) {
                mbar_init(s_full + 8 * (2 * m + i), 1);
                mbar_init(s_empty + 8 * (2 * m + i), 4);
            }
        }
        *failed = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == mma_warp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)M::tmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // ---- the range: a thread sums the steps of a run of sessions, the threads' sums are scanned
    Walk<D, DEEP> w{};
    long long total = 0, mine = 0;
    const int run = (b.rows + M::threads - 1) / M::threads, s0 = min(b.rows, tid * run), s1 = min(b.rows, s0 + run);
    bool any_bad = false;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        bool bad;
        newest_of(p, b, a, s, &bad);
        any_bad |= bad;
        w.enter(p, b, a, s);
        if (w.x.len > 0) mine += w.steps(a) * p.H;
    }
    if (any_bad && blockIdx.x == 0) atomicOr(status, kStRange);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(kFull, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) sums[wid] = upto;
    fence_before();
    __syncthreads();
    long long ahead = upto - mine;
#pragma unroll 1
    for (int v = 0; v < M::threads / 32; ++v) {
        if (v < wid) ahead += sums[v];
        total += sums[v];
    }
    const int workers = (int)min((long long)gridDim.x, total), me = blockIdx.x;
    const long long t0 = me < workers ? total * me / workers : total, t1 = me < workers ? total * (me + 1) / workers : total, steps = t1 - t0;
    if (t0 < t1 && t0 >= ahead && t0 < ahead + mine) {
        long long at = ahead;
        int s = s0;
#pragma unroll 1
        for (; s < s1; ++s) {
            w.enter(p, b, a, s);
            const long long f = w.x.len > 0 ? w.steps(a) * p.H : 0;
            if (t0 < at + f) break;
            at += f;
        }
        range_at[0] = s;
        range_at[1] = t0 - at;
    }
    __syncthreads();
    fence_after();
    if (steps > 0) w.start(p, b, a, (int)range_at[0], range_at[1]);
    if (tid == 0) a.first[me] = steps > 0 ? make_int4(w.s, w.h, w.pt, w.rt - w.begin_of(a, w.pt)) : make_int4(-1, 0, 0, 0);
    const uint32_t tmem = *tmem_slot;

    if (wid < copy_warp) {
        // ---- exponentials: a thread a position
        const int group = wid >> 2, pos = tid;                                 // of the tile
        const uint32_t s_at = tmem + ((uint32_t)(wid & 3) << 21) + group * M::rows;
        const float c = a.scale * kLog2e;
        const unsigned long long c2 = pack2(c, c);
        float sum = 0.f;
        bool began = steps > 0 && w.rt == w.begin_of(a, w.pt);                 // the item's first row tile was this CTA's
        int item = 0, first_row = 0, full_row = 0;                             // the rows that see this thread's position, and all of the tile's
        auto enter = [&]() {
            const int start = w.x.len - w.x.n;
            first_row = max(w.pt * M::pos + pos - start, 0) * a.group;         // (at most the session's rows)
            full_row = max(w.pt * M::pos + M::pos - 1 - start, 0) * a.group;
        };
        if (steps > 0) enter();
        const uint32_t full = s_full + 16 * group, empty = s_empty + 16 * group;
        for (long long i = 0; i < steps; ++i) {
            const int buf = (int)i & 1, ring = (int)i & (kRing - 1), row0 = w.rt * M::rows;
            if (!__all_sync(kFull, mbar_wait(full + 8 * buf, (uint32_t)(i >> 1) & 1u, failed, status))) break;
            fence_after();
            const float* l = neg + ring * M::rows;
            const uint4 odd = *reinterpret_cast<const uint4*>(none + ring * 4);
            const bool plain = (odd.x | odd.y | odd.z | odd.w) == 0 && full_row <= row0;
            unsigned long long acc[4] = {0ull, 0ull, 0ull, 0ull};
            const uint32_t at = s_at + buf * M::groups * M::rows;
            if (plain) {                          // (rows behind the session's last one count for nothing)       // the next columns come while these are summed
                uint32_t r[2][32];
                tmem_ld32(at, r[0]);
#pragma unroll
                for (int ch = 0; ch < M::rows / 32; ++ch) {
                    wait_ld(r[ch & 1]);
                    if (ch + 1 < M::rows / 32) tmem_ld32(at + ch * 32 + 32, r[(ch + 1) & 1]);
                    add_up<true>(r[ch & 1], l + ch * 32, c2, 0, acc);
                }
            } else {
                for (int ch = 0; ch < (w.cols(a) + 31) / 32; ++ch) {
                    uint32_t r[32];
                    tmem_ld32(at + ch * 32, r);
                    wait_ld(r);
                    add_up<false>(r, l + ch * 32, c2, first_row - row0 - ch * 32, acc);
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * buf);
            {
                float lo, hi;
                unpack2(add2(add2(acc[0], acc[1]), add2(acc[2], acc[3])), lo, hi);
                sum += lo + hi;
            }
            const bool ended = w.rt + 1 == w.row_tiles;
            if (ended || i + 1 == steps) {
                const bool have = there[(item & (kRing - 1)) * M::words + (pos >> 5)] >> lane & 1u;
                const int t = w.pt * M::pos + pos;
                if (began && ended) {
                    if (t < w.x.len) put_weight(a, w.x, w.s, w.h, t, sum, have, status);
                } else a.part[((int64_t)2 * me + (item ? 1 : 0)) * M::pos + pos] = have ? sum : 0.f;
                sum = 0.f;
                began = true;
            }
            if (w.next(p, b, a)) {
                ++item;
                if (i + 1 < steps) enter();
            }
        }
    } else if (wid < box_warp) {
        // ---- copies, four warps that do not wait for each other: queries for every row tile (as a box: by the first warp), and where keys do not come in boxes those
        // at the start of an item.  Pieces of 16 bytes are shared by all, a warp a quarter of the vectors.
        const int lt = tid - M::soft, cw = wid - copy_warp;
        const uint32_t k_s = smem_u32(ks), q_s = smem_u32(qs);
        bool fresh = true, ok = true;
        int item = 0;
        long long q_last = -1;                    // the last row tile whose box has been issued
        // this thread's row of a row tile; its log-sum-exp is loaded a tile ahead
        int row = -1;
        const uint16_t* row_q = nullptr;
        float row_lse = 0.f;
        auto look_up = [&](const Walk<D, DEEP>& v) {
            const int r = v.rt * M::rows + lt;
            row = -1;
            if (lt < M::rows && r < v.x.n * a.group) {
                const int entry = r / a.group, head = v.h * a.group + r - entry * a.group;
                row = a.rows ? a.rows[v.x.first + entry] : v.x.first + entry;
                if (row < -1 || row >= a.n_rows) { atomicOr(status, kStRange); row = -1; }
                if (row >= 0) {
                    row_lse = a.lse[(int64_t)row * a.heads + head];
                    row_q = a.q + (int64_t)row * a.qs_row + (int64_t)head * a.qs_head;
                }
            }
        };
        auto page_of = [&](int t) -> int {        // of a position of the item; -1: none
            if (t >= w.x.len) return -1;
            const int page = b.table[(int64_t)w.s * b.max_pages + t / p.page_pos];
            if (page >= 0 && page < p.n_pages) return page;
            atomicOr(status, kStRange);
            return -1;
        };
        // N vectors that the lanes know the addresses of (0: none) into rows v0 ... of a block of `all` vectors
        auto pieces_of = [&](uint64_t at, int n, uint32_t to, int v0, int all) {
#pragma unroll 4
            for (int u = lane; u < n * pieces; u += 32) {
                const int v = u / pieces, c = u % pieces, r = v0 + v;
                const uint64_t from = __shfl_sync(kFull, at, v);
                copy16(to + (c >> 3) * (all * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), from ? reinterpret_cast<const uint8_t*>(from) + c * 16 : p.base, from != 0);
            }
        };
        if (steps > 0) look_up(w);
        for (long long i = 0; i < steps; ++i) {
            const int qb = (int)i & (QS - 1), kb = item & (KS - 1), ring = (int)i & (kRing - 1);
            const uint64_t row_at = row >= 0 && !isinf(row_lse) ? reinterpret_cast<uint64_t>(row_q) : 0ull;
            if (lt < M::rows) neg[ring * M::rows + lt] = row_at ? -row_lse * kLog2e : -INFINITY;
            const uint32_t odd = __ballot_sync(kFull, lt < M::rows && row_at == 0);
            if (lane == 0) none[ring * 4 + cw] = odd;
            if (fresh && !a.box_pos) {
                uint64_t at[M::pos / 128];
#pragma unroll
                for (int g = 0; g < M::pos / 128; ++g) {
                    const int k = cw * (M::pos / 4) + g * 32 + lane, t = w.pt * M::pos + k, page = page_of(t);
                    at[g] = page < 0 ? 0ull
                                     : reinterpret_cast<uint64_t>(p.base + (int64_t)a.layer * p.sl + (int64_t)w.h * p.sh + (int64_t)page * p.spage + (int64_t)(t % p.page_pos) * p.sp);
                    const uint32_t have = __ballot_sync(kFull, page >= 0);
                    if (lane == 0) there[(item & (kRing - 1)) * M::words + (k >> 5)] = have;
                }
                ok = __all_sync(kFull, ok && mbar_wait(k_empty + 8 * kb, ((uint32_t)(item / KS) & 1u) ^ 1u, failed, status));
                if (!ok) break;
#pragma unroll
                for (int g = 0; g < M::pos / 128; ++g) pieces_of(at[g], 32, k_s + kb * M::k_bytes, cw * (M::pos / 4) + g * 32, M::pos);
                mbar_arrive_copies(k_full + 8 * kb);
                __syncwarp();
                if (lane == 0) mbar_arrive(k_full + 8 * kb);
            }
            const int cols = w.cols(a), q_row = w.x.first + w.rt * (M::rows / a.group), q_head = w.h * a.group;
            fresh = w.next(p, b, a);
            item += fresh;
            if (i + 1 < steps) look_up(w);
            ok = __all_sync(kFull, ok && mbar_wait(q_empty + 8 * qb, ((uint32_t)(i / QS) & 1u) ^ 1u, failed, status));
            if (!ok) break;
            if (a.q_boxes) {
                if (cw == 0 && lane == 0) {
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(q_full + 8 * qb), "r"(M::q_bytes) : "memory");
#pragma unroll
                    for (int k = 0; k < M::blocks; ++k)
                        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                                         q_s + qb * M::q_bytes + k * (M::rows * 128)),
                                     "l"(&q_map), "r"(k * 64), "r"(q_head), "r"(q_row), "r"(q_full + 8 * qb)
                                     : "memory");
                }
                q_last = i;
            } else {
                if (cw * 32 < M::rows && cw * 32 < cols) pieces_of(row_at, 32, q_s + qb * M::q_bytes, cw * 32, M::rows);
                mbar_arrive_copies(q_full + 8 * qb);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full + 8 * qb);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (!ok && cw == 0)                       // boxes still in flight (none after a complete run) land before the CTA ends
            for (long long k = max(0ll, q_last - QS + 1); k <= q_last; ++k) land(q_full + 8 * ((int)k & (QS - 1)), (uint32_t)(k / QS) & 1u);
    } else if (wid == box_warp) {
        // ---- boxes of keys: a lane looks a box's page up, an item ahead
        const uint32_t k_s = smem_u32(ks);
        const int boxes = a.box_pos ? M::pos / a.box_pos : 0;
        int t = 0, page = -1, last = -1;
        bool ok = true;
        auto look_up = [&]() {                    // -1: behind the last position, -2: no page
            t = w.pt * M::pos + lane * a.box_pos;
            page = lane < boxes && t < w.x.len ? b.table[(int64_t)w.s * b.max_pages + t / p.page_pos] : -1;
            if (page == -1 && lane < boxes && t < w.x.len) page = -2;
        };
        long long left = boxes ? steps : 0;
        if (left > 0) look_up();
        for (int item = 0; left > 0; ++item) {
            const int kb = item & (KS - 1), at = t, h = w.h;
            const bool there_is = page >= 0 && page < p.n_pages;
            if (page < -1 || page >= p.n_pages) atomicOr(status, kStRange);
            const int here = page;
            const uint32_t have = __ballot_sync(kFull, there_is);
            left -= w.row_tiles - w.rt;
            w.rt = w.row_tiles - 1;
            if (left > 0) { w.next(p, b, a); look_up(); }
            ok = __all_sync(kFull, mbar_wait(k_empty + 8 * kb, ((uint32_t)(item / KS) & 1u) ^ 1u, failed, status));
            if (!ok) break;
            if (lane < M::words) {                // 32 positions' words
                uint32_t word = 0;
                if (a.box_pos >= 32) word = have >> (lane * 32 / a.box_pos) & 1u ? ~0u : 0u;
                else
                    for (int e = 0; e < 32 / a.box_pos; ++e)
                        if (have >> (lane * (32 / a.box_pos) + e) & 1u) word |= ((1u << a.box_pos) - 1u) << (e * a.box_pos);
                there[(item & (kRing - 1)) * M::words + lane] = word;
            }
            __syncwarp();                         // the words, which lane 0's arrival tells of
            if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(k_full + 8 * kb), "r"(__popc(have) * a.box_pos * M::blocks * 128) : "memory");
            __syncwarp();
            if (there_is) {
                int c[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) c[k] = a.box_dim[k] == 0 ? at % p.page_pos : a.box_dim[k] == 1 ? h : a.box_dim[k] == 2 ? here : 0;
#pragma unroll
                for (int k = 0; k < M::blocks; ++k)
                    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(
                                     k_s + kb * M::k_bytes + k * (M::pos * 128) + lane * a.box_pos * 128),
                                 "l"(&k_map), "r"(k * 64), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]), "r"(k_full + 8 * kb)
                                 : "memory");
            }
            last = item;
        }
        if (!ok)
            for (int k = max(0, last - KS + 1); k <= last; ++k) land(k_full + 8 * (k & (KS - 1)), (uint32_t)(k / KS) & 1u);
    } else if (lane == 0) {
        // ---- products
        int item = 0;
        bool fresh = true, ok = true;
        for (long long i = 0; i < steps; ++i) {
            const int buf = (int)i & 1, qb = (int)i & (QS - 1), kb = item & (KS - 1);
            const uint32_t n = (uint32_t)min(M::rows, (w.cols(a) + 15) & ~15);
            if (fresh) ok = ok && mbar_wait(k_full + 8 * kb, (uint32_t)(item / KS) & 1u, failed, status);
            ok = ok && mbar_wait(q_full + 8 * qb, (uint32_t)(i / QS) & 1u, failed, status);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            const uint32_t id = (1u << 4) | (Kind<T>::format << 7) | (Kind<T>::format << 10) | (8u << 24) | ((n >> 3) << 17);
            const uint64_t q_at = desc_k(smem_u32(qs) + qb * M::q_bytes);
#pragma unroll
            for (int m = 0; m < M::groups; ++m) {
                ok = ok && mbar_wait(s_empty + 8 * (2 * m + buf), ((uint32_t)(i >> 1) & 1u) ^ 1u, failed, status);
                if (!ok) break;
                fence_after();
                const uint64_t k_at = desc_k(smem_u32(ks) + kb * M::k_bytes + m * 128 * 128);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_ss(tmem + (buf * M::groups + m) * M::rows, k_at + (k >> 2) * (M::pos * 128 / 16) + 2 * (k & 3), q_at + (k >> 2) * (M::rows * 128 / 16) + 2 * (k & 3), id, k ? 1u : 0u);
                mma_commit(s_full + 8 * (2 * m + buf));
            }
            if (!ok) break;
            mma_commit(q_empty + 8 * qb);
            fresh = w.next(p, b, a);
            if (fresh) {
                mma_commit(k_empty + 8 * kb);
                ++item;
            }
        }
    }
    fence_before();
    __syncthreads();
    if (wid == mma_warp) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)M::tmem) : "memory");
    }
}

// Adds the pieces of items that more than one CTA had: block c looks at the boundary between CTAs c - 1 and c, and takes the item if that is the first
// boundary inside it.
template <int D>
__global__ void __launch_bounds__(Many<D, true>::pos) weigh_join_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b, const __grid_constant__ WeighArgs a, int workers,
                                                                  uint32_t* status) {
    using M = Many<D, true>;
    chain_wait();
    const int c = blockIdx.x + 1, pos = threadIdx.x;
    const int4 f = a.first[c], prev = a.first[c - 1];
    if (f.x < 0 || f.w == 0) return;
    auto same = [&](const int4& o) { return o.x == f.x && o.y == f.y && o.z == f.z; };
    if (same(prev) && prev.w > 0) return;
    float sum = a.part[((int64_t)2 * (c - 1) + (same(prev) ? 0 : 1)) * M::pos + pos];
    for (int k = c; k < workers; ++k) {
        const int4 o = a.first[k];
        if (!same(o) || o.w == 0) break;
        sum += a.part[(int64_t)2 * k * M::pos + pos];
    }
    bool bad;
    const Newest x = newest_of(p, b, a, f.x, &bad);
    const int t = f.z * M::pos + pos;
    if (t < x.len) put_weight(a, x, f.x, f.y, t, sum, true, status);           // (a position without a page has sums of 0)
}

// The queries of a row tile as one box: the heads of a group by as many rows as make up the tile.  Where rows are picked, the group does not divide the tile, or strides are not
// positive, they come in pieces.
template <int D, bool DEEP> bool query_boxes(const WeighArgs& a, bool bf16, CUtensorMap* map) {
    using M = Many<D, DEEP>;
    if (a.rows || D < 64 || M::rows % a.group || a.qs_row <= 0 || a.qs_head <= 0 || a.qs_row >= (1ll << 38) || a.qs_head >= (1ll << 38)) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.heads, (cuuint64_t)a.n_rows}, strides[2] = {(cuuint64_t)a.qs_head * 2, (cuuint64_t)a.qs_row * 2};
    const cuuint32_t boxes[3] = {64, (cuuint32_t)a.group, (cuuint32_t)(M::rows / a.group)}, ones[3] = {1, 1, 1};
    const EncodeTiledFn fn = encode_tiled_fn();
    return fn && fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<uint16_t*>(a.q), dims, strides, boxes, ones,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int D, bool DEEP>
cudaError_t launch(const PoolDev& p, const BookDev& b, const WeighArgs& args, uint32_t* status, cudaStream_t st) {
    using M = Many<D, DEEP>;
    cudaError_t e = cudaFuncSetAttribute(weigh_many_kernel<T, D, DEEP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)M::smem);
    if (e != cudaSuccess) return e;
    WeighArgs a = args;
    CUtensorMap k_map{}, q_map{};
    const bool bf16 = Kind<T>::format == 1;
    const int even = p.page_pos & -p.page_pos, box = even > 128 ? 128 : even;     // the largest power of two that divides a page, so that boxes fill a tile
    a.box_pos = box >= 8 && page_boxes(p, a.layer, bf16, box, &k_map, a.box_dim) ? box : 0;
    a.q_boxes = query_boxes<D, DEEP>(a, bf16, &q_map);
    const int grid = sm_count();
    e = launch_kernel(weigh_many_kernel<T, D, DEEP>, grid, M::threads, M::smem, st, false, 1, p, b, a, k_map, q_map, status);
    return e != cudaSuccess ? e : launch_kernel(weigh_join_kernel<D>, grid - 1, M::pos, 0, st, true, 1, p, b, a, grid, status);
}
template <class T, bool DEEP>
cudaError_t launch_by_dim(const PoolDev& p, const BookDev& b, const WeighArgs& a, uint32_t* status, cudaStream_t st) {
    switch (p.d) {
        case 32: return launch<T, 32, DEEP>(p, b, a, status, st);
        case 64: return launch<T, 64, DEEP>(p, b, a, status, st);
        case 128: return launch<T, 128, DEEP>(p, b, a, status, st);
        default: return launch<T, 256, DEEP>(p, b, a, status, st);
    }
}

}  // namespace

uint64_t weigh_many_bytes() { return (uint64_t)sm_count() * (16 + 2 * 256 * 4); }

cudaError_t launch_weigh_many(const PoolDev& p, const BookDev& b, const WeighArgs& args, void* workspace, bool bf16, uint32_t* status, cudaStream_t st) {
    WeighArgs a = args;
    a.first = static_cast<int4*>(workspace);
    a.part = reinterpret_cast<float*>(a.first + sm_count());
    // By the mean of the columns a session.  16 sessions of up to 4000 positions, 8 KV heads, us with keys ahead and with queries ahead: 120 columns of 64 / 128 / 256 components
    // 29.1 / 30.2 / 48.1 and 28.8 / 30.4 / 52.3, 240 columns 43.4 / 45.1 / 76.2 and 43.3 / 43.5 / 67.8, 800 columns 111 / 116 / 218 and 110 / 114 / 169.
    const bool deep = (long long)a.n_list * a.group > 192ll * b.rows;
    if (deep) return bf16 ? launch_by_dim<__nv_bfloat16, true>(p, b, a, status, st) : launch_by_dim<__half, true>(p, b, a, status, st);
    return bf16 ? launch_by_dim<__nv_bfloat16, false>(p, b, a, status, st) : launch_by_dim<__half, false>(p, b, a, status, st);
}

}  // namespace plc
