// Attention weights where the sessions have many rows (entries times the query heads of a group): chunks of prompts, drafts of many heads.
//
// As in the other kernel positions are the rows of S = K Q^T, here the 128 lanes of tensor memory: a thread has a position, and the exponentials of the
// tile's columns are summed in its register, from row tile to row tile.  A CTA holds a tile of positions in shared memory (two of them, so that the next one arrives meanwhile)
// and goes through the row tiles that see any of it; Q and S have two buffers each.  Bound by the exponentials (16 a clock and SM; the products need half as long)
// or, where there is one row tile, by HBM.
//
// Work: all (session, head, position tile, row tile) form one sequence, cut into equal ranges, one a CTA.  The first and the last piece of a range may be parts of an
// item (session, head, position tile); those leave their sums in the workspace, and a second launch adds them in a fixed order.
#include "plc_tensor.cuh"
#include "plc_weigh.cuh"

namespace plc {
namespace {

constexpr float kLog2e = 1.44269504088896f;
// Row tiles whose normalisers, and items whose positions, are kept: the copies run up to four of them ahead of the exponentials.
constexpr int kRing = 8;

template <int D> struct Many {
    static constexpr int blocks = (D + 63) / 64;                       // 128-byte wide column blocks (32 components: half of one)
    static constexpr int groups = D == 256 ? 1 : 2, pos = 128 * groups;  // positions of a tile; four warps for each 128
    static constexpr int rows = D == 256 ? 64 : 128;                   // of a row tile
    static constexpr int k_bytes = blocks * pos * 128, q_bytes = blocks * rows * 128;
    static constexpr int soft = 128 * groups, copy = 128, threads = soft + copy + 32;
    static constexpr int tmem = 2 * groups * rows;                     // S twice
    static constexpr int words = pos / 32;
    static constexpr size_t used = 2 * (size_t)k_bytes + 2 * q_bytes + 2 * pos * 8 + 2 * rows * 8 + kRing * (rows + words + 4) * 4 + 256 + 1024;
    static constexpr size_t smem = used > 120 * 1024 ? used : 120 * 1024;                    // one CTA an SM: it takes the tensor memory
};

// Where a CTA's range stands: item (session, head, position tile) and row tile in it.
template <int D> struct Walk {
    using M = Many<D>;
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

template <class T, int D>
__global__ void __launch_bounds__(Many<D>::threads, 1) weigh_many_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b, const __grid_constant__ WeighArgs a,
                                                                         uint32_t* status) {
    using M = Many<D>;
    constexpr int pieces = D / 8, copy_warp = M::soft / 32, mma_warp = copy_warp + M::copy / 32;
    extern __shared__ uint8_t smem_raw[];
    __shared__ long long sums[M::threads / 32];
    __shared__ long long range_at[2];
    uint8_t* ks = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* qs = ks + 2 * M::k_bytes;
    uint64_t* k_from = reinterpret_cast<uint64_t*>(qs + 2 * M::q_bytes);       // [2][pos] where a position's key stands
    uint64_t* q_from = k_from + 2 * M::pos;                                    // [2][rows] where a row stands
    float* neg = reinterpret_cast<float*>(q_from + 2 * M::rows);               // [kRing][rows] - lse log2 e; -inf: no row
    uint32_t* there = reinterpret_cast<uint32_t*>(neg + kRing * M::rows);          // [kRing][words] positions that have a page
    uint32_t* none = there + kRing * M::words;                                     // [kRing][4] row tiles with rows that count for nothing
    uint64_t* bars = reinterpret_cast<uint64_t*>(none + kRing * 4);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 12);
    volatile uint32_t* failed = tmem_slot + 1;
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const uint32_t k_full = smem_u32(bars), k_empty = k_full + 16, q_full = k_full + 32, q_empty = k_full + 48, s_full = k_full + 64, s_empty = k_full + 80;
    chain_next();
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(k_full + 8 * i, M::copy + M::copy / 32);
            mbar_init(k_empty + 8 * i, 1);
            mbar_init(q_full + 8 * i, M::copy + M::copy / 32);
            mbar_init(q_empty + 8 * i, 1);
            mbar_init(s_full + 8 * i, 1);
            mbar_init(s_empty + 8 * i, M::soft / 32);
        }
        *failed = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == mma_warp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)M::tmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // ---- the range: a thread sums the steps of a run of sessions, the threads' sums are scanned
    Walk<D> w{};
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
        int item = 0;
        for (long long i = 0; i < steps; ++i) {
            const int buf = (int)(i & 1), cols = w.cols(a), t = w.pt * M::pos + pos;
            const int row0 = w.rt * M::rows;
            // columns from this one on see the position
            const int first_row = (int)min(max((long long)(t - (w.x.len - w.x.n)) * a.group - row0, 0ll), (long long)M::rows);
            if (!__all_sync(kFull, mbar_wait(s_full + 8 * buf, (uint32_t)(i >> 1) & 1u, failed, status))) break;
            fence_after();
            const float* l = neg + (int)(i & (kRing - 1)) * M::rows;
            const uint32_t* odd = none + (int)(i & (kRing - 1)) * 4;
            const int last_t = w.pt * M::pos + M::pos - 1;
            const bool plain = !(odd[0] | odd[1] | odd[2] | odd[3]) && (long long)(last_t - (w.x.len - w.x.n)) * a.group <= row0;
            unsigned long long acc[4] = {0ull, 0ull, 0ull, 0ull};
            const uint32_t at = s_at + buf * M::groups * M::rows;
            if (plain && cols == M::rows) {       // the next columns come while these are summed
                uint32_t r[2][32];
                tmem_ld32(at, r[0]);
#pragma unroll
                for (int ch = 0; ch < M::rows / 32; ++ch) {
                    wait_ld(r[ch & 1]);
                    if (ch + 1 < M::rows / 32) tmem_ld32(at + ch * 32 + 32, r[(ch + 1) & 1]);
                    add_up<true>(r[ch & 1], l + ch * 32, c2, 0, acc);
                }
            } else {
                for (int ch = 0; ch < (cols + 31) / 32; ++ch) {
                    uint32_t r[32];
                    tmem_ld32(at + ch * 32, r);
                    wait_ld(r);
                    add_up<false>(r, l + ch * 32, c2, first_row - ch * 32, acc);
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(s_empty + 8 * buf);
            {
                float lo, hi;
                unpack2(add2(add2(acc[0], acc[1]), add2(acc[2], acc[3])), lo, hi);
                sum += lo + hi;
            }
            const Newest x = w.x;
            const int s = w.s, h = w.h, ended = w.rt + 1 == w.row_tiles, words = item & (kRing - 1);
            const bool other = w.next(p, b, a);
            if (ended || i + 1 == steps) {
                if (began && ended) {
                    if (t < x.len) put_weight(a, x, s, h, t, sum, there[words * M::words + (pos >> 5)] >> lane & 1u, status);
                } else a.part[((int64_t)2 * me + (item ? 1 : 0)) * M::pos + pos] = there[words * M::words + (pos >> 5)] >> lane & 1u ? sum : 0.f;
                sum = 0.f;
                began = true;
            }
            item += other;
        }
    } else if (wid < mma_warp) {
        // ---- copies, four warps: keys at the start of an item, queries for every row tile
        const int lt = tid - M::soft;
        constexpr int step = M::copy / pieces > 0 ? M::copy / pieces : 1;      // vectors a round
        const int cc = lt % pieces, r0 = lt / pieces;
        const uint32_t to = (cc >> 3) * 128, k_s = smem_u32(ks), q_s = smem_u32(qs);
        bool fresh = true, ok = true;
        int item = 0;
        // this thread's row of a row tile, looked up a tile ahead
        uint64_t row_at = 0;
        float row_neg = 0.f;
        auto look_up = [&](const Walk<D>& v) {
            const int r = v.rt * M::rows + lt;
            row_at = 0;
            row_neg = -INFINITY;
            if (lt < M::rows && r < v.x.n * a.group) {
                const int entry = r / a.group, head = v.h * a.group + r - entry * a.group;
                const int row = a.rows ? a.rows[v.x.first + entry] : v.x.first + entry;
                if (row >= 0 && row < a.n_rows) {
                    const float l = a.lse[(int64_t)row * a.heads + head];
                    if (!isinf(l)) {
                        row_neg = -l * kLog2e;
                        row_at = reinterpret_cast<uint64_t>(a.q + (int64_t)row * a.qs_row + (int64_t)head * a.qs_head);
                    }
                } else if (row != -1) atomicOr(status, kStRange);
            }
        };
        if (steps > 0) look_up(w);
        for (long long i = 0; i < steps; ++i) {
            const int buf = (int)(i & 1), kb = item & 1;
            if (lt < M::rows) {
                q_from[buf * M::rows + lt] = row_at;
                neg[(int)(i & (kRing - 1)) * M::rows + lt] = row_neg;
            }
            const uint32_t odd = __ballot_sync(kFull, lt < M::rows && row_at == 0);
            if (lane == 0) none[(int)(i & (kRing - 1)) * 4 + (wid - copy_warp)] = odd;
            if (fresh) {
#pragma unroll
                for (int g = 0; g < M::groups; ++g) {
                    const int k = g * 128 + lt, t = w.pt * M::pos + k;
                    uint64_t at = 0;
                    if (t < w.x.len) {
                        const int page = b.table[(int64_t)w.s * b.max_pages + t / p.page_pos];
                        if (page >= 0 && page < p.n_pages)
                            at = reinterpret_cast<uint64_t>(p.base + (int64_t)a.layer * p.sl + (int64_t)w.h * p.sh + (int64_t)page * p.spage + (int64_t)(t % p.page_pos) * p.sp);
                        else atomicOr(status, kStRange);
                    }
                    k_from[kb * M::pos + k] = at;
                    const uint32_t have = __ballot_sync(kFull, at != 0);
                    if (lane == 0) there[(item & (kRing - 1)) * M::words + (k >> 5)] = have;
                }
            }
            asm volatile("bar.sync 1, %0;" ::"n"(M::copy) : "memory");
            if (fresh) {
                ok = __all_sync(kFull, ok && mbar_wait(k_empty + 8 * kb, ((uint32_t)(item >> 1) & 1u) ^ 1u, failed, status));
                if (ok) {
#pragma unroll 8
                    for (int r = r0; r < M::pos; r += step) {
                        const uint64_t at = k_from[kb * M::pos + r];
                        copy16(k_s + kb * M::k_bytes + to * M::pos + r * 128 + (((cc & 7) ^ (r & 7)) << 4), at ? reinterpret_cast<const uint8_t*>(at) + cc * 16 : p.base, at != 0);
                    }
                    mbar_arrive_copies(k_full + 8 * kb);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(k_full + 8 * kb);
                }
            }
            const int cols = w.cols(a);
            fresh = w.next(p, b, a);
            item += fresh;
            if (i + 1 < steps) look_up(w);
            ok = __all_sync(kFull, ok && mbar_wait(q_empty + 8 * buf, ((uint32_t)(i >> 1) & 1u) ^ 1u, failed, status));
            if (ok) {
                const int upto = min(M::rows, (cols + 15) & ~15);
#pragma unroll 8
                for (int r = r0; r < upto; r += step) {
                    const uint64_t at = q_from[buf * M::rows + r];
                    copy16(q_s + buf * M::q_bytes + to * M::rows + r * 128 + (((cc & 7) ^ (r & 7)) << 4), at ? reinterpret_cast<const uint8_t*>(at) + cc * 16 : p.base, at != 0);
                }
                mbar_arrive_copies(q_full + 8 * buf);
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full + 8 * buf);
            }
            // (all four warps go on to the next barrier, so that none waits there alone; each leaves once all see that somebody has given up)
            uint32_t stop;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 2, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                         : "=r"(stop) : "r"((uint32_t)!ok), "n"(M::copy) : "memory");
            if (stop) break;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (lane == 0) {
        // ---- products
        int item = 0;
        bool fresh = true, ok = true;
        for (long long i = 0; i < steps; ++i) {
            const int buf = (int)(i & 1), kb = item & 1;
            const uint32_t n = (uint32_t)min(M::rows, (w.cols(a) + 15) & ~15);
            if (fresh) ok = ok && mbar_wait(k_full + 8 * kb, (uint32_t)(item >> 1) & 1u, failed, status);
            ok = ok && mbar_wait(q_full + 8 * buf, (uint32_t)(i >> 1) & 1u, failed, status);
            ok = ok && mbar_wait(s_empty + 8 * buf, ((uint32_t)(i >> 1) & 1u) ^ 1u, failed, status);
            if (!ok) break;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            fence_after();
            const uint32_t id = (1u << 4) | (Kind<T>::format << 7) | (Kind<T>::format << 10) | (8u << 24) | ((n >> 3) << 17);
            const uint64_t q_at = desc_k(smem_u32(qs) + buf * M::q_bytes);
#pragma unroll
            for (int m = 0; m < M::groups; ++m) {
                const uint64_t k_at = desc_k(smem_u32(ks) + kb * M::k_bytes + m * 128 * 128);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_ss(tmem + (buf * M::groups + m) * M::rows, k_at + (k >> 2) * (M::pos * 128 / 16) + 2 * (k & 3), q_at + (k >> 2) * (M::rows * 128 / 16) + 2 * (k & 3), id, k ? 1u : 0u);
            }
            mma_commit(s_full + 8 * buf);
            mma_commit(q_empty + 8 * buf);
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
__global__ void __launch_bounds__(Many<D>::pos) weigh_join_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b, const __grid_constant__ WeighArgs a, int workers,
                                                                  uint32_t* status) {
    using M = Many<D>;
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

template <class T, int D>
cudaError_t launch(const PoolDev& p, const BookDev& b, const WeighArgs& a, uint32_t* status, cudaStream_t st) {
    using M = Many<D>;
    cudaError_t e = cudaFuncSetAttribute(weigh_many_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)M::smem);
    if (e != cudaSuccess) return e;
    const int grid = sm_count();
    e = launch_kernel(weigh_many_kernel<T, D>, grid, M::threads, M::smem, st, false, 1, p, b, a, status);
    return e != cudaSuccess ? e : launch_kernel(weigh_join_kernel<D>, grid - 1, M::pos, 0, st, true, 1, p, b, a, grid, status);
}
template <class T>
cudaError_t launch_by_dim(const PoolDev& p, const BookDev& b, const WeighArgs& a, uint32_t* status, cudaStream_t st) {
    switch (p.d) {
        case 32: return launch<T, 32>(p, b, a, status, st);
        case 64: return launch<T, 64>(p, b, a, status, st);
        case 128: return launch<T, 128>(p, b, a, status, st);
        default: return launch<T, 256>(p, b, a, status, st);
    }
}

}  // namespace

uint64_t weigh_many_bytes() { return (uint64_t)sm_count() * (16 + 2 * 256 * 4); }

cudaError_t launch_weigh_many(const PoolDev& p, const BookDev& b, const WeighArgs& args, void* workspace, bool bf16, uint32_t* status, cudaStream_t st) {
    WeighArgs a = args;
    a.first = static_cast<int4*>(workspace);
    a.part = reinterpret_cast<float*>(a.first + sm_count());
    return bf16 ? launch_by_dim<__nv_bfloat16>(p, b, a, status, st) : launch_by_dim<__half>(p, b, a, status, st);
}

}  // namespace plc
