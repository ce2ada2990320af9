// Tree attention of few rows: single tokens, short drafts and small trees, where each K and V is read for at most 64 rows (a KV head's drafted
// tokens times its query heads) and HBM is the bound.
//
// The products are turned round, so that the 128 lanes of tensor memory are positions, not rows that are mostly empty:
//   S = K Q^T     [128 positions x N]      a lane a position, a column a row; N = the rows rounded up to 16
//   P = exp2(c S - m)                      a thread a position: the exponentials of a tile are spread over all four warps
//   O = O + V^T P [d x N]                  V as it lies in the page, P through shared memory
// Per tile that is N / 128 of the other layout's work in the products and the softmax, which leaves the copies ahead: they run in rings
// of K and of V that do not stop between items, Q has two buffers, and S two, so that the scores of a tile are formed while the one before is
// in the softmax.
// A row's maximum is common to the CTA and raised only where some score passes it by 2^3 (a vote of the four warps a tile); each thread sums the
// weights of its positions, and the sums are joined at the end of an item.
//
// Measured, components in 16 bits: one token of 4 heads a KV head, 37 sessions x 8192 positions x 8 KV heads x 128 components 182 us (6.8 TB/s at 1965 MHz; as
// many bytes at d = 64 6.7, d = 256 6.8 TB/s; caches flushed before each call 6.2).  Position by position, caches flushed: pages of 100 positions 6.1 TB/s, of 20 5.8, of one 5.0; of 100 at
// d = 64 4.4, d = 32 2.4: copies of 16 bytes each, and a vector has few of them.  Boxes that do not fill a tile: pages of 24 (120 of 128 positions) 5.3, of 72
// (72) 5.0, since every tile then has positions to hide.  256 sessions of up to 512 positions 74 us (353 MB, 4.8 TB/s): items end inside
// tiles there and each has a maximum, sums and results of its own, chains of votes that the copies wait for.  Code that is run once an item is
// fetched anew by then, so it is kept short: with its loops unrolled that call took 107 us, 0.34 of the warps' time without an instruction.
// Slower or the same: two slots of K or of V an SM's CTA in place of the second Q (74 -> 75 and 77 us), more CTAs than fit at once (7 to 40 %).
#pragma once
#include "plc_attend.cuh"

namespace plc {
namespace {

constexpr int kTN = 128;
constexpr int kWords = 16;                        // tiles whose validity words are kept: more than the ring holds

// N: most rows of an item, and the columns of its products.
template <int D, int N, bool BOX> struct Few {
    static constexpr int blocks = (D + 63) / 64;                       // 128-byte wide column blocks (32 components: half of one)
    static constexpr int slot = blocks * kTN * 128;
    // Rings of K and of V: each slot has one producer, in order, so that no wait can be a phase early.
    // Two CTAs an SM where the rows are fewest (their chains of small steps hide each other's latencies), else one with all of the shared memory.
    static constexpr int per_sm = BOX && N <= 32 && D != 256 ? 2 : 1;
    static constexpr int wide = D == 128 ? 1 : 2;                      // slots in the room of one of 128 components
    static constexpr int k_slots = D == 256 ? 1 : wide * (per_sm == 2 ? 1 : N == 16 ? 3 : 2), v_slots = D == 256 ? 2 : wide * (per_sm == 2 ? 1 : N == 64 ? 2 : 3);
    static constexpr int slots = k_slots + v_slots;
    static constexpr int q_bytes = blocks * N * 128, q_bufs = D == 256 ? 1 : 2;
    static constexpr int p_bytes = N * kTN * 2, p_bufs = D == 256 ? 1 : 2;
    static constexpr int o_blocks = D == 256 ? 2 : 1;
    // softmax: groups of four warps, which share the rows; N / groups of them a thread
    static constexpr int groups = N == 16 || per_sm == 2 ? 1 : 2, C = N / groups, soft = 128 * groups;
    static constexpr int pair = per_sm == 2 ? 1 : 2;                   // warps that copy keys in boxes, and as many for values
    static constexpr int copy = BOX ? 64 * pair : 128, q_copy = BOX ? 32 * pair : 128, threads = soft + copy + 64;
    static constexpr int tmem = N == 64 || o_blocks * N == 64 ? 256 : 128;   // S twice, O twice
    static constexpr size_t smem = (size_t)q_bufs * q_bytes + p_bufs * p_bytes + slots * slot + (BOX ? 0 : 3 * kTN * 8) + N * (8 + 4 * 13) + 768 + 1024;
};

// Of N threads at a barrier of their own: whether any, or all, say so.
template <int ID, int N> __device__ __forceinline__ bool vote_any(bool mine) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)mine), "n"(ID), "n"(N) : "memory");
    return r != 0;
}
template <int ID, int N> __device__ __forceinline__ bool vote_all(bool mine) { return !vote_any<ID, N>(!mine); }
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld4(uint32_t addr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ float warp_max(float x) {
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
// Sixteen values over the warp at once: lane l returns the sum of value l / 2 (lanes 2 r and 2 r + 1 the same).
__device__ __forceinline__ float warp_sums(const float* x, int lane) {
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i];
#pragma unroll
    for (int o = 16, n = 8; n > 0; o >>= 1, n >>= 1) {
        const bool high = lane & o;                  // keeps the upper half of what is left
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float give = high ? y[i] : y[n + i], keep = high ? y[n + i] : y[i];
            y[i] = keep + __shfl_xor_sync(kFull, give, o);
        }
    }
    return y[0] + __shfl_xor_sync(kFull, y[0], 1);
}
// P: blocks of 8 rows, in each 16 bytes a position (MN-major without swizzle: 128 bytes from eight positions to the next eight,
// 2048 from eight rows to the next eight).
__device__ __forceinline__ uint64_t desc_p(uint32_t addr) { return (uint64_t)((addr & 0x3FFFFu) >> 4) | (8ull << 16) | (128ull << 32) | (1ull << 46); }

// What rows row0 .. row0 + n - 1 (n <= 32) see of a warp's 32 positions t .. t+31, turned round: bit r says whether row row0 + r sees this lane's.
__device__ __noinline__ uint32_t seen_rows(const AttendArgs& a, const Session x, int row0, int n, int t, uint32_t valid) {
    const int lane = threadIdx.x & 31;
    uint32_t v = lane < n ? valid & seen_bits(a, x, (row0 + lane) / a.group, t) : 0u;
    uint32_t low = 0x0000ffffu;                   // a 32 x 32 transposition: blocks of 16, 8, ... 1 bits change places with the lane that far away
#pragma unroll
    for (int j = 16; j > 0; j >>= 1) {
        const uint32_t other = __shfl_xor_sync(kFull, v, j);
        v = lane & j ? (v & ~low) | (other >> j & low) : (v & low) | (other & low) << j;
        low ^= low << (j >> 1);
    }
    return v;
}

template <class T>
__device__ __noinline__ void put_back(const PoolDev& p, const BookDev& b, const AttendArgs& a, const Session x, int s, int h, int t0, int t1, int row0, int rows, int d,
                                      const int64_t* row_at, bool whole) {
    for (int t = max(t0, x.len); t < min(t1, x.kv); ++t) {
        const int page = b.table[(int64_t)s * b.max_pages + t / p.page_pos];
        if (page < 0 || page >= p.n_pages) continue;
        const uint16_t v = reinterpret_cast<const uint16_t*>(p.base + (int64_t)a.layer * p.sl + (int64_t)h * p.sh + p.skv + (int64_t)page * p.spage +
                                                             (int64_t)(t % p.page_pos) * p.sp)[d];
        if ((v & Kind<T>::exponent) != Kind<T>::exponent) continue;
        for (int r = 0; r < rows; ++r) {
            if (!(seen_bits(a, x, (row0 + r) / a.group, t) & 1u)) continue;
            if (!whole) { reinterpret_cast<float*>(row_at[r])[d] += Kind<T>::widen(v); continue; }
            uint16_t* o = reinterpret_cast<uint16_t*>(row_at[r]) + d;
            *o = (uint16_t)(Kind<T>::pack(Kind<T>::widen(*o) + Kind<T>::widen(v), 0.f) & 0xffffu);
        }
    }
}

template <class T, int D, int N, bool BOX>
__global__ void __launch_bounds__(Few<D, N, BOX>::threads, Few<D, N, BOX>::per_sm)
few_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b, const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map,
           uint32_t* status) {
    using F = Few<D, N, BOX>;
    using Tl = Tiles<N>;
    constexpr int slots = F::slots, k_slots = F::k_slots, v_slots = F::v_slots, C = F::C, soft_warps = F::soft / 32, qk_warp = F::threads / 32 - 2;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* qs = ring + slots * F::slot;
    uint8_t* ps = qs + F::q_bufs * F::q_bytes;
    uint64_t* from = reinterpret_cast<uint64_t*>(ps + F::p_bufs * F::p_bytes);                               // [3][kTN] where a position's key stands (without boxes)
    int64_t* row_at = reinterpret_cast<int64_t*>(from + (BOX ? 0 : 3 * kTN));                       // [N] the address that a row of the result goes to
    float* base_s = reinterpret_cast<float*>(row_at + N);                               // [N] what the weights' exponents are relative to
    float* top_s = base_s + N;                                                          // [N] maximum (scaled, base 2)
    float* factor_s = top_s + N;                                                        // [N]
    float* warp_s = factor_s + N;                                                       // [4][N]
    float* sum_s = warp_s + 4 * N;                                                      // [4][N] the last finished piece's: sums, maxima, 1 / sum
    float* last_top_s = sum_s + 4 * N;                                                  // [N]
    float* inv_s = last_top_s + N;                                                      // [N]
    uint32_t* words = reinterpret_cast<uint32_t*>(inv_s + N);                           // [kWords][4] positions that exist
    Tl* done = reinterpret_cast<Tl*>(words + kWords * 4);                               // the softmax's last finished piece
    uint64_t* bars = reinterpret_cast<uint64_t*>(done + 1);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * slots + 12);
    volatile uint32_t* failed = tmem_slot + 1;
    volatile uint32_t* dirty = tmem_slot + 2;     // [2] by a piece's parity: number + 1 of the last one whose V holds infinities or NaN at drafted positions
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const uint32_t full = smem_u32(bars), empty = full + 8 * slots, v_full = full + 8 * k_slots, v_empty = empty + 8 * k_slots, qfull = empty + 8 * slots, qempty = qfull + 16, sfull = qempty + 16, pfull = sfull + 16,
                   ofull = pfull + 16, drain = ofull + 16;
    chain_next();
    if (tid == 0) {
        for (int i = 0; i < slots; ++i) { mbar_init(full + 8 * i, BOX ? F::pair : F::copy + F::copy / 32); mbar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(qfull + 8 * i, F::q_copy);
            mbar_init(qempty + 8 * i, 1);
            mbar_init(sfull + 8 * i, 1);
            mbar_init(pfull + 8 * i, soft_warps);
            mbar_init(ofull + 8 * i, 1);
            mbar_init(drain + 8 * i, 1);
        }
        *failed = dirty[0] = dirty[1] = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == qk_warp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)F::tmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const int tile_pos = BOX ? a.tile_pos : kTN;
    if (BOX && tile_pos < kTN) {                  // positions of a tile that no box fills: zeros once and for all
        for (int i = tid; i < slots * F::blocks * kTN * 8; i += F::threads)          // pieces of 16 bytes as they lie there, eight a position
            if ((i >> 3) % kTN >= tile_pos) *reinterpret_cast<uint4*>(ring + i * 16) = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    fence_before();
    Walk<N> w0{};
    const long long total = find_range<N, F::threads>(p, b, a, status, w0);
    fence_after();
    const uint32_t tmem = *tmem_slot, ring_s = smem_u32(ring), v_ring_s = ring_s + k_slots * F::slot, q_s = smem_u32(qs), p_s = smem_u32(ps);

    if (wid >= soft_warps && wid < qk_warp) {
        const int lt = tid - F::soft;
        constexpr int pieces = D / 8;                // 16-byte pieces of a vector
        auto load_q = [&](const Tl& x, bool ok) -> bool {    // a piece's rows of Q; whole warps
            const int q = x.piece % F::q_bufs, rows = x.w.rows(a);
            ok = __all_sync(kFull, ok && mbar_wait(qempty + 8 * q, ((uint32_t)(x.piece / F::q_bufs) & 1u) ^ 1u, failed, status));
            if (!ok) return false;
            constexpr int halves = (N + 31) / 32;
            unsigned long long row[halves];          // where a row stands, found by one lane
#pragma unroll
            for (int e = 0; e < halves; ++e) {
                const int r = 32 * e + lane, rr = x.w.rt * N + r, i = rr / a.group;
                row[e] = r < rows ? (unsigned long long)a.q + 2 * ((int64_t)(x.w.x.first + i) * a.qs_row + (int64_t)(x.w.h * a.group + rr - i * a.group) * a.qs_head) : 0ull;
            }
#pragma unroll 2
            for (int u = lt; u < N * pieces; u += F::q_copy) {
                const int r = u / pieces, c = u % pieces;
                unsigned long long src = __shfl_sync(kFull, row[0], r & 31);
                if (halves > 1) { const unsigned long long up = __shfl_sync(kFull, row[halves - 1], r & 31); src = r < 32 ? src : up; }
                copy16(q_s + q * F::q_bytes + (c >> 3) * (N * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), reinterpret_cast<const uint8_t*>(src ? src + c * 16 : (unsigned long long)a.q), src != 0);
            }
            mbar_arrive_copies(qfull + 8 * q);
            return true;
        };
        if constexpr (BOX) {
            // ---- copies: a warp or two for the keys, as many for the values
            const int kv = lt / F::q_copy;
            copy_boxes<N, F::blocks, kTN>(p, b, a, map, w0, total, kv, (lt >> 5) % F::pair, F::pair, kv ? v_ring_s : ring_s, F::slot, kv ? v_slots : k_slots,
                                          kv ? v_full : full, kv ? v_empty : empty, words, kWords, failed, status, load_q);
        } else {
            // ---- copies, four warps, position by position (pages of any size)
            constexpr int step = F::copy / pieces, rounds = kTN / step;   // vectors a round
            const int c = lt % pieces, r0 = lt / pieces;
            const uint32_t to = (c >> 3) * (kTN * 128) + r0 * 128;
            Tl kx, vx;
            kx.start(w0, total);
            vx.start(w0, total);
            int kt = 0, vt = 0;
            bool ok = true;
            auto fill = [&](int tile, bool values) {           // a tile's keys or values into the next slot of their ring
                const int s = tile % (values ? v_slots : k_slots);
                const uint32_t ph = (uint32_t)(tile / (values ? v_slots : k_slots)) & 1u, bar = (values ? v_full : full) + 8 * s;
                ok = __all_sync(kFull, ok && mbar_wait((values ? v_empty : empty) + 8 * s, ph ^ 1u, failed, status));
                if (!ok) return;
                const uint32_t dst = (values ? v_ring_s : ring_s) + s * F::slot + to;
                const int64_t delta = (values ? p.skv : 0) + c * 16;
                const uint64_t* src = from + tile % 3 * kTN + r0;
                const uint32_t* valid = words + tile % kWords * 4;
                const bool all = (valid[0] & valid[1] & valid[2] & valid[3]) == ~0u;
#pragma unroll
                for (int k0 = 0; k0 < rounds; k0 += 8) {
                    uint64_t at[8];
#pragma unroll
                    for (int k = 0; k < 8 && k0 + k < rounds; ++k) at[k] = src[(k0 + k) * step];
                    if (all) {
#pragma unroll
                        for (int k = 0; k < 8 && k0 + k < rounds; ++k)
                            copy16(dst + (k0 + k) * step * 128 + (((c & 7) ^ ((r0 + (k0 + k) * step) & 7)) << 4), reinterpret_cast<const uint8_t*>(at[k] + delta));
                    } else {
#pragma unroll
                        for (int k = 0; k < 8 && k0 + k < rounds; ++k) {
                            const int r = r0 + (k0 + k) * step;
                            copy16(dst + (k0 + k) * step * 128 + (((c & 7) ^ (r & 7)) << 4), reinterpret_cast<const uint8_t*>(at[k] + delta), valid[r >> 5] >> (r & 31) & 1u);
                        }
                    }
                }
                mbar_arrive_copies(bar);
                __syncwarp();
                if (lane == 0) mbar_arrive(bar);                        // the validity words, too, are there
            };
            int slot_in = 0, page = -1;                  // this thread's position of K's next tile: slot in its page, the page
            auto look_up = [&]() {                       // issued a tile ahead of its use
                const int t = (kx.w.tile + kx.j) * kTN + lt, pg = t / p.page_pos;
                const bool have = t < kx.w.x.kv;
                slot_in = have ? t - pg * p.page_pos : -1;
                page = have ? b.table[(int64_t)kx.w.s * b.max_pages + pg] : 0;
            };
            if (kx.more()) look_up();
            for (;;) {
                const bool more = kx.more();
                if (!more && !vx.more()) break;
                if (more) {
                    if (kx.j == 0) ok = load_q(kx, ok);
                    const bool there = page >= 0 && page < p.n_pages, have = slot_in >= 0 && there;
                    if (!there) atomicOr(status, kStRange);
                    // (a position that does not exist: anywhere in the pool, nothing is read)
                    from[kt % 3 * kTN + lt] = reinterpret_cast<uint64_t>(p.base) +
                                              (have ? (int64_t)a.layer * p.sl + (int64_t)kx.w.h * p.sh + (int64_t)page * p.spage + (int64_t)slot_in * p.sp : 0);
                    const uint32_t valid = __ballot_sync(kFull, have);
                    if (lane == 0) words[kt % kWords * 4 + (lt >> 5)] = valid;
                }
                if (!vote_all<1, F::copy>(ok)) break;
                if (more) {
                    fill(kt, false);
                    ++kt;
                    kx.next(p, b, a);
                    if (kx.more()) look_up();
                }
                if (kt > 1 || !more) {                                           // V of a tile after K of the next
                    fill(vt, true);
                    ++vt;
                    vx.next(p, b, a);
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
    } else if (wid >= qk_warp) {
        if (lane == 0) {
            // ---- products, a thread for each of the two
            constexpr uint32_t id_qk = (1u << 4) | (Kind<T>::format << 7) | (Kind<T>::format << 10) | (8u << 24) | ((uint32_t)(N >> 3) << 17), id_pv = id_qk | (3u << 15);
            Tl tl;
            tl.start(w0, total);
            bool ok = true;
            auto ready = [&](uint32_t bar, uint32_t phase) {
                ok = ok && mbar_wait(bar, phase & 1u, failed, status);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                fence_after();
            };
            if (wid == qk_warp) {
                for (int x = 0; tl.more(); ++x, tl.next(p, b, a)) {
                    const int q = tl.piece % F::q_bufs, i = x % k_slots;
                    if (tl.j == 0) ok = ok && mbar_wait(qfull + 8 * q, (uint32_t)(tl.piece / F::q_bufs) & 1u, failed, status);
                    if (x >= 2) ok = ok && mbar_wait(pfull + 8 * (x & 1), (uint32_t)((x - 2) >> 1) & 1u, failed, status);   // S has been read
                    ready(full + 8 * i, (uint32_t)(x / k_slots));
                    if (!ok) break;
                    const uint64_t k_at = desc_k(ring_s + i * F::slot), q_at = desc_k(q_s + q * F::q_bytes);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_ss(tmem + (x & 1) * N, k_at + (k >> 2) * (kTN * 128 / 16) + 2 * (k & 3), q_at + (k >> 2) * (N * 128 / 16) + 2 * (k & 3), id_qk, k ? 1u : 0u);
                    mma_commit(sfull + 8 * (x & 1));
                    mma_commit(empty + 8 * i);
                    if (tl.last()) mma_commit(qempty + 8 * q);
                }
            } else {
                for (int x = 0; tl.more(); ++x, tl.next(p, b, a)) {
                    const int i = x % v_slots;
                    ok = ok && mbar_wait(pfull + 8 * (x & 1), (uint32_t)(x >> 1) & 1u, failed, status);
                    ready(v_full + 8 * i, (uint32_t)(x / v_slots));
                    if (!ok) break;
                    // lanes past the components of a vector take the first block again
                    const uint64_t v_at = desc_mn(v_ring_s + i * F::slot, D >= 128 ? kTN * 128 : 0), p_at = desc_p(p_s + x % F::p_bufs * F::p_bytes);
                    const uint32_t o_to = tmem + 2 * N + (tl.piece & 1) * F::o_blocks * N;
#pragma unroll
                    for (int o = 0; o < F::o_blocks; ++o)
#pragma unroll
                        for (int k = 0; k < kTN / 16; ++k)
                            mma_ss(o_to + o * N, v_at + (o * 2 * kTN * 128 + k * 2048) / 16, p_at + k * 16, id_pv, tl.j | k ? 1u : 0u);
                    mma_commit(ofull + 8 * (x & 1));
                    mma_commit(v_empty + 8 * i);
                }
            }
            const uint32_t mine = drain + 8 * (wid - qk_warp);
            mma_commit(mine);                         // nothing issued runs when the CTA frees its tensor memory
            for (uint32_t i = 0; i < kSpin; ++i) {
                uint32_t done;
                asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], 0;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(mine) : "memory");
                if (done) break;
            }
        }
    } else {
        // ---- softmax and results: a thread a position, then a component
        const int quarter = wid & 3, col0 = (wid >> 2) * C, pos = tid & 127;                 // the warp's positions (components), its group's rows
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, o_at = tmem + 2 * N + col0 + lanes;
        const unsigned long long c2 = pack2(a.scale * 1.44269504088896f, a.scale * 1.44269504088896f);
        Tl sx;
        sx.start(w0, total);
        unsigned long long sum[C / 2];                // of this thread's weights, pairs of rows
        bool ok = true;
        auto results = [&](int last) -> bool {        // of the piece that *done tells of; a thread a component
            ok = ok && mbar_wait(ofull + 8 * (last & 1), (uint32_t)(last >> 1) & 1u, failed, status);
            if (!vote_all<2, F::soft>(ok)) return false;
            const Tl f = *done;
            const int rows = f.w.rows(a), row0 = f.w.rt * N;
            const bool whole = f.w.tile == 0 && f.m == f.w.tiles;
            const int64_t slot = ((int64_t)2 * blockIdx.x + (f.piece > 0)) * a.part_rows;
            if (tid < rows) {
                const float l = (sum_s[tid] + sum_s[N + tid]) + (sum_s[2 * N + tid] + sum_s[3 * N + tid]), top = last_top_s[tid];
                const int rr = row0 + tid, i = (int)((uint32_t)rr / (uint32_t)a.group);
                const int64_t n_row = f.w.x.first + i, head = (int64_t)f.w.h * a.group + (rr - i * a.group);
                row_at[tid] = whole ? reinterpret_cast<int64_t>(a.out) + 2 * (n_row * a.os_row + head * a.os_head) : reinterpret_cast<int64_t>(a.part_o + (slot + tid) * D);
                inv_s[tid] = l == 0.f ? 0.f : whole ? 1.f / l : 1.f;             // 0: nothing was seen
                if (!whole) a.part_ml[slot + tid] = make_float2(top, l);
                else if (a.lse) a.lse[n_row * a.heads + head] = l == 0.f ? -INFINITY : (top - Kind<T>::shift + log2f(l)) * 0.693147180559945f;
            }
            vote_all<2, F::soft>(true);
            fence_after();
            // four rows at a time: this code is fetched anew for most pieces, and short code costs less than more loads at a time give
#pragma unroll 1
            for (int o = 0; o < F::o_blocks; ++o) {
                const int d = o * 128 + pos;
#pragma unroll 1
                for (int r0 = col0; r0 < min(rows, col0 + C); r0 += 4) {
                    uint32_t y[4];
                    tmem_ld4(o_at - col0 + ((f.piece & 1) * F::o_blocks + o) * N + r0, y);
                    wait_ld(y);
                    if (d >= D) continue;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (r0 + r < rows) {
                            const float g = inv_s[r0 + r], v = g == 0.f ? 0.f : __uint_as_float(y[r]) * g;
                            const int64_t to = row_at[r0 + r];
                            if (whole) reinterpret_cast<uint16_t*>(to)[d] = (uint16_t)(Kind<T>::pack(v, 0.f) & 0xffffu);
                            else reinterpret_cast<float*>(to)[d] = v;
                        }
                }
            }
            if (dirty[f.piece & 1] == (uint32_t)f.piece + 1u && vote_all<2, F::soft>(true))       // every group's rows are written
                for (int d = tid; d < D; d += F::soft)
                    put_back<T>(p, b, a, f.w.x, f.w.s, f.w.h, f.w.tile * tile_pos, (f.w.tile + f.m) * tile_pos, row0, rows, d, row_at, whole);
            fence_before();
            return true;
        };
        for (int x = 0;; ++x) {
            const bool more = x < total, first = more && sx.j == 0;
            if (more) {
                const int t0 = (sx.w.tile + sx.j) * tile_pos;
                const int in_use = (sx.w.rows(a) - col0 + 3) & ~3;   // of the group's rows, in fours; the others' weights may be anything
                const bool drafted = t0 + tile_pos > sx.w.x.len;
                ok = ok && mbar_wait(sfull + 8 * (x & 1), (uint32_t)(x >> 1) & 1u, failed, status);
                if (x >= F::p_bufs) ok = ok && mbar_wait(ofull + 8 * ((x - F::p_bufs) & 1), (uint32_t)((x - F::p_bufs) >> 1) & 1u, failed, status);
                ok = __all_sync(kFull, ok);
                fence_after();
                const uint32_t s_at = tmem + (x & 1) * N + col0 + lanes;
                const uint4 valid = *reinterpret_cast<const uint4*>(words + x % kWords * 4);
                const bool may_hide = a.mask != nullptr || sx.w.x.n > 1, hide = may_hide && drafted;
                const bool masked = hide || (valid.x & valid.y & valid.z & valid.w) != ~0u;
                uint32_t vis = 0;                         // the group's rows that see this thread's position
                if (masked) {
                    const uint32_t mine = words[x % kWords * 4 + quarter];
                    vis = hide ? seen_rows(a, sx.w.x, sx.w.rt * N + col0, sx.w.rows(a) - col0, t0 + 32 * quarter, mine) : mine >> lane & 1u ? ~0u : 0u;
                }
                uint32_t s[16];                           // 16 rows' scores at a time; more of them stay in tensor memory meanwhile
                auto scores = [&](int ch) {
                    tmem_ld16(s_at + 16 * ch, s);
                    wait_ld(s);
                    if (masked) {
                        const uint32_t mine = vis >> (16 * ch);
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[r] = mine >> r & 1u ? s[r] : 0xff800000u;
                    }
                };
                // exponents relative to base, four rows from r on
                auto exponents = [&](int r, float* e) {
                    const ulonglong2 base = *reinterpret_cast<const ulonglong2*>(base_s + col0 + r);
                    const int k = r & 15;
                    unpack2(fma2(pack2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, base.x), e[0], e[1]);
                    unpack2(fma2(pack2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])), c2, base.y), e[2], e[3]);
                };
                if (C == 16) scores(0);
                float high = -INFINITY;                   // one above the border asks for a new maximum (rows without one have a base far below)
                if (!first) {
#pragma unroll
                    for (int r = 0; r < C; r += 4) {
                        if (r >= in_use) break;
                        if (C > 16 && (r & 15) == 0) scores(r >> 4);
                        float e[4];
                        exponents(r, e);
                        high = fmaxf(high, fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3])));
                    }
                }
                if (vote_any<2, F::soft>(first || !ok || high > kRaise + Kind<T>::shift)) {
                    // some row's maximum rises: all warps' maxima, the factors, and what has been summed so far
#pragma unroll
                    for (int r = 0; r < C; ++r) {
                        if (r >= in_use) break;
                        if (C > 16 && (r & 15) == 0) scores(r >> 4);
                        const float m = warp_max(__uint_as_float(s[r & 15]));
                        if (lane == r) warp_s[quarter * N + col0 + r] = m;
                    }
                    if (!first) ok = ok && mbar_wait(ofull + 8 * ((x - 1) & 1), (uint32_t)((x - 1) >> 1) & 1u, failed, status);
                    if (!vote_all<2, F::soft>(ok)) { ok = false; break; }
                    if (tid < N) {
                        const float now = fmaxf(fmaxf(warp_s[tid], warp_s[N + tid]), fmaxf(warp_s[2 * N + tid], warp_s[3 * N + tid])) * (a.scale * 1.44269504088896f);
                        const float old = first ? -INFINITY : top_s[tid];
                        const float top = now > old + kRaise ? now : old;
                        top_s[tid] = top;
                        base_s[tid] = top == -INFINITY ? 1e30f : Kind<T>::shift - top;
                        factor_s[tid] = top == old ? 1.f : old == -INFINITY ? 0.f : exp2_approx(old - top);
                    }
                    vote_all<2, F::soft>(true);
                    if (first) {
#pragma unroll
                        for (int r = 0; r < C / 2; ++r) sum[r] = 0ull;
                    } else {
                        fence_after();
#pragma unroll
                        for (int r = 0; r < C; r += 2) {
                            float lo, hi;
                            unpack2(sum[r / 2], lo, hi);
                            sum[r / 2] = pack2(lo * factor_s[col0 + r], hi * factor_s[col0 + r + 1]);
                        }
#pragma unroll 1
                        for (int ch = 0; ch < F::o_blocks * C / 16; ++ch) {
                            uint32_t y[16];
                            const uint32_t at = o_at + ((sx.piece & 1) * F::o_blocks + 16 * ch / C) * N + 16 * ch % C;
                            tmem_ld16(at, y);
                            wait_ld(y);
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const float f = factor_s[col0 + (16 * ch + r) % C];
                                y[r] = __float_as_uint(f == 0.f ? 0.f : __uint_as_float(y[r]) * f);
                            }
                            tmem_st16(at, y);
                        }
                        wait_st();
                    }
                }
                uint8_t* pp = ps + x % F::p_bufs * F::p_bytes + col0 / 8 * 2048 + pos * 16;
#pragma unroll
                for (int r = 0; r < C; r += 8) {
                    if (r >= in_use) break;
                    if (C > 16 && (r & 15) == 0) scores(r >> 4);
                    uint32_t y[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < 8; k += 4) {
                        if (r + k >= in_use) break;
                        float e[4];
                        exponents(r + k, e);
#pragma unroll
                        for (int i = 0; i < 4; ++i) e[i] = exp2_approx(e[i]);                 // a score of -inf has the weight 0
                        sum[(r + k) / 2] = add2(sum[(r + k) / 2], pack2(e[0], e[1]));
                        sum[(r + k) / 2 + 1] = add2(sum[(r + k) / 2 + 1], pack2(e[2], e[3]));
                        y[k / 2] = Kind<T>::pack(e[0], e[1]);
                        y[k / 2 + 1] = Kind<T>::pack(e[2], e[3]);
                    }
                    *reinterpret_cast<uint4*>(pp + (r / 8) * 2048) = make_uint4(y[0], y[1], y[2], y[3]);
                }
                // V of positions that do not exist is whatever the boxes brought or left: zeros instead, since weights of 0 do not hide it
                const bool blank = BOX && masked && pos < tile_pos && !(words[x % kWords * 4 + quarter] >> lane & 1u);
                if ((hide || (BOX && masked)) && wid < 4) {
                    // with one slot the tile before may still be awaited, and a parity tells only one tile from the next: its product first
                    if (v_slots == 1 && x > 0) ok = ok && mbar_wait(ofull + 8 * ((x - 1) & 1), (uint32_t)((x - 1) >> 1) & 1u, failed, status);
                    ok = ok && mbar_wait(v_full + 8 * (x % v_slots), (uint32_t)(x / v_slots) & 1u, failed, status);
                    uint8_t* tile = ring + (k_slots + x % v_slots) * F::slot;
                    if (ok && blank)
#pragma unroll 2
                        for (int e = 0; e < F::blocks * 8; ++e)
                            *reinterpret_cast<uint4*>(tile + (e >> 3) * (kTN * 128) + pos * 128 + (((e & 7) ^ (pos & 7)) << 4)) = make_uint4(0, 0, 0, 0);
                    else if (ok && hide && pos < tile_pos && t0 + pos >= sx.w.x.len && t0 + pos < sx.w.x.kv && special<T, D, kTN>(tile, pos) && take_out<T, D, kTN>(tile, pos))
                        dirty[sx.piece & 1] = (uint32_t)sx.piece + 1u;
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // P (and V) as the product reads them
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pfull + 8 * (x & 1));
            }
            // the results of the piece before, whose last product has had this tile's time to finish
            if (x > 0 && (first || !more) && !(ok = results(x - 1))) break;
            if (!more) break;
            if (sx.last()) {                          // the piece is done: its sums over the positions
                if (tid == 0) *done = sx;
#pragma unroll
                for (int ch = 0; ch < C / 16; ++ch) {
                    float l[16];
#pragma unroll
                    for (int r = 0; r < 16; r += 2) unpack2(sum[8 * ch + r / 2], l[r], l[r + 1]);
                    const float v = warp_sums(l, lane);
                    if (!(lane & 1)) sum_s[quarter * N + col0 + 16 * ch + lane / 2] = v;
                }
                if (tid < N) last_top_s[tid] = top_s[tid];
            }
            sx.next(p, b, a);
        }
    }
    fence_before();
    __syncthreads();
    if (wid == qk_warp) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)F::tmem) : "memory");
    }
}

template <class T, int D, int N, bool BOX>
cudaError_t launch(const PoolDev& p, const BookDev& b, const AttendArgs& a, const CUtensorMap& map, const AttendPlan& x, uint32_t* status, cudaStream_t st) {
    using F = Few<D, N, BOX>;
    cudaError_t e = cudaFuncSetAttribute(few_kernel<T, D, N, BOX>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)F::smem);
    if (e != cudaSuccess) return e;
    AttendPlan y = x;
    y.grid = F::per_sm * sm_count();
    if (a.whole && a.whole < y.grid) y.grid = a.whole;
    e = launch_kernel(few_kernel<T, D, N, BOX>, y.grid, F::threads, F::smem, st, false, 1, p, b, a, map, status);
    return e != cudaSuccess || a.whole ? e : launch_join<T, D, N>(p, b, a, y, st);
}
template <class T>
cudaError_t launch_few(const PoolDev& p, const BookDev& b, const AttendArgs& args, const AttendPlan& x, bool bf16, uint32_t* status, cudaStream_t st) {
    AttendArgs a = args;
    a.tile_pos = kTN;
    CUtensorMap map{};
    const bool boxes = make_boxes(p, a, bf16, kTN, &map), least = x.row_tile == 16, mid = x.row_tile == 32;
    if (boxes) switch (p.d) {
            case 64: return least ? launch<T, 64, 16, true>(p, b, a, map, x, status, st) : mid ? launch<T, 64, 32, true>(p, b, a, map, x, status, st) : launch<T, 64, 64, true>(p, b, a, map, x, status, st);
            case 128: return least ? launch<T, 128, 16, true>(p, b, a, map, x, status, st) : mid ? launch<T, 128, 32, true>(p, b, a, map, x, status, st) : launch<T, 128, 64, true>(p, b, a, map, x, status, st);
            default: return least ? launch<T, 256, 16, true>(p, b, a, map, x, status, st) : launch<T, 256, 32, true>(p, b, a, map, x, status, st);
        }
    switch (p.d) {
        case 32: return least ? launch<T, 32, 16, false>(p, b, a, map, x, status, st) : mid ? launch<T, 32, 32, false>(p, b, a, map, x, status, st) : launch<T, 32, 64, false>(p, b, a, map, x, status, st);
        case 64: return least ? launch<T, 64, 16, false>(p, b, a, map, x, status, st) : mid ? launch<T, 64, 32, false>(p, b, a, map, x, status, st) : launch<T, 64, 64, false>(p, b, a, map, x, status, st);
        case 128: return least ? launch<T, 128, 16, false>(p, b, a, map, x, status, st) : mid ? launch<T, 128, 32, false>(p, b, a, map, x, status, st) : launch<T, 128, 64, false>(p, b, a, map, x, status, st);
        default: return least ? launch<T, 256, 16, false>(p, b, a, map, x, status, st) : launch<T, 256, 32, false>(p, b, a, map, x, status, st);
    }
}

}  // namespace
}  // namespace plc
