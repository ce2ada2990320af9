// Tree attention of many rows: wide trees, long drafts and chunks of prompts, where each K and V is read for 128 or 256 rows (a KV head's drafted tokens
// times its query heads) and the products and exponentials are the bound.
//
//   S = Q K^T        [128 rows x TN]      tcgen05.mma, both operands in shared memory, S in tensor memory: a lane a row
//   P = exp2(c S - m)                     a thread a row; P takes S's columns in tensor memory, in 16 bits
//   O = O + P V      [128 rows x d]       tcgen05.mma, P from tensor memory, V as it lies in the page (d contiguous)
//
// NT = 1: 128 rows, two CTAs an SM.  NT = 2: two row tiles that share each K and V tile, one CTA an SM: while the weights of one tile are
// formed, the products of the other run.  Masks are written into S first, so that the loops over the scores have none: a masked tile is rare where boxes
// fill a tile (pages that divide it); elsewhere every tile is one.
//
// Measured, bf16, 8 KV heads of 128 components.  131072 positions, 512 rows a KV head: the kernel by itself 310 us (885 TFLOP/s, 0.53 of the measured rate of a
// product by itself), call after call 341 to 351 us (under the power cap, 1650 MHz), each waited for 348 (1717 MHz), caches flushed between
// them 323 to 336 (1750 MHz).  37 sessions x 8192 x 256 rows 331 us at first, 397 call after call (1600 MHz); x 128 rows 234 and 250; 8 sessions x 8192 x 256 rows of 256
// components 221 and 234.  Without a mask every row tile goes through all of its session's positions: a chunk of 2048 behind nothing 179 us, behind 8192 positions
// 433.  Pages whose boxes do not fill a tile, 37 x 8192 x 256 rows: of 24 positions 478 us, of 72 761; position by position, of 100, 452.
// With NT = 2 a pair of tiles takes 4400 clocks, of which the tensor pipe is busy for 2050 and the exponentials' unit for 2050: a row tile's
// weights (2200 clocks in the softmax's four warps) and its products (1050) follow each other, with four signals between them, and tensor memory
// has no room for a second S beside two O.  What did not help: S in halves of 64 positions, each with its own turn (products of 64 and 128 columns in turn run at a third of
// the rate: 445 us); a quarter or a half of the exponentials by a polynomial on the multiply-add units (328 and 349 us); the scores held in registers between
// maximum and exponentials, with registers moved to the softmax (the same); a second thread that issues products (410 us).
#pragma once
#include "plc_attend.cuh"

namespace plc {
namespace {

constexpr int kWordRing = 8;                      // tiles whose validity words are kept: more than the copies can be ahead of the softmax

template <int D, int NT, bool BOX> struct Shape {
    static constexpr int TN = D == 256 ? 64 : 128;                     // positions a tile: S and O of a CTA's row tiles fit in tensor memory
    static constexpr int blocks = (D + 63) / 64;                       // 128-byte wide column blocks (32 components: half of one)
    static constexpr int DV = blocks * 64;                             // columns of O
    // tiles kept of K and of V: as many as fit, of K one more (its next tile is waited for first)
    static constexpr int vstages = D == 128 ? NT : NT == 1 ? 2 : BOX ? 4 : 3, kstages = BOX && (D != 128 || NT == 2) ? vstages + 1 : vstages;
    static constexpr int q_bytes = blocks * 128 * 128, kv_bytes = blocks * TN * 128;
    static constexpr int bufs = D == 256 ? 2 : 1;                      // of scores, a row tile: as many as fit
    static constexpr int tmem = NT * (bufs * TN + DV) > 256 ? 512 : 256;
    static constexpr int rows = NT * 128, soft = NT * 128, threads = soft + 128;
    static constexpr int per_sm = NT == 1 && D != 256 ? 2 : 1;
    static constexpr size_t smem = (size_t)NT * q_bytes + (kstages + vstages) * kv_bytes + (BOX ? 0 : 2 * TN * 8) + 1024 + 512;
};

// Scores of positions that the row does not see become -inf, in place.
template <int TN>
__device__ __noinline__ void hide_scores(uint32_t s_at, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3) {
#pragma unroll 1
    for (int e = 0; e < TN / 32; ++e) {
        const uint32_t vis = e == 0 ? v0 : e == 1 ? v1 : e == 2 ? v2 : v3;
        uint32_t x[32];
        tmem_ld32(s_at + 32 * e, x);
        wait_ld(x);
#pragma unroll
        for (int k = 0; k < 32; ++k) x[k] = vis >> k & 1u ? x[k] : 0xff800000u;
        tmem_st32(s_at + 32 * e, x);
    }
    wait_st();
}

// Adds what take_out has taken out of V at the drafted positions t0 .. t1 - 1 to what a row that sees them has written.
template <class T>
__device__ __noinline__ void put_back_row(const PoolDev& p, const BookDev& b, const AttendArgs& a, const Session x, int s, int h, int t0, int t1, int i, void* row, bool whole) {
    for (int t = max(t0, x.len); t < min(t1, x.kv); ++t) {
        if (!(seen_bits(a, x, i, t) & 1u)) continue;
        const int page = b.table[(int64_t)s * b.max_pages + t / p.page_pos];
        if (page < 0 || page >= p.n_pages) continue;
        const uint16_t* v = reinterpret_cast<const uint16_t*>(p.base + (int64_t)a.layer * p.sl + (int64_t)h * p.sh + p.skv + (int64_t)page * p.spage +
                                                              (int64_t)(t % p.page_pos) * p.sp);
        for (int d = 0; d < p.d; ++d) {
            if ((v[d] & Kind<T>::exponent) != Kind<T>::exponent) continue;
            if (whole) {
                uint16_t* o = static_cast<uint16_t*>(row) + d;
                *o = (uint16_t)(Kind<T>::pack(Kind<T>::widen(*o) + Kind<T>::widen(v[d]), 0.f) & 0xffffu);
            } else static_cast<float*>(row)[d] += Kind<T>::widen(v[d]);
        }
    }
}

template <class T, int D, int NT, bool BOX>
__global__ void __launch_bounds__(Shape<D, NT, BOX>::threads, Shape<D, NT, BOX>::per_sm)
many_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b, const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map, uint32_t* status) {
    using Sh = Shape<D, NT, BOX>;
    using Wk = Walk<Sh::rows>;
    constexpr int TN = Sh::TN, bufs = Sh::bufs, kst = Sh::kstages, vst = Sh::vstages, soft_warps = Sh::soft / 32, mma_warp = soft_warps + 3, loaders = BOX ? 64 : 96;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ks = smem + NT * Sh::q_bytes;
    uint8_t* vs = ks + kst * Sh::kv_bytes;
    int64_t* offs = reinterpret_cast<int64_t*>(vs + vst * Sh::kv_bytes);             // [2][TN], without boxes
    uint32_t* words = reinterpret_cast<uint32_t*>(offs + (BOX ? 0 : 2 * TN));                       // [kWordRing][4]
    uint64_t* bars = reinterpret_cast<uint64_t*>(words + kWordRing * 4);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * (kst + vst) + 3 + 3 * bufs * NT);
    volatile uint32_t* failed = tmem_slot + 1;
    // V that held infinities or NaN at drafted positions: [row tile][2] piece number + 1, by its parity (no warp is two pieces behind the others of its row
    // tile, but a row tile may be many behind the other); [kWordRing] tile number + 1, by which a row tile knows of what the other has taken out before it
    volatile uint32_t *dirty = tmem_slot + 2, *taken = dirty + 2 * NT;
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const uint32_t kfull = smem_u32(bars), vfull = kfull + 8 * kst, kempty = vfull + 8 * vst, vempty = kempty + 8 * kst;
    const uint32_t qfull = vempty + 8 * vst, qempty = qfull + 8, drain = qempty + 8, sfull = drain + 8, pfull = sfull + 8 * bufs * NT, ofull = pfull + 8 * bufs * NT;
    chain_next();
    if (tid == 0) {
        for (int i = 0; i < kst; ++i) {
            mbar_init(kfull + 8 * i, BOX ? 1 : loaders + loaders / 32);
            mbar_init(kempty + 8 * i, 1);
        }
        for (int i = 0; i < vst; ++i) {
            mbar_init(vfull + 8 * i, BOX ? 1 : loaders);
            mbar_init(vempty + 8 * i, 1);
        }
        mbar_init(qfull, BOX ? 32 : loaders);
        mbar_init(qempty, 1);
        mbar_init(drain, 1);
        for (int i = 0; i < bufs * NT; ++i) {
            mbar_init(sfull + 8 * i, 1);
            mbar_init(pfull + 8 * i, 4);
            mbar_init(ofull + 8 * i, 1);
        }
        for (int i = 1; i < 2 + 2 * NT + kWordRing; ++i) tmem_slot[i] = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == mma_warp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)Sh::tmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const int tile_pos = BOX ? a.tile_pos : TN;
    if (BOX && tile_pos < TN) {                   // positions of a tile that no box fills: zeros once and for all
        for (int i = tid; i < (kst + vst) * Sh::blocks * TN * 8; i += Sh::threads)      // pieces of 16 bytes as they lie there, eight a position
            if ((i >> 3) % TN >= tile_pos) *reinterpret_cast<uint4*>(ks + i * 16) = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    fence_before();
    Wk w{};
    long long left = find_range<Sh::rows, Sh::threads>(p, b, a, status, w);
    fence_after();
    const uint32_t tmem = *tmem_slot;
    const int me = blockIdx.x;
    const uint32_t q_s = smem_u32(smem), k_s = smem_u32(ks), v_s = smem_u32(vs);
    constexpr int pieces = D * 2 / 16;

    if (wid >= soft_warps && wid < mma_warp) {
        const int lt = tid - Sh::soft;
        int item = 0;
        // a piece's rows of Q, by `threads` threads, the first of them `lt0`: a thread has one piece of 16 bytes in every step-th row
        auto load_q = [&](const Wk& x, int threads, int lt0, bool ok) -> bool {
            ok = ok && mbar_wait(qempty, (uint32_t)(item & 1) ^ 1u, failed, status);
            ++item;
            if (!ok) return false;
            const int step = threads / pieces, r0 = (lt - lt0) / pieces, c = (lt - lt0) - r0 * pieces;
            const int rows = x.rows(a), i0 = (x.rt * Sh::rows + r0) / a.group, di = step / a.group, dg = step - di * a.group;
            int g = x.rt * Sh::rows + r0 - i0 * a.group;
            const int64_t wrap = 2 * (a.qs_row - (int64_t)a.group * a.qs_head), ahead = 2 * (di * a.qs_row + dg * a.qs_head);
            const uint8_t* src = static_cast<const uint8_t*>(a.q) + 2 * ((int64_t)(x.x.first + i0) * a.qs_row + (int64_t)(x.h * a.group + g) * a.qs_head) + c * 16;
            const uint32_t dst = q_s + (c >> 3) * 16384;
#pragma unroll 4
            for (int r = r0; r < Sh::rows; r += step) {
                copy16(dst + (r >> 7) * Sh::q_bytes + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4), r < rows ? src : static_cast<const uint8_t*>(a.q), r < rows);
                src += ahead;
                g += dg;
                if (g >= a.group) { g -= a.group; src += wrap; }
            }
            mbar_arrive_copies(qfull);
            return true;
        };
        if constexpr (BOX) {
            // ---- copies in boxes: a warp for the keys, one for the values, one for the queries, so that the next piece's tiles are on their way while
            // its queries wait for the last products of this one
            if (lt < 64) {
                const int kv = lt >> 5;
                copy_boxes<Sh::rows, Sh::blocks, TN>(p, b, a, map, w, left, kv, 0, 1, kv ? v_s : k_s, Sh::kv_bytes, kv ? vst : kst, kv ? vfull : kfull, kv ? vempty : kempty, words, kWordRing,
                                                     failed, status, [](const Tiles<Sh::rows>&, bool ok) -> bool { return ok; });
            } else {
                bool ok = true;
                while (left > 0 && ok) {
                    ok = __all_sync(kFull, load_q(w, 32, 64, ok));
                    left -= min(left, (long long)(w.tiles - w.tile));
                    if (left > 0) w.next_item(p, b, a);
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
            }
        } else {
            // ---- copies, three warps, position by position (pages of any size).  A tile's addresses are found by one thread a position and
            // passed on in shared memory.
            int done = 0;
            bool ok = true, go = true;                    // this thread's waits; all loaders' (they leave together: they share a barrier)
            while (left > 0 && go) {
                const int m = (int)min(left, (long long)(w.tiles - w.tile));
                const int32_t* row = b.table + (int64_t)w.s * b.max_pages;
                const uint8_t* kb = p.base + (int64_t)a.layer * p.sl + (int64_t)w.h * p.sh;
                ok = load_q(w, loaders, 0, ok);
                for (int j = 0; j < m; ++j, ++done) {
                    const int st = done % kst;                   // without boxes the rings are alike
                    const uint32_t ph = (uint32_t)(done / kst) & 1u;
                    int64_t* off = offs + (done & 1) * TN;
                    uint32_t valid[2] = {0, 0};
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int word = (lt >> 5) + e * (loaders / 32);
                        if (word >= TN / 32) break;
                        const int t = (w.tile + j) * TN + word * 32 + lane;
                        bool have = t < w.x.kv;
                        int64_t at = 0;
                        if (have) {
                            const int pg = t / p.page_pos, page = row[pg];
                            if (page >= 0 && page < p.n_pages) at = (int64_t)page * p.spage + (int64_t)(t - pg * p.page_pos) * p.sp;
                            else { have = false; atomicOr(status, kStRange); }
                        }
                        off[word * 32 + lane] = have ? at : INT64_MIN;
                        valid[e] = __ballot_sync(kFull, have);
                    }
                    ok = ok && mbar_wait(kempty + 8 * st, ph ^ 1u, failed, status);
                    uint32_t all;
                    asm volatile(
                        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
                        "barrier.cta.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                        : "=r"(all) : "r"((uint32_t)ok), "n"(loaders) : "memory");
                    go = all != 0;
                    if (!go) break;
                    if (lane == 0) {
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if ((lt >> 5) + e * (loaders / 32) < TN / 32) words[(done % kWordRing) * 4 + (lt >> 5) + e * (loaders / 32)] = valid[e];
                    }
#pragma unroll 8
                    for (int u = lt; u < TN * pieces; u += loaders) {
                        const int r = u / pieces, c = u % pieces;
                        const int64_t o = off[r];
                        copy16(k_s + st * Sh::kv_bytes + (c >> 3) * (TN * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), o == INT64_MIN ? kb : kb + o + c * 16, o != INT64_MIN);
                    }
                    mbar_arrive_copies(kfull + 8 * st);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(kfull + 8 * st);            // the validity words, too, are there
                    ok = mbar_wait(vempty + 8 * st, ph ^ 1u, failed, status);
                    if (ok) {
#pragma unroll 8
                        for (int u = lt; u < TN * pieces; u += loaders) {
                            const int r = u / pieces, c = u % pieces;
                            const int64_t o = off[r];
                            copy16(v_s + st * Sh::kv_bytes + (c >> 3) * (TN * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4),
                                   o == INT64_MIN ? kb : kb + p.skv + o + c * 16, o != INT64_MIN);
                        }
                        mbar_arrive_copies(vfull + 8 * st);
                    }
                }
                left -= m;
                if (left > 0) w.next_item(p, b, a);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
    } else if (wid == mma_warp) {
        if (lane == 0) {
            // ---- products: the scores of the first tiles, as many as there are buffers for; then for every tile P V and the scores of the tile that takes
            // the columns of that P, the row tiles in turn.  They run in the order in which they are issued.
            constexpr uint32_t common = (1u << 4) | (Kind<T>::format << 7) | (Kind<T>::format << 10) | (8u << 24);
            constexpr uint32_t id_qk = common | ((uint32_t)(TN >> 3) << 17), id_pv = common | (1u << 16) | ((uint32_t)(Sh::DV >> 3) << 17);
            int kd = 0, vd = 0, item = 0;
            uint32_t cs = 0, cp = 0;                   // scores and products P V, modulo 4, a byte a row tile
            auto next = [](uint32_t& c, int n) -> uint32_t {
                const uint32_t v = c >> (8 * n) & 3u;
                c = (c & ~(3u << (8 * n))) | ((v + 1u) & 3u) << (8 * n);
                return v;
            };
            bool ok = true;
            auto qk = [&](int n, bool last) {
                const int st = kd % kst, at = n * bufs + (int)(next(cs, n) % bufs);
                const uint32_t s_at = tmem + at * TN;
                const uint64_t q_at = desc_k(q_s + n * Sh::q_bytes), k_at = desc_k(k_s + st * Sh::kv_bytes);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_ss(s_at, q_at + (k >> 2) * (16384 >> 4) + 2 * (k & 3), k_at + (k >> 2) * (TN * 128 >> 4) + 2 * (k & 3), id_qk, k ? 1u : 0u);
                mma_commit(sfull + 8 * at);
                if (last) { mma_commit(kempty + 8 * st); ++kd; }
            };
            auto wait_k = [&]() {
                ok = ok && mbar_wait(kfull + 8 * (kd % kst), (uint32_t)(kd / kst) & 1u, failed, status);
                // boxes and products are of one proxy; what threads wrote to V is fenced by those who wrote it
                if (!BOX) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            };
            while (left > 0 && ok) {
                const int m = (int)min(left, (long long)(w.tiles - w.tile)), nt = NT == 2 && w.rows(a) > 128 ? 2 : 1;
                ok = mbar_wait(qfull, (uint32_t)(item & 1), failed, status);
                if (BOX) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                for (int j = 0; j < bufs && j < m && ok; ++j) {
                    wait_k();
                    if (!ok) break;
                    fence_after();
                    for (int n = 0; n < nt; ++n) qk(n, n == nt - 1);
                }
                if (m <= bufs) mma_commit(qempty);
                for (int j = 0; j < m && ok; ++j, ++vd) {
                    const int st = vd % vst;
                    const bool more = j + bufs < m;
                    // the tiles first: they are there long before the weights, and the time from the weights to the next scores counts
                    ok = mbar_wait(vfull + 8 * st, (uint32_t)(vd / vst) & 1u, failed, status);
                    if (more) wait_k();
                    if (!BOX) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    const uint64_t v_at = desc_mn(v_s + st * Sh::kv_bytes, TN * 128);
                    for (int n = 0; n < nt && ok; ++n) {
                        const uint32_t turn = next(cp, n);
                        const int at = n * bufs + (int)(turn % bufs);
                        ok = mbar_wait(pfull + 8 * at, turn / bufs & 1u, failed, status);
                        if (!ok) break;
                        fence_after();
                        const uint32_t o_at = tmem + NT * bufs * TN + n * Sh::DV, p_at = tmem + at * TN;
#pragma unroll
                        for (int k = 0; k < TN / 16; ++k) mma_ts(o_at, p_at + 8 * k, v_at + k * (2048 >> 4), id_pv, j | k ? 1u : 0u);
                        mma_commit(ofull + 8 * at);
                        if (n == nt - 1) mma_commit(vempty + 8 * st);
                        if (more) {
                            qk(n, n == nt - 1);
                            if (j + bufs + 1 == m && n == nt - 1) mma_commit(qempty);
                        }
                    }
                }
                left -= m;
                ++item;
                if (left > 0) w.next_item(p, b, a);
            }
            mma_commit(drain);                        // nothing issued runs when the CTA frees its TMEM
            for (uint32_t i = 0; i < kSpin; ++i) {
                uint32_t done;
                asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], 0;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(drain) : "memory");
                if (done) break;
            }
        }
    } else if (wid < soft_warps) {
        // ---- softmax and results: a thread a row
        const int nt = wid >> 2, r_tile = (wid & 3) * 32 + lane, r_item = nt * 128 + r_tile;
        const uint32_t lanes = (uint32_t)((wid & 3) * 32) << 16, s_0 = tmem + nt * bufs * TN + lanes, o_at = tmem + NT * bufs * TN + nt * Sh::DV + lanes;
        const float c = a.scale * 1.44269504088896f;
        const unsigned long long c2 = pack2(c, c);
        int done = 0, tiles_done = 0, part = 0;       // tiles of this row tile, of the CTA
        bool ok = true;
        // the last product of the row tile, and so all before it.  Two buffers have a barrier each: of two products on their way one parity would not tell.
        auto wait_o = [&]() -> bool {
            return __all_sync(kFull, mbar_wait(ofull + 8 * (nt * bufs + (done - 1) % bufs), (uint32_t)((done - 1) / bufs) & 1u, failed, status));
        };
        while (left > 0 && ok) {
            const int m = (int)min(left, (long long)(w.tiles - w.tile)), rows = w.rows(a);
            const bool in_use = nt == 0 || rows > 128, works = r_tile - lane + nt * 128 < rows;   // the row tile; this warp
            const int rr = w.rt * Sh::rows + r_item, i = rr / a.group;
            float top = -INFINITY, sum = 0.f;         // top: what the weights are relative to, scaled, base 2
            const bool may_hide = a.mask != nullptr || w.x.n > 1;
            for (int j = 0; j < m && in_use; ++j, ++done) {
                const int t = (w.tile + j) * tile_pos, buf = done % bufs;
                const uint32_t s_at = s_0 + buf * TN;
                ok = __all_sync(kFull, mbar_wait(sfull + 8 * (nt * bufs + buf), (uint32_t)(done / bufs) & 1u, failed, status));
                if (!ok) break;
                fence_after();
                const uint32_t* valid = words + ((tiles_done + j) % kWordRing) * 4;
                const bool drafted = t + tile_pos > w.x.len, hide = may_hide && drafted;
                bool masked = hide;
#pragma unroll
                for (int e = 0; e < TN / 32; ++e) masked |= valid[e] != ~0u;
                if (works) {
                    if (masked) {
                        uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int e = 0; e < TN / 32; ++e) v[e] = valid[e] & (!hide ? ~0u : r_item < rows ? seen_bits(a, w.x, i, t + 32 * e) : 0u);
                        hide_scores<TN>(s_at, v[0], v[1], v[2], v[3]);
                    }
                    float x_top = -INFINITY;
#pragma unroll
                    for (int e = 0; e < TN / 32; ++e) {
                        uint32_t x[32];
                        tmem_ld32(s_at + 32 * e, x);
                        wait_ld(x);
                        float y = -INFINITY;
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            x_top = max3(x_top, __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
                            y = max3(y, __uint_as_float(x[k + 2]), __uint_as_float(x[k + 3]));
                        }
                        x_top = fmaxf(x_top, y);
                    }
                    const float now = x_top * c;
                    const bool raise = now > top + kRaise;            // also the first finite score
                    if (__any_sync(kFull, raise)) {
                        const float f = raise && top > -INFINITY ? exp2_approx(top - now) : raise ? 0.f : 1.f;
                        if (raise) top = now;
                        sum *= f;
                        if (j > 0) {
                            ok = wait_o();
                            if (!ok) break;
                            fence_after();
#pragma unroll 1
                            for (int e = 0; e < Sh::DV / 32; ++e) {
                                uint32_t o[32];
                                tmem_ld32(o_at + 32 * e, o);
                                wait_ld(o);
#pragma unroll
                                for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(f == 0.f ? 0.f : __uint_as_float(o[k]) * f);
                                tmem_st32(o_at + 32 * e, o);
                            }
                        }
                    }
                    const float base = top == -INFINITY ? 0.f : Kind<T>::shift - top;
                    const unsigned long long base2 = pack2(base, base);
                    unsigned long long s0 = 0ull, s1 = 0ull;
#pragma unroll
                    for (int e = 0; e < TN / 32; ++e) {
                        uint32_t x[32], y[16];
                        tmem_ld32(s_at + 32 * e, x);
                        wait_ld(x);
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            float e0, e1, e2, e3;
                            unpack2(fma2(pack2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), c2, base2), e0, e1);
                            unpack2(fma2(pack2(__uint_as_float(x[k + 2]), __uint_as_float(x[k + 3])), c2, base2), e2, e3);
                            e0 = exp2_approx(e0); e1 = exp2_approx(e1); e2 = exp2_approx(e2); e3 = exp2_approx(e3);   // a score of -inf has the weight 0
                            s0 = add2(s0, pack2(e0, e1));
                            s1 = add2(s1, pack2(e2, e3));
                            y[k / 2] = Kind<T>::pack(e0, e1);
                            y[k / 2 + 1] = Kind<T>::pack(e2, e3);
                        }
                        tmem_st16(s_at + 16 * e, y);
                    }
                    float lo, hi;
                    unpack2(add2(s0, s1), lo, hi);
                    sum += lo + hi;
                    wait_st();
                }
                if (hide || (BOX && masked)) {
                    // V of positions that do not exist is whatever the boxes brought or left: zeros instead, since weights of 0 do not hide it; and
                    // what drafted positions have of infinities and NaN is taken out.  Both row tiles do the same to it.
                    const int st = (tiles_done + j) % vst, pos = r_tile;
                    ok = __all_sync(kFull, mbar_wait(vfull + 8 * st, (uint32_t)((tiles_done + j) / vst) & 1u, failed, status));
                    if (!ok) break;
                    uint8_t* tile = vs + st * Sh::kv_bytes;
                    if (pos < min(TN, tile_pos)) {
                        const bool there = valid[pos >> 5] >> (pos & 31) & 1u;
                        if (BOX && !there)
                            for (int e = 0; e < Sh::blocks * 8; ++e)
                                *reinterpret_cast<uint4*>(tile + (e >> 3) * (TN * 128) + pos * 128 + (((e & 7) ^ (pos & 7)) << 4)) = make_uint4(0, 0, 0, 0);
                        else if (hide && t + pos >= w.x.len && t + pos < w.x.kv) {
                            const bool found = special<T, D, TN>(tile, pos);
                            __threadfence_block();            // who finds the zeros finds the word
                            volatile uint32_t& word = taken[(tiles_done + j) % kWordRing];
                            if (found || word == (uint32_t)(tiles_done + j) + 1u) dirty[2 * nt + (part & 1)] = (uint32_t)part + 1u;
                            if (found) {
                                word = (uint32_t)(tiles_done + j) + 1u;
                                __threadfence_block();
                                take_out<T, D, TN>(tile, pos);
                            }
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pfull + 8 * (nt * bufs + buf));
            }
            tiles_done += m;
            if (ok && in_use) ok = wait_o();
            if (!ok) break;
            if (in_use && works) {
                fence_after();
                const bool whole = w.tile == 0 && m == w.tiles, live = r_item < rows;
                const int64_t n_row = w.x.first + i, head = (int64_t)w.h * a.group + (rr - i * a.group), slot = ((int64_t)2 * me + (part > 0)) * a.part_rows + r_item;
                const float inv = sum == 0.f ? 0.f : 1.f / sum;       // 0: nothing was seen, whatever the product made of it
                uint16_t* out = static_cast<uint16_t*>(a.out) + n_row * a.os_row + head * a.os_head;
                float* mid = a.part_o + slot * D;
#pragma unroll 1
                for (int e = 0; e < (D + 31) / 32; ++e) {
                    uint32_t o[32];
                    tmem_ld32(o_at + 32 * e, o);
                    wait_ld(o);
                    if (!live) continue;
                    if (sum == 0.f) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = 0u;
                    }
                    if (whole) {
                        uint4* dst = reinterpret_cast<uint4*>(out + 32 * e);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t y[4];
#pragma unroll
                            for (int l = 0; l < 4; ++l) y[l] = Kind<T>::pack(__uint_as_float(o[8 * k + 2 * l]) * inv, __uint_as_float(o[8 * k + 2 * l + 1]) * inv);
                            dst[k] = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    } else {
                        uint4* dst = reinterpret_cast<uint4*>(mid + 32 * e);
#pragma unroll
                        for (int k = 0; k < 8; ++k) dst[k] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                    }
                }
                if (live) {
                    if (may_hide && dirty[2 * nt + (part & 1)] == (uint32_t)part + 1u)
                        put_back_row<T>(p, b, a, w.x, w.s, w.h, w.tile * tile_pos, (w.tile + m) * tile_pos, i, whole ? static_cast<void*>(out) : mid, whole);
                    if (!whole) a.part_ml[slot] = make_float2(top, sum);
                    else if (a.lse) a.lse[n_row * a.heads + head] = sum == 0.f ? -INFINITY : (top - Kind<T>::shift + log2f(sum)) * 0.693147180559945f;
                }
                fence_before();
            }
            left -= m;
            ++part;
            if (left > 0) w.next_item(p, b, a);
        }
    }
    fence_before();
    __syncthreads();
    if (wid == mma_warp) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)Sh::tmem) : "memory");
    }
}

template <class T, int D, int NT, bool BOX>
cudaError_t launch_many_as(const PoolDev& p, const BookDev& b, const AttendArgs& a, const CUtensorMap& map, const AttendPlan& x, uint32_t* status, cudaStream_t st) {
    using Sh = Shape<D, NT, BOX>;
    cudaError_t e = cudaFuncSetAttribute(many_kernel<T, D, NT, BOX>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Sh::smem);
    if (e != cudaSuccess) return e;
    e = launch_kernel(many_kernel<T, D, NT, BOX>, a.whole && a.whole < x.grid ? a.whole : x.grid, Sh::threads, Sh::smem, st, false, 1, p, b, a, map, status);
    return e != cudaSuccess || a.whole ? e : launch_join<T, D, Sh::rows>(p, b, a, x, st);
}
template <class T>
cudaError_t launch_many(const PoolDev& p, const BookDev& b, const AttendArgs& args, const AttendPlan& x, bool bf16, uint32_t* status, cudaStream_t st) {
    AttendArgs a = args;
    a.tile_pos = p.d == 256 ? 64 : 128;
    CUtensorMap map{};
    const bool boxes = make_boxes(p, a, bf16, a.tile_pos, &map), two = x.row_tile == 256;
    if (boxes) switch (p.d) {
            case 64: return two ? launch_many_as<T, 64, 2, true>(p, b, a, map, x, status, st) : launch_many_as<T, 64, 1, true>(p, b, a, map, x, status, st);
            case 128: return two ? launch_many_as<T, 128, 2, true>(p, b, a, map, x, status, st) : launch_many_as<T, 128, 1, true>(p, b, a, map, x, status, st);
            default: return launch_many_as<T, 256, 1, true>(p, b, a, map, x, status, st);
        }
    switch (p.d) {
        case 32: return two ? launch_many_as<T, 32, 2, false>(p, b, a, map, x, status, st) : launch_many_as<T, 32, 1, false>(p, b, a, map, x, status, st);
        case 64: return two ? launch_many_as<T, 64, 2, false>(p, b, a, map, x, status, st) : launch_many_as<T, 64, 1, false>(p, b, a, map, x, status, st);
        case 128: return two ? launch_many_as<T, 128, 2, false>(p, b, a, map, x, status, st) : launch_many_as<T, 128, 1, false>(p, b, a, map, x, status, st);
        default: return launch_many_as<T, 256, 1, false>(p, b, a, map, x, status, st);
    }
}

}  // namespace
}  // namespace plc
