// Tree attention of few rows: single tokens, short drafts and small trees, where each K and V is read for at most 64 rows (a KV head's drafted
// tokens times its query heads) and HBM is the bound.
//
// The products are turned round, so that the 128 lanes of tensor memory are positions, not rows that are mostly empty:
//   S = K Q^T     [128 positions x N]      a lane a position, a column a row; N = the rows rounded up to 16
//   P = exp2(c S - m)                      a thread a position: the exponentials of a tile are spread over all four warps
//   O = O + V^T P [d x N]                  V as it lies in the page, P through shared memory
// Per tile that is N / 128 of the other layout's work in the products and the softmax, which leaves the copies ahead: they run in one
// ring of tiles (K of the next tile before V of this one) that does not stop between items, Q has two buffers, and S two, so that the
// scores of a tile are formed while the one before is in the softmax.
// A row's maximum is common to the CTA and raised only where some score passes it by 2^3 (a vote of the four warps a tile); each thread sums the
// weights of its positions, and the sums are joined at the end of an item.
#include "plc_attend.cuh"

namespace plc {
namespace {

constexpr int kTN = 128, kSoft = 128, kCopy = 128, kFewThreads = kSoft + kCopy + 32;
constexpr int kWords = 16;                        // tiles whose validity words are kept: more than the ring holds

template <int D> struct Few {
    static constexpr int N = D == 256 ? 32 : 64;                       // most rows
    static constexpr int blocks = (D + 63) / 64;                       // 128-byte wide column blocks (32 components: half of one)
    static constexpr int slot = blocks * kTN * 128, slots = D == 256 ? 3 : D == 128 ? 4 : 8;
    static constexpr int q_bytes = blocks * N * 128, q_bufs = D == 256 ? 1 : 2;
    static constexpr int p_bytes = N * kTN * 2, p_bufs = D == 256 ? 1 : 2;
    static constexpr int o_blocks = D == 256 ? 2 : 1;
    static constexpr int tmem = 256;                                   // S twice, O
    static constexpr size_t smem = (size_t)q_bufs * q_bytes + p_bufs * p_bytes + slots * slot + 3 * kTN * 8 + 4096 + 1024;
};

__device__ __forceinline__ bool vote(uint32_t mine, bool all) {        // of the four softmax warps
    uint32_t r;
    if (all)
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(mine) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(mine) : "memory");
    return r != 0;
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ float warp_max(float x) {
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
// P: blocks of 8 rows, in each 16 bytes a position (MN-major without swizzle: 128 bytes from eight positions to the next eight,
// 2048 from eight rows to the next eight).
__device__ __forceinline__ uint64_t desc_p(uint32_t addr) { return (uint64_t)((addr & 0x3FFFFu) >> 4) | (8ull << 16) | (128ull << 32) | (1ull << 46); }

template <class T, int D>
__global__ void __launch_bounds__(kFewThreads, 1) few_kernel(PoolDev p, BookDev b, const __grid_constant__ AttendArgs a, uint32_t* status) {
    using F = Few<D>;
    using Tl = Tiles<kTN, F::N>;
    constexpr int N = F::N, chunks = N / 16, slots = F::slots;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* qs = ring + slots * F::slot;
    uint8_t* ps = qs + F::q_bufs * F::q_bytes;
    int64_t* offs = reinterpret_cast<int64_t*>(ps + F::p_bufs * F::p_bytes);            // [3][kTN]
    int64_t* row_at = offs + 3 * kTN;                                                   // [N] where a row of the result goes
    uint64_t* bars = reinterpret_cast<uint64_t*>(row_at + N);
    float* base_s = reinterpret_cast<float*>(bars + 2 * slots + 12);                    // [N] what the weights' exponents are relative to
    float* top_s = base_s + N;                                                          // [N] maximum (scaled, base 2)
    float* factor_s = top_s + N;                                                        // [N]
    float* warp_s = factor_s + N;                                                       // [4][N]
    uint32_t* words = reinterpret_cast<uint32_t*>(warp_s + 4 * N);                      // [kWords][4] positions that exist
    uint32_t* tmem_slot = words + kWords * 4;
    volatile uint32_t* failed = tmem_slot + 1;
    volatile uint32_t* dirty = tmem_slot + 2;     // number + 1 of the last piece whose V holds infinities or NaN at drafted positions
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const uint32_t full = smem_u32(bars), empty = full + 8 * slots, qfull = empty + 8 * slots, qempty = qfull + 16, sfull = qempty + 16, pfull = sfull + 16,
                   ofull = pfull + 16, drain = ofull + 16;
    chain_next();
    if (tid == 0) {
        for (int i = 0; i < slots; ++i) { mbar_init(full + 8 * i, kCopy + kCopy / 32); mbar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(qfull + 8 * i, kCopy);
            mbar_init(qempty + 8 * i, 1);
            mbar_init(sfull + 8 * i, 1);
            mbar_init(pfull + 8 * i, kSoft / 32);
            mbar_init(ofull + 8 * i, 1);
        }
        mbar_init(drain, 1);
        *failed = *dirty = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    constexpr int mma_warp = kFewThreads / 32 - 1;
    if (wid == mma_warp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)F::tmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    Walk<kTN, N> w0{};
    const long long total = find_range<kTN, N, kFewThreads>(p, b, a, status, w0);
    fence_after();
    const uint32_t tmem = *tmem_slot, ring_s = smem_u32(ring), q_s = smem_u32(qs), p_s = smem_u32(ps);

    if (wid >= 4 && wid < mma_warp) {
        // ---- copies
        const int lt = tid - kSoft;
        constexpr int pieces = D / 8, step = kCopy / pieces;                // 16-byte pieces of a vector; vectors a round
        const int c = lt % pieces, r0 = lt / pieces;
        Tl kx, vx;
        kx.start(w0, total);
        vx.start(w0, total);
        int kt = 0, vt = 0, sl = 0;
        bool ok = true;
        auto fill = [&](const uint8_t* src, const int64_t* off) {            // a tile into the next slot of the ring
            const int s = sl % slots;
            ok = __all_sync(kFull, ok && mbar_wait(empty + 8 * s, ((uint32_t)(sl / slots) & 1u) ^ 1u, failed, status));
            ++sl;
            if (!ok) return;
            const uint32_t dst = ring_s + s * F::slot + (c >> 3) * (kTN * 128);
            const uint8_t* mine = src + c * 16;
#pragma unroll
            for (int k = 0; k < kTN / step; ++k) {
                const int r = r0 + k * step;
                const int64_t o = off[r];
                copy16(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4), o == INT64_MIN ? src : mine + o, o != INT64_MIN);
            }
            mbar_arrive_copies(full + 8 * s);
            __syncwarp();
            if (lane == 0) mbar_arrive(full + 8 * s);                        // the validity words, too, are there
        };
        for (;;) {
            const bool more = kx.more();
            if (!more && !vx.more()) break;
            if (more) {
                if (kx.j == 0) {
                    const int q = kx.piece % F::q_bufs, rows = kx.w.rows(a), up = (rows + 15) & ~15;
                    ok = ok && mbar_wait(qempty + 8 * q, ((uint32_t)(kx.piece / F::q_bufs) & 1u) ^ 1u, failed, status);
                    if (ok) {
                        for (int r = r0; r < up; r += step) {
                            const int rr = kx.w.rt * N + r, i = rr / a.group, g = rr - i * a.group;
                            const uint8_t* src = static_cast<const uint8_t*>(a.q);
                            if (r < rows) src += 2 * ((int64_t)(kx.w.x.first + i) * a.qs_row + (int64_t)(kx.w.h * a.group + g) * a.qs_head) + c * 16;
                            copy16(q_s + q * F::q_bytes + (c >> 3) * (N * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), src, r < rows);
                        }
                        mbar_arrive_copies(qfull + 8 * q);
                    }
                }
                const int t = (kx.w.tile + kx.j) * kTN + lt;
                bool have = t < kx.w.x.kv;
                int64_t at = 0;
                if (have) {
                    const int pg = t / p.page_pos, page = b.table[(int64_t)kx.w.s * b.max_pages + pg];
                    if (page >= 0 && page < p.n_pages) at = (int64_t)page * p.spage + (int64_t)(t - pg * p.page_pos) * p.sp;
                    else { have = false; atomicOr(status, kStRange); }
                }
                offs[kt % 3 * kTN + lt] = have ? at : INT64_MIN;
                const uint32_t valid = __ballot_sync(kFull, have);
                if (lane == 0) words[kt % kWords * 4 + (lt >> 5)] = valid;
            }
            uint32_t all;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                         : "=r"(all) : "r"((uint32_t)ok) : "memory");
            if (!all) break;
            if (more) {
                fill(p.base + (int64_t)a.layer * p.sl + (int64_t)kx.w.h * p.sh, offs + kt % 3 * kTN);
                ++kt;
                kx.next(p, b, a);
            }
            if (kt > 1 || !more) {                                           // V of a tile after K of the next
                fill(p.base + (int64_t)a.layer * p.sl + (int64_t)vx.w.h * p.sh + p.skv, offs + vt % 3 * kTN);
                ++vt;
                vx.next(p, b, a);
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (wid == mma_warp) {
        if (lane == 0 && total > 0) {
            // ---- products
            constexpr uint32_t common = (1u << 4) | (Kind<T>::format << 7) | (Kind<T>::format << 10) | (8u << 24);
            Tl qx, vx;
            qx.start(w0, total);
            vx.start(w0, total);
            int sl = 0;
            bool ok = true;
            auto ready = [&]() {                      // the next slot of the ring
                ok = ok && mbar_wait(full + 8 * (sl % slots), (uint32_t)(sl / slots) & 1u, failed, status);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                fence_after();
            };
            auto columns = [&](const Tl& x) { return (uint32_t)((x.w.rows(a) + 15) & ~15); };
            auto qk = [&](int x) {
                const int q = qx.piece % F::q_bufs;
                if (qx.j == 0) ok = ok && mbar_wait(qfull + 8 * q, (uint32_t)(qx.piece / F::q_bufs) & 1u, failed, status);
                ready();
                if (!ok) return;
                const uint32_t k_at = ring_s + sl % slots * F::slot, q_at = q_s + q * F::q_bytes, id = common | (columns(qx) >> 3 << 17);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_ss(tmem + (x & 1) * N, desc_k(k_at + (k >> 2) * (kTN * 128)) + 2 * (k & 3), desc_k(q_at + (k >> 2) * (N * 128)) + 2 * (k & 3), id, k ? 1u : 0u);
                mma_commit(sfull + 8 * (x & 1));
                mma_commit(empty + 8 * (sl % slots));
                if (qx.last()) mma_commit(qempty + 8 * q);
                ++sl;
                qx.next(p, b, a);
            };
            qk(0);
            for (int x = 0; vx.more() && ok; ++x) {
                if (qx.more()) qk(x + 1);
                ok = ok && mbar_wait(pfull + 8 * (x & 1), (uint32_t)(x >> 1) & 1u, failed, status);
                ready();
                if (!ok) break;
                const uint32_t v_at = ring_s + sl % slots * F::slot, p_at = p_s + x % F::p_bufs * F::p_bytes, id = common | (3u << 15) | (columns(vx) >> 3 << 17);
#pragma unroll
                for (int o = 0; o < F::o_blocks; ++o)
#pragma unroll
                    for (int k = 0; k < kTN / 16; ++k)               // lanes past the components of a vector take the first block again
                        mma_ss(tmem + 2 * N + o * N, desc_mn(v_at + o * 2 * kTN * 128 + k * 2048, D >= 128 ? kTN * 128 : 0), desc_p(p_at + k * 256), id, vx.j | k ? 1u : 0u);
                mma_commit(ofull + 8 * (x & 1));
                mma_commit(empty + 8 * (sl % slots));
                ++sl;
                vx.next(p, b, a);
            }
            mma_commit(drain);                        // nothing issued runs when the CTA frees its tensor memory
            for (uint32_t i = 0; i < kSpin; ++i) {
                uint32_t done;
                asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], 0;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(drain) : "memory");
                if (done) break;
            }
        }
    } else {
        // ---- softmax and results: a thread a position, then a component
        const uint32_t lanes = (uint32_t)(wid * 32) << 16;
        const float c = a.scale * 1.44269504088896f;
        Tl sx;
        sx.start(w0, total);
        float sum[N];
        bool ok = true;
        for (int x = 0; sx.more(); ++x, sx.next(p, b, a)) {
            const Session& ses = sx.w.x;
            const int rows = sx.w.rows(a), n_ch = (rows + 15) >> 4, t0 = (sx.w.tile + sx.j) * kTN, t = t0 + tid, row0 = sx.w.rt * N;
            const bool first = sx.j == 0, may_hide = a.mask != nullptr || ses.n > 1;
            ok = ok && mbar_wait(sfull + 8 * (x & 1), (uint32_t)(x >> 1) & 1u, failed, status);
            if (x >= F::p_bufs) ok = ok && mbar_wait(ofull + 8 * ((x - F::p_bufs) & 1), (uint32_t)((x - F::p_bufs) >> 1) & 1u, failed, status);
            ok = __all_sync(kFull, ok);
            fence_after();
            uint32_t s[N];
#pragma unroll
            for (int ch = 0; ch < chunks; ++ch)
                if (ch < n_ch) tmem_ld16(tmem + (x & 1) * N + lanes + 16 * ch, s + 16 * ch);
            wait_ld(s);
            const uint32_t* valid = words + x % kWords * 4;
            const bool masked = t0 + kTN > ses.len || (valid[0] & valid[1] & valid[2] & valid[3]) != ~0u;
            uint32_t vis[(N + 31) / 32];
            if (masked) {                             // a lane finds what a row sees of the warp's 32 positions; a ballot a position turns that round
#pragma unroll
                for (int e = 0; e < (N + 31) / 32; ++e) {
                    const int r = 32 * e + lane;
                    uint32_t see = 0;
                    if (r < rows) see = valid[wid] & seen_bits(a, ses, (row0 + r) / a.group, t0 + 32 * wid);
                    vis[e] = 0;
                    for (int k = 0; k < 32; ++k) {
                        const uint32_t who = __ballot_sync(kFull, see >> k & 1u);
                        if (k == lane) vis[e] = who;
                    }
                }
#pragma unroll
                for (int r = 0; r < N; ++r) s[r] = vis[r >> 5] >> (r & 31) & 1u ? s[r] : 0xff800000u;
            }
            bool need = first || !ok;
            if (!first) {
#pragma unroll
                for (int ch = 0; ch < chunks; ++ch)
                    if (ch < n_ch) {
#pragma unroll
                        for (int r = 16 * ch; r < 16 * ch + 16; ++r) need |= __uint_as_float(s[r]) * c > top_s[r] + kRaise;
                    }
            }
            if (vote(need, false)) {
                // some row's maximum rises: all warps' maxima, the factors, and what has been summed so far
#pragma unroll
                for (int ch = 0; ch < chunks; ++ch)
                    if (ch < n_ch) {
#pragma unroll
                        for (int r = 16 * ch; r < 16 * ch + 16; ++r) {
                            const float m = warp_max(__uint_as_float(s[r]));
                            if (lane == (r & 31)) warp_s[wid * N + r] = m;
                        }
                    }
                if (!first) ok = ok && mbar_wait(ofull + 8 * ((x - 1) & 1), (uint32_t)((x - 1) >> 1) & 1u, failed, status);
                if (!vote(ok, true)) { ok = false; break; }
                if (tid < N) {
                    const float now = fmaxf(fmaxf(warp_s[tid], warp_s[N + tid]), fmaxf(warp_s[2 * N + tid], warp_s[3 * N + tid])) * c;
                    const float old = first ? -INFINITY : top_s[tid];
                    const float top = now > old + kRaise ? now : old;
                    top_s[tid] = top;
                    base_s[tid] = top == -INFINITY ? 0.f : top - Kind<T>::shift;
                    factor_s[tid] = top == old ? 1.f : old == -INFINITY ? 0.f : exp2_approx(old - top);
                }
                vote(1u, true);
                if (first) {
#pragma unroll
                    for (int r = 0; r < N; ++r) sum[r] = 0.f;
                } else {
                    fence_after();
#pragma unroll
                    for (int ch = 0; ch < chunks; ++ch)
                        if (ch < n_ch) {
#pragma unroll
                            for (int r = 16 * ch; r < 16 * ch + 16; ++r) sum[r] *= factor_s[r];
                            for (int o = 0; o < F::o_blocks; ++o) {
                                uint32_t y[16];
                                const uint32_t at = tmem + 2 * N + o * N + lanes + 16 * ch;
                                tmem_ld16(at, y);
                                wait_ld(y);
#pragma unroll
                                for (int r = 0; r < 16; ++r) {
                                    const float f = factor_s[16 * ch + r];
                                    y[r] = __float_as_uint(f == 0.f ? 0.f : __uint_as_float(y[r]) * f);
                                }
                                tmem_st16(at, y);
                            }
                        }
                    wait_st();
                }
            }
            uint8_t* pp = ps + x % F::p_bufs * F::p_bytes + tid * 16;
#pragma unroll
            for (int ch = 0; ch < chunks; ++ch)
                if (ch < n_ch) {
                    uint32_t y[8];
#pragma unroll
                    for (int r = 16 * ch; r < 16 * ch + 16; ++r) {
                        float v = exp2_approx(fmaf(__uint_as_float(s[r]), c, -base_s[r]));
                        if (masked) v = vis[r >> 5] >> (r & 31) & 1u ? v : 0.f;
                        sum[r] += v;
                        s[r] = __float_as_uint(v);
                    }
#pragma unroll
                    for (int r = 0; r < 8; ++r) y[r] = Kind<T>::pack(__uint_as_float(s[16 * ch + 2 * r]), __uint_as_float(s[16 * ch + 2 * r + 1]));
                    *reinterpret_cast<uint4*>(pp + (2 * ch) * 2048) = make_uint4(y[0], y[1], y[2], y[3]);
                    *reinterpret_cast<uint4*>(pp + (2 * ch + 1) * 2048) = make_uint4(y[4], y[5], y[6], y[7]);
                }
            if (may_hide && t0 + kTN > ses.len) {
                // Weights of 0 do not hide infinities and NaN from the product: at drafted positions they are taken out of V, and added to the rows
                // that see them at the end.
                const int sl = x + 1 < total ? 2 * x + 2 : 2 * x + 1;       // V's place in the order of the ring
                ok = ok && mbar_wait(full + 8 * (sl % slots), (uint32_t)(sl / slots) & 1u, failed, status);
                if (ok && t >= ses.len && t < ses.kv)
#pragma unroll 4
                    for (int e = 0; e < D / 8; ++e) {
                        uint4* at = reinterpret_cast<uint4*>(ring + sl % slots * F::slot + (e >> 3) * (kTN * 128) + tid * 128 + (((e & 7) ^ (tid & 7)) << 4));
                        uint4 v = *at;
                        uint32_t* h = reinterpret_cast<uint32_t*>(&v);
                        bool hit = false;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if ((h[k] & Kind<T>::exponent) == Kind<T>::exponent) { h[k] &= 0xffff0000u; hit = true; }
                            if ((h[k] >> 16 & Kind<T>::exponent) == Kind<T>::exponent) { h[k] &= 0xffffu; hit = true; }
                        }
                        if (hit) { *dirty = (uint32_t)sx.piece + 1u; *at = v; }
                    }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // P (and V) as the product reads them
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(pfull + 8 * (x & 1));
            if (!sx.last()) continue;

            // ---- the piece is done: sums over the positions, then a thread a component
#pragma unroll
            for (int ch = 0; ch < chunks; ++ch)
                if (ch < n_ch) {
#pragma unroll
                    for (int r = 16 * ch; r < 16 * ch + 16; ++r) {
                        const float v = warp_sum(sum[r]);
                        if (lane == (r & 31)) warp_s[wid * N + r] = v;
                    }
                }
            ok = ok && mbar_wait(ofull + 8 * (x & 1), (uint32_t)(x >> 1) & 1u, failed, status);
            if (!vote(ok, true)) { ok = false; break; }
            const bool whole = sx.w.tile == 0 && sx.m == sx.w.tiles;
            const int64_t slot = ((int64_t)2 * blockIdx.x + (sx.piece > 0)) * a.part_rows;
            if (tid < rows) {
                const float l = (warp_s[tid] + warp_s[N + tid]) + (warp_s[2 * N + tid] + warp_s[3 * N + tid]), top = top_s[tid];
                const int rr = row0 + tid, i = rr / a.group;
                const int64_t n_row = ses.first + i, head = (int64_t)sx.w.h * a.group + (rr - i * a.group);
                row_at[tid] = n_row * a.os_row + head * a.os_head;
                factor_s[tid] = l == 0.f ? 0.f : whole ? 1.f / l : 1.f;          // 0: nothing was seen
                if (!whole) a.part_ml[slot + tid] = make_float2(top, l);
                else if (a.lse) a.lse[n_row * a.heads + head] = l == 0.f ? -INFINITY : (top - Kind<T>::shift + log2f(l)) * 0.693147180559945f;
            }
            vote(1u, true);
            fence_after();
            const bool special = may_hide && *dirty == (uint32_t)sx.piece + 1u;
            for (int o = 0; o < F::o_blocks; ++o) {
                const int d = o * 128 + tid;
                for (int ch = 0; ch < n_ch; ++ch) {
                    uint32_t y[16];
                    tmem_ld16(tmem + 2 * N + o * N + lanes + 16 * ch, y);
                    wait_ld(y);
                    if (d >= D) continue;
                    if (special) {
                        for (int u = max(sx.w.tile * kTN, ses.len); u < min((sx.w.tile + sx.m) * kTN, ses.kv); ++u) {
                            const int page = b.table[(int64_t)sx.w.s * b.max_pages + u / p.page_pos];
                            if (page < 0 || page >= p.n_pages) continue;
                            const uint16_t v = reinterpret_cast<const uint16_t*>(p.base + (int64_t)a.layer * p.sl + (int64_t)sx.w.h * p.sh + p.skv +
                                                                                 (int64_t)page * p.spage + (int64_t)(u % p.page_pos) * p.sp)[d];
                            if ((v & Kind<T>::exponent) != Kind<T>::exponent) continue;
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                if (16 * ch + r < rows && (seen_bits(a, ses, (row0 + 16 * ch + r) / a.group, u) & 1u))
                                    y[r] = __float_as_uint(__uint_as_float(y[r]) + Kind<T>::widen(v));
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int q = 16 * ch + r;
                        if (q >= rows) break;
                        const float f = factor_s[q], v = f == 0.f ? 0.f : __uint_as_float(y[r]) * f;
                        if (whole) static_cast<uint16_t*>(a.out)[row_at[q] + d] = (uint16_t)(Kind<T>::pack(v, 0.f) & 0xffffu);
                        else a.part_o[(slot + q) * D + d] = v;
                    }
                }
            }
            fence_before();
        }
    }
    fence_before();
    __syncthreads();
    if (wid == mma_warp) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)F::tmem) : "memory");
    }
}

template <class T, int D>
cudaError_t launch(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st) {
    using F = Few<D>;
    cudaError_t e = cudaFuncSetAttribute(few_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)F::smem);
    if (e != cudaSuccess) return e;
    e = launch_kernel(few_kernel<T, D>, x.grid, kFewThreads, F::smem, st, false, 1, p, b, a, status);
    return e != cudaSuccess ? e : launch_join<T, D, F::N>(p, b, a, x, st);
}
template <class T>
cudaError_t launch_type(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st) {
    switch (p.d) {
        case 32: return launch<T, 32>(p, b, a, x, status, st);
        case 64: return launch<T, 64>(p, b, a, x, status, st);
        case 128: return launch<T, 128>(p, b, a, x, status, st);
        default: return launch<T, 256>(p, b, a, x, status, st);
    }
}

}  // namespace

cudaError_t launch_attend_few(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, bool bf16, uint32_t* status, cudaStream_t st) {
    return bf16 ? launch_type<__nv_bfloat16>(p, b, a, x, status, st) : launch_type<__half>(p, b, a, x, status, st);
}

}  // namespace plc
