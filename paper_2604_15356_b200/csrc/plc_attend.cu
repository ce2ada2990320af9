// Attention of drafted tokens over their session's pages (plc_tree_attention).
//
// For a session's KV head the rows are its drafted tokens times the query heads of the group.  Per tile of TN positions:
//   S = Q K^T        [128 x TN]  tcgen05.mma, both operands in shared memory, S in TMEM
//   P = exp2(c S - m)            a thread a row: running maximum m and sum l in binary32, P rounded to the pool's type
//   O = O + P V      [128 x d]   tcgen05.mma, P read from TMEM (over S's columns), V as it lies in the page (d contiguous)
// and out = O / l at the end.  K and V are read once per 128 (or 256) rows: for the few rows of single tokens and small
// trees that is the floor, and HBM bounds the kernel; from about 128 rows on the products and the exponentials do.
//
// Work.  All (session, head, row tile, position tile) form one sequence, cut into equal ranges, one a CTA: lengths that
// differ, and one long context, fill the GPU alike.  A CTA's first and last piece may be parts of an item (session, head,
// row tile); those leave O, m and l in the workspace and a second, small launch joins them in a fixed order.
//
// Roles in a CTA: warps that each own 32 rows (softmax, epilogue), three warps that copy (cp.async, 16 bytes a lane, each position's
// address from the page table, since a page may be any size and lie anywhere), one thread that issues the products.  Two layouts: NT = 1 (128
// rows; two CTAs an SM, whose phases overlap) and NT = 2 (two row tiles that share each K and V tile; one CTA an SM).
//
// The weights are rounded to the type of V because the product takes both operands in one type; l sums them unrounded.  For f16
// they are formed as 2^12 times themselves, so that weights down to 2^-26 of the largest keep all their bits.  A
// row's maximum is raised only when it would grow by more than 2^3 (a weight is at most 2^15 then), which spares most passes over O.
#include "plc_attend.cuh"

namespace plc {
namespace {

constexpr int kLoaders = 96;                      // threads that copy: three warps, so that a CTA has a whole number of warps a scheduler
constexpr int kWordRing = 4;                      // tiles whose validity words are kept: more than the loader can be ahead of the softmax

template <int D, int NT> struct Shape {
    static constexpr int TN = D == 256 ? 64 : 128;                     // positions a tile: S and O of a CTA's row tiles fit in TMEM, K and V in shared memory
    static constexpr int blocks = (D + 63) / 64;                       // 128-byte wide column blocks (32 components: half of one)
    static constexpr int DV = blocks * 64;                             // columns of O
    static constexpr int stages = D == 128 ? NT : NT == 2 ? 3 : 2;
    static constexpr int q_bytes = blocks * 128 * 128, kv_bytes = blocks * TN * 128;
    static constexpr int tmem = NT * (TN + DV) > 256 ? 512 : 256;
    static constexpr int rows = NT * 128, threads = NT * 128 + kLoaders + 32;
    static constexpr int per_sm = NT == 1 && D != 256 ? 2 : 1;
    static constexpr size_t smem = (size_t)NT * q_bytes + 2 * stages * kv_bytes + 2 * TN * 8 + 1024 + 512;
};

template <class T, int D, int NT>
__global__ void __launch_bounds__(Shape<D, NT>::threads, Shape<D, NT>::per_sm)
attend_kernel(PoolDev p, BookDev b, const __grid_constant__ AttendArgs a, uint32_t* status) {
    using Sh = Shape<D, NT>;
    using Wk = Walk<Sh::rows>;
    constexpr int TN = Sh::TN, stages = Sh::stages, n_warps = Sh::threads / 32;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ks = smem + NT * Sh::q_bytes;
    uint8_t* vs = ks + stages * Sh::kv_bytes;
    int64_t* offs = reinterpret_cast<int64_t*>(vs + stages * Sh::kv_bytes);             // [2][TN]
    uint64_t* bars = reinterpret_cast<uint64_t*>(offs + 2 * TN);
    uint32_t* words = reinterpret_cast<uint32_t*>(bars + 4 * stages + 3 + 3 * NT);      // [kWordRing][4]
    uint32_t* tmem_slot = words + kWordRing * 4;
    volatile uint32_t* failed = tmem_slot + 1;
    // [2]: piece number + 1 of the last pieces whose V holds infinities or NaN at drafted positions, by its parity (no row tile is a whole piece behind)
    volatile uint32_t* dirty = tmem_slot + 2;
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const uint32_t kfull = smem_u32(bars), vfull = kfull + 8 * stages, kempty = vfull + 8 * stages, vempty = kempty + 8 * stages;
    const uint32_t qfull = vempty + 8 * stages, qempty = qfull + 8, drain = qempty + 8, sfull = drain + 8, pfull = sfull + 8 * NT, ofull = pfull + 8 * NT;
    chain_next();

    constexpr int mma_warp = n_warps - 1;
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(kfull + 8 * i, kLoaders + kLoaders / 32);
            mbar_init(vfull + 8 * i, kLoaders);
            mbar_init(kempty + 8 * i, 1);
            mbar_init(vempty + 8 * i, 1);
        }
        mbar_init(qfull, kLoaders);
        mbar_init(qempty, 1);
        mbar_init(drain, 1);
        for (int i = 0; i < NT; ++i) {
            mbar_init(sfull + 8 * i, 1);
            mbar_init(pfull + 8 * i, 4);
            mbar_init(ofull + 8 * i, 1);
        }
        *failed = dirty[0] = dirty[1] = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == mma_warp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)Sh::tmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();

    Wk w{};
    long long left = find_range<Sh::rows, Sh::threads>(p, b, a, status, w);
    fence_after();
    const uint32_t tmem = *tmem_slot;
    const int me = blockIdx.x;

    if (wid >= NT * 4 && wid < mma_warp) {
        // ---- copies.  A tile's addresses are found by one thread a position and passed on in shared memory.
        const int lt = tid - NT * 128;
        constexpr int pieces = D * 2 / 16;
        const uint32_t q_s = smem_u32(smem), k_s = smem_u32(ks), v_s = smem_u32(vs);
        int done = 0, item = 0;
        bool ok = true, go = true;                    // this thread's waits; all loaders' (they leave together: they share a barrier)
        while (left > 0 && go) {
            const int m = (int)min(left, (long long)(w.tiles - w.tile)), rows = w.rows(a), row0 = w.rt * Sh::rows;
            const int32_t* row = b.table + (int64_t)w.s * b.max_pages;
            const uint8_t* kb = p.base + (int64_t)a.layer * p.sl + (int64_t)w.h * p.sh;
            ok = ok && mbar_wait(qempty, (uint32_t)(item & 1) ^ 1u, failed, status);
            if (ok)
                for (int u = lt; u < Sh::rows * pieces; u += kLoaders) {
                    const int r = u / pieces, c = u - r * pieces, rr = row0 + r, i = rr / a.group, g = rr - i * a.group;
                    const uint8_t* src = static_cast<const uint8_t*>(a.q);
                    if (r < rows) src += 2 * ((int64_t)(w.x.first + i) * a.qs_row + (int64_t)(w.h * a.group + g) * a.qs_head) + c * 16;
                    copy16(q_s + (r >> 7) * Sh::q_bytes + (c >> 3) * 16384 + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4), src, r < rows);
                }
            mbar_arrive_copies(qfull);
            for (int j = 0; j < m; ++j, ++done) {
                const int st = done % stages;
                const uint32_t ph = (uint32_t)(done / stages) & 1u;
                int64_t* off = offs + (done & 1) * TN;
                uint32_t valid[2] = {0, 0};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int word = (lt >> 5) + e * (kLoaders / 32);
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
                    : "=r"(all) : "r"((uint32_t)ok), "n"(kLoaders) : "memory");
                go = all != 0;
                if (!go) break;
                if (lane == 0) {
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if ((lt >> 5) + e * (kLoaders / 32) < TN / 32) words[(done % kWordRing) * 4 + (lt >> 5) + e * (kLoaders / 32)] = valid[e];
                }
#pragma unroll 8
                for (int u = lt; u < TN * pieces; u += kLoaders) {
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
                    for (int u = lt; u < TN * pieces; u += kLoaders) {
                        const int r = u / pieces, c = u % pieces;
                        const int64_t o = off[r];
                        copy16(v_s + st * Sh::kv_bytes + (c >> 3) * (TN * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4),
                               o == INT64_MIN ? kb : kb + p.skv + o + c * 16, o != INT64_MIN);
                    }
                    mbar_arrive_copies(vfull + 8 * st);
                }
            }
            left -= m;
            ++item;
            if (left > 0) w.next_item(p, b, a);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (wid == mma_warp) {
        if (lane == 0) {
            // ---- products, in the order QK(0), then for every tile PV(j), QK(j+1), the row tiles in turn.  They run in the order in which they are
            // issued, so that S of the next tile may take the columns of P of this one.
            constexpr uint32_t common = (1u << 4) | (Kind<T>::format << 7) | (Kind<T>::format << 10) | (8u << 24);
            constexpr uint32_t id_qk = common | ((uint32_t)(TN >> 3) << 17), id_pv = common | (1u << 16) | ((uint32_t)(Sh::DV >> 3) << 17);
            const uint32_t q_s = smem_u32(smem), k_s = smem_u32(ks), v_s = smem_u32(vs);
            int kd = 0, vd = 0, item = 0;
            uint32_t pph[NT];
            for (int i = 0; i < NT; ++i) pph[i] = 0;
            bool ok = true;
            auto qk = [&](int n, bool last) {          // every row tile in use against the next K tile is two calls: see below
                const int st = kd % stages;
                const uint32_t kaddr = k_s + st * Sh::kv_bytes, s_at = tmem + n * TN;
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_ss(s_at, desc_k(q_s + n * Sh::q_bytes + (k >> 2) * 16384) + 2 * (k & 3), desc_k(kaddr + (k >> 2) * (TN * 128)) + 2 * (k & 3), id_qk, k ? 1u : 0u);
                mma_commit(sfull + 8 * n);
                if (last) { mma_commit(kempty + 8 * st); ++kd; }
            };
            auto wait_k = [&]() {
                ok = ok && mbar_wait(kfull + 8 * (kd % stages), (uint32_t)(kd / stages) & 1u, failed, status);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                fence_after();
            };
            while (left > 0 && ok) {
                const int m = (int)min(left, (long long)(w.tiles - w.tile)), nt = NT == 2 && w.rows(a) > 128 ? 2 : 1;
                ok = mbar_wait(qfull, (uint32_t)(item & 1), failed, status);
                wait_k();
                if (!ok) break;
                for (int n = 0; n < nt; ++n) qk(n, n == nt - 1);
                if (m == 1) mma_commit(qempty);
                for (int j = 0; j < m && ok; ++j, ++vd) {
                    const int st = vd % stages;
                    for (int n = 0; n < nt && ok; ++n) {
                        ok = mbar_wait(pfull + 8 * n, pph[n], failed, status);
                        pph[n] ^= 1u;
                        if (n == 0) ok = ok && mbar_wait(vfull + 8 * st, (uint32_t)(vd / stages) & 1u, failed, status);
                        if (!ok) break;
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        fence_after();
                        const uint32_t vaddr = v_s + st * Sh::kv_bytes, o_at = tmem + NT * TN + n * Sh::DV, p_at = tmem + n * TN;
#pragma unroll
                        for (int k = 0; k < TN / 16; ++k) mma_ts(o_at, p_at + 8 * k, desc_mn(vaddr + k * 2048, TN * 128), id_pv, j | k ? 1u : 0u);
                        mma_commit(ofull + 8 * n);
                        if (n == nt - 1) mma_commit(vempty + 8 * st);
                        if (j + 1 < m) {
                            if (n == 0) wait_k();
                            if (!ok) break;
                            qk(n, n == nt - 1);
                            if (j + 2 == m && n == nt - 1) mma_commit(qempty);
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
    } else {
        // ---- softmax and epilogue: a thread a row
        const int nt = wid >> 2, r_tile = (wid & 3) * 32 + lane, r_item = nt * 128 + r_tile;
        const uint32_t lanes = (uint32_t)((wid & 3) * 32) << 16, s_at = tmem + nt * TN + lanes, o_at = tmem + NT * TN + nt * Sh::DV + lanes;
        const float c = a.scale * 1.44269504088896f;
        int done = 0, tiles_done = 0, part = 0;       // tiles of this row tile, of the CTA
        bool ok = true;
        while (left > 0 && ok) {
            const int m = (int)min(left, (long long)(w.tiles - w.tile)), rows = w.rows(a);
            const bool in_use = nt == 0 || rows > 128, works = r_tile - lane + nt * 128 < rows;   // the row tile; this warp
            const int rr = w.rt * Sh::rows + r_item, i = rr / a.group;
            float top = -INFINITY, sum = 0.f;         // top: what the weights are relative to, scaled, base 2
            const bool may_hide = a.mask != nullptr || w.x.n > 1;
            for (int j = 0; j < m && in_use; ++j, ++done) {
                const int t = (w.tile + j) * TN;
                ok = mbar_wait(sfull + 8 * nt, (uint32_t)done & 1u, failed, status);
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                fence_after();
                const uint32_t* valid = words + ((tiles_done + j) % kWordRing) * 4;
                bool masked = t + TN > w.x.len;
#pragma unroll
                for (int e = 0; e < TN / 32; ++e) masked |= valid[e] != ~0u;
                if (works) {
                    uint32_t vis[TN / 32];
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < TN / 32; ++e) vis[e] = valid[e] & (r_item < rows ? seen_bits(a, w.x, i, t + 32 * e) : 0u);
                    }
                    float x_top = -INFINITY;
#pragma unroll
                    for (int e = 0; e < TN / 32; ++e) {
                        uint32_t x[32];
                        tmem_ld32(s_at + 32 * e, x);
                        wait_ld(x);
                        if (masked) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) x[k] = vis[e] >> k & 1u ? x[k] : 0xff800000u;
                        }
#pragma unroll
                        for (int k = 0; k < 32; ++k) x_top = fmaxf(x_top, __uint_as_float(x[k]));
                    }
                    const float now = x_top * c;
                    const bool raise = now > top + kRaise;            // also the first finite score
                    if (__any_sync(kFull, raise)) {
                        const float f = raise && top > -INFINITY ? exp2_approx(top - now) : raise ? 0.f : 1.f;
                        if (raise) top = now;
                        sum *= f;
                        if (j > 0) {
                            ok = mbar_wait(ofull + 8 * nt, (uint32_t)(done - 1) & 1u, failed, status);
                            ok = __all_sync(kFull, ok);
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
                    const float base = top == -INFINITY ? 0.f : top - Kind<T>::shift;
                    float part_sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < TN / 32; ++e) {
                        uint32_t x[32], y[16];
                        tmem_ld32(s_at + 32 * e, x);
                        wait_ld(x);
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            float v = exp2_approx(fmaf(__uint_as_float(x[k]), c, -base));
                            if (masked) v = vis[e] >> k & 1u ? v : 0.f;
                            x[k] = __float_as_uint(v);
                            part_sum[k & 3] += v;
                        }
#pragma unroll
                        for (int k = 0; k < 16; ++k) y[k] = Kind<T>::pack(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1]));
                        tmem_st16(s_at + 16 * e, y);
                    }
                    sum += (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
                    wait_st();
                }
                if (may_hide && t + TN > w.x.len) {
                    // Weights of 0 do not hide infinities and NaN from the product: at drafted positions they are taken out of V, and added
                    // to the rows that see them at the end.
                    const int st = (tiles_done + j) % stages;
                    ok = mbar_wait(vfull + 8 * st, (uint32_t)((tiles_done + j) / stages) & 1u, failed, status);
                    ok = __all_sync(kFull, ok);
                    if (!ok) break;
                    bool found = false;
                    for (int u = (wid & 3) * 32 + lane; u < TN * Sh::blocks * 8; u += 128) {
                        const int r = (u >> 3) % TN;
                        if (t + r < w.x.len || (D == 32 && (((u & 7) ^ (r & 7)) >= 4))) continue;
                        uint4* at = reinterpret_cast<uint4*>(vs + st * Sh::kv_bytes + u * 16);
                        uint4 v = *at;
                        uint32_t* h = reinterpret_cast<uint32_t*>(&v);
                        bool hit = false;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if ((h[k] & Kind<T>::exponent) == Kind<T>::exponent) { h[k] &= 0xffff0000u; hit = true; }
                            if ((h[k] >> 16 & Kind<T>::exponent) == Kind<T>::exponent) { h[k] &= 0xffffu; hit = true; }
                        }
                        if (hit) {
                            dirty[part & 1] = (uint32_t)part + 1u;
                            __threadfence_block();            // who finds the zeros finds the flag
                            *at = v;
                            found = true;
                        }
                    }
                    if (found) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pfull + 8 * nt);
            }
            tiles_done += m;
            if (ok && in_use) {
                ok = mbar_wait(ofull + 8 * nt, (uint32_t)(done - 1) & 1u, failed, status);
                ok = __all_sync(kFull, ok);
            }
            if (!ok) break;
            if (in_use && works) {
                fence_after();
                const bool whole = w.tile == 0 && m == w.tiles, live = r_item < rows;
                const int64_t n_row = w.x.first + i, head = (int64_t)w.h * a.group + (rr - i * a.group), slot = ((int64_t)2 * me + (part > 0)) * a.part_rows + r_item;
                const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;   // NaN stays NaN
                const bool special = may_hide && dirty[part & 1] == (uint32_t)part + 1u;
#pragma unroll 1
                for (int e = 0; e < (D + 31) / 32; ++e) {
                    uint32_t o[32];
                    tmem_ld32(o_at + 32 * e, o);
                    wait_ld(o);
                    if (!live) continue;
                    if (sum == 0.f) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = 0u;        // nothing was seen: whatever the product made of it
                    }
                    if (special) {
                        for (int t = max(w.tile * TN, w.x.len); t < min((w.tile + m) * TN, w.x.kv); ++t) {
                            if (!(seen_bits(a, w.x, i, t) & 1u)) continue;
                            const int page = b.table[(int64_t)w.s * b.max_pages + t / p.page_pos];
                            if (page < 0 || page >= p.n_pages) continue;
                            const uint16_t* v = reinterpret_cast<const uint16_t*>(p.base + (int64_t)a.layer * p.sl + (int64_t)w.h * p.sh + p.skv +
                                                                                  (int64_t)page * p.spage + (int64_t)(t % p.page_pos) * p.sp) + 32 * e;
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if ((v[k] & Kind<T>::exponent) == Kind<T>::exponent) o[k] = __float_as_uint(__uint_as_float(o[k]) + Kind<T>::widen(v[k]));
                        }
                    }
                    if (whole) {
                        uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + n_row * a.os_row + head * a.os_head + 32 * e);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t y[4];
#pragma unroll
                            for (int l = 0; l < 4; ++l) y[l] = Kind<T>::pack(__uint_as_float(o[8 * k + 2 * l]) * inv, __uint_as_float(o[8 * k + 2 * l + 1]) * inv);
                            dst[k] = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    } else {
                        uint4* dst = reinterpret_cast<uint4*>(a.part_o + slot * D + 32 * e);
#pragma unroll
                        for (int k = 0; k < 8; ++k) dst[k] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                    }
                }
                if (live) {
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

template <int D, int NT> AttendPlan plan_of(long long rows) {
    using Sh = Shape<D, NT>;
    AttendPlan x;
    x.row_tile = Sh::rows;
    x.grid = Sh::per_sm * sm_count();
    x.part_rows = (int)(rows < Sh::rows ? rows : Sh::rows);
    x.bytes = (uint64_t)x.grid * 16 + 2ull * x.grid * x.part_rows * (8 + 4 * D);
    return x;
}
// Up to kFewRows rows a session and KV head (32 of 256 components) take the layout for few rows; beyond, two row tiles share K and V where a
// session has more rows than one holds.
constexpr int kFewRows = 64;
AttendPlan plan(const PoolDev& p, int heads, int sessions, int n_rows) {
    const long long rows = (long long)n_rows * (heads / p.H);
    const int few = p.d == 256 ? kFewRows / 2 : kFewRows;
    if (rows <= (long long)few * sessions) {
        AttendPlan x;
        x.row_tile = rows <= 16LL * sessions ? 16 : rows <= 32LL * sessions ? 32 : few;
        x.grid = (x.row_tile <= 32 && p.d != 256 ? 2 : 1) * sm_count();      // at most: see Few::per_sm
        x.part_rows = (int)(rows < x.row_tile ? rows : x.row_tile);
        x.bytes = (uint64_t)x.grid * 16 + 2ull * x.grid * x.part_rows * (8 + 4 * p.d);
        return x;
    }
    const bool two = rows > 128LL * sessions;
    switch (p.d) {
        case 32: return two ? plan_of<32, 2>(rows) : plan_of<32, 1>(rows);
        case 64: return two ? plan_of<64, 2>(rows) : plan_of<64, 1>(rows);
        case 128: return two ? plan_of<128, 2>(rows) : plan_of<128, 1>(rows);
        default: return plan_of<256, 1>(rows);
    }
}

template <class T, int D, int NT>
cudaError_t launch_attend(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st) {
    using Sh = Shape<D, NT>;
    cudaError_t e = cudaFuncSetAttribute(attend_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Sh::smem);
    if (e != cudaSuccess) return e;
    e = launch_kernel(attend_kernel<T, D, NT>, x.grid, Sh::threads, Sh::smem, st, false, 1, p, b, a, status);
    return e != cudaSuccess ? e : launch_join<T, D, Sh::rows>(p, b, a, x, st);
}
template <class T>
cudaError_t launch_type(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st) {
    switch (p.d) {
        case 32: return x.row_tile == 256 ? launch_attend<T, 32, 2>(p, b, a, x, status, st) : launch_attend<T, 32, 1>(p, b, a, x, status, st);
        case 64: return x.row_tile == 256 ? launch_attend<T, 64, 2>(p, b, a, x, status, st) : launch_attend<T, 64, 1>(p, b, a, x, status, st);
        case 128: return x.row_tile == 256 ? launch_attend<T, 128, 2>(p, b, a, x, status, st) : launch_attend<T, 128, 1>(p, b, a, x, status, st);
        default: return launch_attend<T, 256, 1>(p, b, a, x, status, st);
    }
}

plc_status check_heads(const PoolDev& p, int32_t n_heads) {
    if (n_heads < 1) return PLC_E_INVALID;
    return n_heads % p.H || n_heads > (1 << 16) ? PLC_E_SHAPE : PLC_OK;
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" {

plc_status plc_tree_attention_workspace(const plc_page_pool* pool, int32_t sessions, int32_t n_heads, int32_t n_rows, uint64_t* bytes) {
    PoolDev p;
    plc_status rc = check_pool(pool, &p);
    if (rc || (rc = check_heads(p, n_heads))) return rc;
    if (!bytes || sessions < 1 || n_rows < 0) return PLC_E_INVALID;
    *bytes = plan(p, n_heads, sessions, n_rows).bytes;
    return PLC_OK;
}

plc_status plc_tree_attention(const plc_page_pool* pool, int32_t layer, const plc_page_book* book, const plc_tree_queries* t, float scale,
                              void* workspace_dev, uint64_t workspace_bytes, uint32_t* status_dev, void* stream) {
    PoolDev p;
    BookDev b;
    plc_status rc = check_pool(pool, &p);
    if (rc || (rc = check_book(book, &b))) return rc;
    if (!t || !t->q_dev || !t->out_dev || !t->begin_dev || t->n_rows < 0 || !status_dev || !workspace_dev) return PLC_E_INVALID;
    if (layer < 0 || layer >= p.L || pool->dtype == PLC_OUT_F32 || (t->mask_dev && t->mask_words < 1) || !(scale > 0.f) || isinf(scale)) return PLC_E_INVALID;
    if ((rc = check_heads(p, t->n_heads))) return rc;
    const int group = t->n_heads / p.H;
    if ((long long)t->n_rows * group > (1 << 30)) return PLC_E_SHAPE;
    if (!plc_aligned16(t->q_dev) || !plc_aligned16(t->out_dev) || !plc_aligned16(workspace_dev) || t->q_stride_row % 8 || t->q_stride_head % 8 ||
        t->out_stride_row % 8 || t->out_stride_head % 8)
        return PLC_E_ALIGN;
    const AttendPlan x = plan(p, t->n_heads, b.rows, t->n_rows);
    if (workspace_bytes < x.bytes) return PLC_E_CAPACITY;
    if (t->n_rows == 0) return PLC_OK;
    AttendArgs a{t->q_dev, t->q_stride_row, t->q_stride_head, t->out_dev, t->out_stride_row, t->out_stride_head, t->lse_dev, t->begin_dev,
                 t->mask_dev, t->n_rows, t->n_heads, group, t->mask_dev ? t->mask_words : 0, layer, scale, nullptr, nullptr, nullptr, x.part_rows, p.d == 256 ? 64 : 128, 0, 0, {}};
    a.first = static_cast<int4*>(workspace_dev);
    a.part_o = reinterpret_cast<float*>(a.first + x.grid);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + 2ll * x.grid * x.part_rows * p.d);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = x.row_tile <= kFewRows
        ? (pool->dtype == PLC_OUT_F16 ? launch_attend_few_f16(p, b, a, x, status_dev, st) : launch_attend_few_bf16(p, b, a, x, status_dev, st))
        : pool->dtype == PLC_OUT_F16 ? launch_type<__half>(p, b, a, x, status_dev, st) : launch_type<__nv_bfloat16>(p, b, a, x, status_dev, st);
    if (e != cudaSuccess) return PLC_E_CUDA;
    count_launch(2);
    return PLC_OK;
}

}  // extern "C"
