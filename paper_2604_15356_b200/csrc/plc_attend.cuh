// Tree attention: what its kernels share (the sequence of position tiles and a CTA's range of it, masks, the tensor core's instructions).
#pragma once
#include "plc_boxes.cuh"
#include "plc_tensor.cuh"

namespace plc {

constexpr float kRaise = 3.f;

struct AttendArgs {
    const void* q; int64_t qs_row, qs_head;       // elements
    void* out; int64_t os_row, os_head;
    float* lse;
    const int32_t* begin; const uint32_t* mask;
    int rows, heads, group, mask_words, layer;
    float scale;
    float* part_o;                                // [2 * grid][part_rows][d]
    float2* part_ml;                              // [2 * grid][part_rows]: maximum (scaled, base 2), sum
    int4* first;                                  // [grid]: session, head, row tile, first position tile of each CTA's range (-1: none)
    int part_rows;
    int tile_pos;                                 // positions a tile (whole pages, or whole parts of a page, where the copies are boxes)
    int box_pos, boxes;                           // positions a box, boxes a tile; 0: no boxes
    int box_dim[4];                               // what dimensions 1 .. 4 of the boxes' map are: 0 slot, 1 head, 2 page, 3 key or value
    int whole;                                    // not 0: a CTA an item (at most so many), nothing to join
};

// Which kernel a call takes, and what it needs.
struct AttendPlan { int row_tile, grid, part_rows; uint64_t bytes; };

cudaError_t launch_attend_few_f16(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st);
cudaError_t launch_attend_few_bf16(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st);
cudaError_t launch_attend_many_f16(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st);
cudaError_t launch_attend_many_bf16(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, uint32_t* status, cudaStream_t st);

#ifdef __CUDACC__
namespace {

// A session as the call gives it, cut to what there is.
struct Session { int first, n, len, kv; };
__device__ __forceinline__ Session session_of(const PoolDev& p, const BookDev& b, const AttendArgs& a, int s, bool* bad) {
    const int b0 = a.begin[s], b1 = a.begin[s + 1], len = b.len[s], most = most_positions(b, p);
    Session x;
    x.first = min(max(b0, 0), a.rows);
    x.n = min(max(b1, x.first), a.rows) - x.first;
    x.len = min(max(len, 0), most);
    x.kv = x.n > 0 ? (int)min((long long)x.len + x.n, (long long)most) : 0;
    *bad = b0 < 0 || b1 < b0 || b1 > a.rows || len < 0 || len > most || (long long)x.len + x.n > most;
    return x;
}

// Where a range of position tiles stands: item (session, head, row tile) and tile in it.
template <int ROWS> struct Walk {
    int s, h, rt, tile, tiles, row_tiles;
    Session x;
    __device__ __forceinline__ void enter(const PoolDev& p, const BookDev& b, const AttendArgs& a) {
        bool bad;
        x = session_of(p, b, a, s, &bad);
        tiles = (x.kv + a.tile_pos - 1) / a.tile_pos;
        row_tiles = (int)(((long long)x.n * a.group + ROWS - 1) / ROWS);
    }
    __device__ __forceinline__ void start(const PoolDev& p, const BookDev& b, const AttendArgs& a, int session, long long rest) {
        s = session;
        enter(p, b, a);
        const int item = (int)(a.whole ? rest : rest / tiles);
        tile = a.whole ? 0 : (int)(rest - (long long)item * tiles);
        h = item / row_tiles;
        rt = item - h * row_tiles;
    }
    __device__ __forceinline__ void next_item(const PoolDev& p, const BookDev& b, const AttendArgs& a) {
        tile = 0;
        if (++rt < row_tiles) return;
        rt = 0;
        if (++h < p.H) return;
        h = 0;
        do {
            if (++s >= b.rows) return;
            enter(p, b, a);
        } while (x.n == 0);
    }
    __device__ __forceinline__ int rows(const AttendArgs& a) const { return min(ROWS, x.n * a.group - rt * ROWS); }
};

// 32 bits: which of the positions t .. t+31 row i (the i-th drafted token) sees, as far as the mask says.
__device__ __forceinline__ uint32_t seen_bits(const AttendArgs& a, const Session& x, int i, int t) {
    const int j = t - x.len;                      // drafted index of the first one
    if (j <= -32) return ~0u;
    auto word = [&](int w) -> uint32_t {          // drafted positions 32 w ...
        if (w < 0) return ~0u;                    // committed ones
        if (a.mask) return w < a.mask_words ? a.mask[(int64_t)(x.first + i) * a.mask_words + w] : 0u;
        const int up = i - 32 * w;                // bits 0 .. up
        return up < 0 ? 0u : up >= 31 ? ~0u : (2u << up) - 1u;
    };
    const int w = j >> 5;
    return __funnelshift_r(word(w), word(w + 1), j & 31);
}

// A CTA's range [0, left) of the sequence of tiles, from w on (a.whole: of the sequence of items, one of them).  Every thread of the CTA calls it; two barriers.
template <int ROWS, int THREADS>
__device__ __forceinline__ long long find_range(const PoolDev& p, const BookDev& b, const AttendArgs& a, uint32_t* status, Walk<ROWS>& w) {
    __shared__ long long sums[THREADS / 32];
    __shared__ long long range_at[2];             // the range's first session, and the tiles of it that lie before the range
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    // a thread sums a run of sessions, the threads' sums are scanned
    const int run = (b.rows + THREADS - 1) / THREADS, s0 = min(b.rows, tid * run), s1 = min(b.rows, s0 + run);
    auto tiles_of = [&](int s, bool* bad) -> long long {
        const Session x = session_of(p, b, a, s, bad);
        return (long long)(a.whole ? min(x.kv, 1) : (x.kv + a.tile_pos - 1) / a.tile_pos) * (((long long)x.n * a.group + ROWS - 1) / ROWS) * p.H;
    };
    long long mine = 0;
    bool any_bad = false;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
        bool bad;
        mine += tiles_of(s, &bad);
        any_bad |= bad;
    }
    if (any_bad && blockIdx.x == 0) atomicOr(status, kStRange);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(kFull, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) sums[wid] = upto;
    __syncthreads();
    long long total = 0, ahead = upto - mine;
#pragma unroll 1
    for (int v = 0; v < THREADS / 32; ++v) {
        if (v < wid) ahead += sums[v];
        total += sums[v];
    }
    const int workers = (int)min((long long)gridDim.x, total), me = blockIdx.x;
    const long long t0 = me < workers ? total * me / workers : total, t1 = me < workers ? total * (me + 1) / workers : total;
    if (t0 < t1 && t0 >= ahead && t0 < ahead + mine) {
        long long at = ahead;
        bool bad;
        int s = s0;
#pragma unroll 1
        for (; s < s1; ++s) {
            const long long f = tiles_of(s, &bad);
            if (t0 < at + f) break;
            at += f;
        }
        range_at[0] = s;
        range_at[1] = t0 - at;
    }
    __syncthreads();
    if (t1 > t0) w.start(p, b, a, (int)range_at[0], range_at[1]);
    if (tid == 0) a.first[me] = t1 > t0 ? make_int4(w.s, w.h, w.rt, w.tile) : make_int4(-1, 0, 0, 0);
    return a.whole ? (t1 > t0 ? w.tiles : 0) : t1 - t0;
}

// The tiles of a range one after the other; a piece is what the range holds of one item.
template <int ROWS> struct Tiles {
    Walk<ROWS> w;
    long long left;                               // from this piece on
    int j, m, piece;                              // tile of the piece, tiles in it, number of the piece
    __device__ __forceinline__ void start(const Walk<ROWS>& from, long long n) {
        w = from;
        left = n;
        j = piece = 0;
        m = n > 0 ? (int)min(n, (long long)(w.tiles - w.tile)) : 0;
    }
    __device__ __forceinline__ bool more() const { return left > 0; }
    __device__ __forceinline__ bool last() const { return j == m - 1; }
    __device__ __forceinline__ void next(const PoolDev& p, const BookDev& b, const AttendArgs& a) {
        if (++j < m) return;
        left -= m;
        if (left <= 0) return;
        w.next_item(p, b, a);
        j = 0;
        ++piece;
        m = (int)min(left, (long long)(w.tiles - w.tile));
    }
};

// Weights of 0 do not hide infinities and NaN from the product: at drafted positions they are taken out of V (one position's vector in a tile of TN),
// and added to the rows that see them at the end.  Returns whether there were any.
template <class T, int D, int TN>
__device__ __forceinline__ bool special(const uint8_t* tile, int pos) {
    constexpr uint32_t all = Kind<T>::exponent * 0x10001u, one = (0x8000u - Kind<T>::exponent) * 0x10001u;
    uint32_t hit = 0;                             // an exponent of ones carries into the sign
#pragma unroll 4
    for (int e = 0; e < D / 8; ++e) {
        const uint4 v = *reinterpret_cast<const uint4*>(tile + (e >> 3) * (TN * 128) + pos * 128 + (((e & 7) ^ (pos & 7)) << 4));
        hit |= ((v.x & all) + one) | ((v.y & all) + one) | ((v.z & all) + one) | ((v.w & all) + one);
    }
    return hit & 0x80008000u;
}
template <class T, int D, int TN>
__device__ __noinline__ bool take_out(uint8_t* tile, int pos) {
    bool any = false;
    for (int e = 0; e < D / 8; ++e) {
        uint4* at = reinterpret_cast<uint4*>(tile + (e >> 3) * (TN * 128) + pos * 128 + (((e & 7) ^ (pos & 7)) << 4));
        uint4 v = *at;
        uint32_t* h = reinterpret_cast<uint32_t*>(&v);
        bool hit = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if ((h[k] & Kind<T>::exponent) == Kind<T>::exponent) { h[k] &= 0xffff0000u; hit = true; }
            if ((h[k] >> 16 & Kind<T>::exponent) == Kind<T>::exponent) { h[k] &= 0xffffu; hit = true; }
        }
        if (hit) *at = v;
        any |= hit;
    }
    return any;
}

// Copies of the keys (kv = 0) or values (1) of a CTA's range into their ring, by `pair` warps of which each issues every pair-th box of a tile (box_pos positions
// of one page, 64 components wide).  A lane looks a box's page up, a tile ahead.  The first warp of the keys also writes which positions of a
// tile exist (a bit each); load_q(tile, ok) is called at the start of each piece for the keys.
template <int ROWS, int BLOCKS, int TN, class Q>
__device__ __forceinline__ void copy_boxes(const PoolDev& p, const BookDev& b, const AttendArgs& a, const CUtensorMap& map, const Walk<ROWS>& from, long long total, int kv, int half,
                                           int pair, uint32_t ring, int slot_bytes, int slots, uint32_t full, uint32_t empty, uint32_t* words, int word_ring,
                                           volatile uint32_t* failed, uint32_t* status, Q&& load_q) {
    const int lane = threadIdx.x & 31;
    Tiles<ROWS> x;
    x.start(from, total);
    int page = -1, slot = 0, issued = 0;
    bool ok = true;
    const int my_box = 4 * lane / a.box_pos;         // of the four positions whose validity the lane tells
    auto look_up = [&]() {                           // -1: behind the last position
        const int t = (x.w.tile + x.j) * a.tile_pos + lane * a.box_pos, pg = t / p.page_pos;
        slot = t - pg * p.page_pos;
        page = lane < a.boxes && t < x.w.x.kv ? b.table[(int64_t)x.w.s * b.max_pages + pg] : -1;
        if (page == -1 && lane < a.boxes && t < x.w.x.kv) page = -2;
    };
    if (total > 0) look_up();
    for (int n = 0; x.more(); ++n) {
        if (kv == 0 && x.j == 0) ok = load_q(x, ok);
        const bool have = page >= 0 && page < p.n_pages;
        const uint32_t boxes = __ballot_sync(kFull, have);
        const int here = page, at = slot, h = x.w.h;
        if (kv == 0 && half == 0) {
            if (page < -1 || page >= p.n_pages) atomicOr(status, kStRange);
            const int t = (x.w.tile + x.j) * a.tile_pos + 4 * lane;
            const int valid = boxes >> (my_box & 31) & 1u && 4 * lane < a.tile_pos ? min(max(x.w.x.kv - t, 0), 4) : 0;
            const uint32_t word = __reduce_or_sync(0xffu << (lane & 24), ((1u << valid) - 1u) << (4 * (lane & 7)));
            if ((lane & 7) == 0) words[n % word_ring * 4 + (lane >> 3)] = word;
            __syncwarp();                                // four lanes' words, which lane 0's arrival tells of
        }
        x.next(p, b, a);
        if (x.more()) look_up();
        const int s = n % slots;
        ok = __all_sync(kFull, ok && mbar_wait(empty + 8 * s, ((uint32_t)(n / slots) & 1u) ^ 1u, failed, status));
        if (!ok) break;
        const uint32_t mine = pair == 1 ? boxes : boxes & (half ? 0xaaaaaaaau : 0x55555555u), bar = full + 8 * s;
        if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(__popc(mine) * a.box_pos * BLOCKS * 128) : "memory");
        for (int e = half; e < a.boxes; e += pair) {
            const int pg = __shfl_sync(kFull, here, e), sl = __shfl_sync(kFull, at, e);
            if (!(mine >> e & 1u) || lane != 0) continue;
            int c[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) c[k] = a.box_dim[k] == 0 ? sl : a.box_dim[k] == 1 ? h : a.box_dim[k] == 2 ? pg : kv;
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k)
                asm volatile(
                    "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(
                        ring + s * slot_bytes + k * (TN * 128) + e * a.box_pos * 128),
                    "l"(&map), "r"(k * 64), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]), "r"(bar)
                    : "memory");
        }
        issued = n + 1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!ok)                                         // boxes still in flight (none after a complete run) land before the CTA ends
        for (int n = issued > slots ? issued - slots : 0; n < issued; ++n)
            for (uint32_t k = 0; k < kSpin; ++k) {
                uint32_t done;
                asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                             : "=r"(done) : "r"(full + 8 * (n % slots)), "r"((uint32_t)(n / slots) & 1u) : "memory");
                if (done) break;
            }
}

// Joins the pieces of items that more than one CTA had: block c looks at the boundary between CTAs c - 1 and c, and takes the item if that is the
// first boundary inside it.  A warp a row; a lane a piece for the weights, then a lane its components with the pieces' loads eight at a time
// (a piece after the other, 37 pieces took 84 us; so 37 pieces of 512 rows take 13 us).
constexpr int kJoinThreads = 128;
template <int ROWS> struct Join { static constexpr int rows = ROWS < 128 ? 4 : 8; };          // a block's
template <class T, int D, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b, const __grid_constant__ AttendArgs a, int workers) {
    constexpr int VEC = D / 32;                   // a lane's components
    chain_wait();
    const int c = blockIdx.x + 1, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int4 f = a.first[c], prev = a.first[c - 1];
    if (f.x < 0 || f.w == 0) return;
    auto same = [&](const int4& o) { return o.x == f.x && o.y == f.y && o.z == f.z; };
    if (same(prev) && prev.w > 0) return;
    const int r0 = blockIdx.y * Join<ROWS>::rows;
    bool bad;
    const Session x = session_of(p, b, a, f.x, &bad);
    const int rows = min(ROWS, x.n * a.group - f.z * ROWS);
    if (r0 >= rows) return;
    int pieces = 2;                               // CTA c - 1 had the first one, c, c + 1, ... the others
    for (int k = c + 1; k < workers; k += 32) {
        int4 o = make_int4(-1, 0, 0, 0);
        if (k + lane < workers) o = a.first[k + lane];
        const uint32_t in = __ballot_sync(kFull, same(o) && o.w > 0);
        const int run = __ffs(~in) - 1;           // 32 ones: -1
        pieces += run < 0 ? 32 : run;
        if (run >= 0) break;
    }
    const int64_t lead = (int64_t)2 * (c - 1) + (same(prev) ? 0 : 1);      // the piece that the item begins with
    for (int r = r0 + wid; r < min(rows, r0 + Join<ROWS>::rows); r += kJoinThreads / 32) {
        auto at = [&](int k) -> int64_t { return (k == 0 ? lead : (int64_t)2 * (c - 1 + k)) * a.part_rows + r; };
        float top = -INFINITY;
        for (int k = lane; k < pieces; k += 32) top = fmaxf(top, a.part_ml[at(k)].x);
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, w));
        float sum = 0.f, o[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = 0.f;
        for (int k0 = 0; k0 < pieces; k0 += 32) {
            float weight = 0.f;
            if (k0 + lane < pieces) {
                const float2 ml = a.part_ml[at(k0 + lane)];
                if (ml.y != 0.f) { weight = exp2f(ml.x - top); sum = fmaf(ml.y, weight, sum); }   // 0: nothing was seen there
            }
            const int n = min(32, pieces - k0);
            for (int j0 = 0; j0 < n; j0 += 8) {
                float y[8][VEC];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float* from = a.part_o + at(k0 + min(j0 + j, n - 1)) * D + lane * VEC;
#pragma unroll
                    for (int e = 0; e < VEC; e += 4) {
                        if (VEC >= 4) *reinterpret_cast<float4*>(&y[j][e]) = *reinterpret_cast<const float4*>(from + e);
                        else if (VEC == 2) *reinterpret_cast<float2*>(&y[j][0]) = *reinterpret_cast<const float2*>(from);
                        else y[j][0] = *from;
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float w = __shfl_sync(kFull, weight, (j0 + j) & 31);
                    if (j0 + j < n && w != 0.f) {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) o[e] = fmaf(y[j][e], w, o[e]);
                    }
                }
            }
        }
        sum = warp_sum(sum);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int rr = f.z * ROWS + r, i = rr / a.group;
        const int64_t n_row = x.first + i, head = (int64_t)f.y * a.group + (rr - i * a.group);
        uint16_t* out = static_cast<uint16_t*>(a.out) + n_row * a.os_row + head * a.os_head + lane * VEC;
        if constexpr (VEC == 1) *out = (uint16_t)(Kind<T>::pack(o[0] * inv, 0.f) & 0xffffu);
        else
#pragma unroll
            for (int e = 0; e < VEC; e += 2) reinterpret_cast<uint32_t*>(out)[e / 2] = Kind<T>::pack(o[e] * inv, o[e + 1] * inv);
        if (a.lse && lane == 0) a.lse[n_row * a.heads + head] = sum == 0.f ? -INFINITY : (top - Kind<T>::shift + log2f(sum)) * 0.693147180559945f;
    }
}

// The layer's keys and values in boxes of 64 components by as many positions as a page has whole boxes of (a multiple of the eight
// rows that the swizzle repeats after, at most `most`).  False where the pool has no such boxes (page_boxes), or pages of other sizes.
bool make_boxes(const PoolDev& p, AttendArgs& a, bool bf16, int most, CUtensorMap* map) {
    if (p.page_pos % 8) return false;
    int box = 8;
    for (int k = 16; k <= most; k += 8)
        if (p.page_pos % k == 0) box = k;
    if (!page_boxes(p, a.layer, bf16, box, map, a.box_dim)) return false;
    a.box_pos = box;
    a.boxes = most / box;
    a.tile_pos = box * a.boxes;
    return true;
}

template <class T, int D, int ROWS>
cudaError_t launch_join(const PoolDev& p, const BookDev& b, const AttendArgs& a, const AttendPlan& x, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(x.grid - 1, (x.part_rows + Join<ROWS>::rows - 1) / Join<ROWS>::rows);
    cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, join_kernel<T, D, ROWS>, p, b, a, x.grid);
}

}  // namespace
#endif

}  // namespace plc
