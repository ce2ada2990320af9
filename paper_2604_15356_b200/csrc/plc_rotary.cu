// Rotary positions: tensors of queries and keys are turned (plc_rotary_apply), and new tokens' keys are turned on their way into the pages, values
// beside them (plc_pages_append).
//
// A pair (x_a, x_b) of components at position pos becomes s (x_a cos t - x_b sin t, x_b cos t + x_a sin t), t = pos f_i.  The frequency is held in turns a
// position as a fraction of 64 bits, so that the product with the position, cut to its low 64 bits, is the angle modulo a turn to 2^-32 turns at any
// position that an int holds: no product in 64-bit floating point and no reduction.  The functions take it in binary32, which is off by up to 2^-26 turns (half a step just
// below half a turn, 9e-8 rad), about as much as sines of binary32 are off anyway.  They are formed once a row and pair, for all heads.
//
// Bound by HBM where rows are many (each component read and written once, 16 bytes a thread and access), by the launch where they are few.  A block takes a few
// rows with all their heads.
#include <cuda_bf16.h>
#include <math.h>

#include "plc_pages.cuh"

namespace plc {
namespace {

constexpr int kTurnThreads = 256, kMostRows = 8;  // of a block
constexpr int kMostSets = 4, kMostDim = 1024;

struct TurnSet {
    const uint8_t* x; uint8_t* out;
    int64_t xs_row, xs_head, os_row, os_head;     // bytes
    int heads, dim;                               // dim: components that turn
    int per_head;                                 // units of a head: runs, or pairs and components
    int first;                                    // unit of a row that the set begins with
};
struct TurnArgs {
    TurnSet set[kMostSets];
    int sets, units;                              // units of a row
    const uint64_t* turns; int pairs; float scale; bool back; int lanes;             // lanes: of a row, where rows share a warp
    const int32_t* pos; int rows, d, rows_block, shares;             // shares: warps that share a row
    const int32_t* begin; int layer;              // pages: ranges of the sessions' rows
};

template <class T> struct Wide;
template <> struct Wide<float> {
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Wide<__half> {
    static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};
template <> struct Wide<__nv_bfloat16> {
    static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};

// A run of W components: 16, 8 or 4 bytes.
template <class T, int W> struct Run {
    static constexpr int bytes = W * (int)sizeof(T);
    alignas(bytes) T v[W];
    __device__ __forceinline__ void load(const uint8_t* p) {
        if constexpr (bytes == 16) *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(p);
        else if constexpr (bytes == 8) *reinterpret_cast<uint2*>(v) = *reinterpret_cast<const uint2*>(p);
        else *reinterpret_cast<uint32_t*>(v) = *reinterpret_cast<const uint32_t*>(p);
    }
    __device__ __forceinline__ void store(uint8_t* p) const {
        if constexpr (bytes == 16) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(v);
        else if constexpr (bytes == 8) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(v);
        else *reinterpret_cast<uint32_t*>(p) = *reinterpret_cast<const uint32_t*>(v);
    }
};
// Bytes of a run: 16 where strides, addresses, the turned part, its halves and the rest allow it, else 4 (two neighbours of binary32: 8).
constexpr int run_bytes(bool wide, int esz, bool inter) { return wide ? 16 : esz == 4 && inter ? 8 : 4; }

// The session of row i: the last one whose range begins at or before it; -1 where it is in none.  A warp calls it.
__device__ __forceinline__ int session_of_row(const int32_t* begin, int sessions, int i) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = sessions;
    for (;;) {
        const int step = (hi - lo + 31) / 32, at = lo + min(lane, (hi - lo - 1) / step) * step;
        const uint32_t m = __ballot_sync(kFull, begin[at] <= i);
        if (m == 0) return -1;
        const int j = min(31 - __clz(m), (hi - lo - 1) / step);
        lo += j * step;
        hi = min(hi, lo + step);
        if (step == 1) break;
    }
    return begin[lo] <= i && i < begin[lo + 1] ? lo : -1;
}

// The angle of a pair at a position: cosine and sine, times the magnitude.
__device__ __forceinline__ float2 turn_of(const TurnArgs& a, int pos, int pair) {
    const uint64_t angle = (uint64_t)(int64_t)pos * a.turns[pair] + (1ull << 31);
    float s, c;
    sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, &s, &c);
    return make_float2(c * a.scale, a.back ? -s * a.scale : s * a.scale);
}

// Where row i stands: its session's position and the place of its key, in bytes from the layer's first one (kNowhere: it has none; offsets are
// multiples of 16, of either sign).  A warp calls it; false where the row is in no range.
constexpr int64_t kNowhere = -1;
__device__ __forceinline__ bool place_of(const TurnArgs& a, const PoolDev& p, const BookDev& b, int i, int* pos, int64_t* to, uint32_t* status) {
    const int s = session_of_row(a.begin, b.rows, i);
    if (s < 0) return false;
    const int len = b.len[s];
    const long long t = (long long)len + (i - a.begin[s]);
    int page = -1;
    if (len >= 0 && t < most_positions(b, p)) page = b.table[(int64_t)s * b.max_pages + t / p.page_pos];
    *to = page >= 0 && page < p.n_pages && b.ref[page] == 1 ? (int64_t)page * p.spage + (int64_t)(t % p.page_pos) * p.sp : kNowhere;
    if (*to == kNowhere && (threadIdx.x & 31) == 0) atomicOr(status, kStRange);
    *pos = a.pos ? a.pos[i] : (int)t;
    return true;
}
// Ranges that do not rise.
__device__ __forceinline__ void check_ranges(const TurnArgs& a, const BookDev& b, uint32_t* status) {
    bool bad = false;
    for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < b.rows; s += gridDim.x * blockDim.x) bad |= a.begin[s] < 0 || a.begin[s + 1] < a.begin[s] || a.begin[s + 1] > a.rows;
    if (bad) atomicOr(status, kStRange);
}

// A warp takes a row's heads, or a share of them: a lane has the same run of every head, whose cosines and sines it keeps in registers, and as
// many heads at a time as the runs of one leave lanes for.  64 bytes a lane on their way and eight blocks an SM: 16384 rows of 32 + 8 heads of 128 in bf16 63.7 us (5.3 TB/s),
// with twice as many bytes a lane and four blocks 70; cosines and sines read again for each head 66 to 74.  INTER: pairs are neighbours, else half a turned part away.
constexpr int kRowThreads = 128;
template <class T, bool INTER, bool PAGES, bool WIDE>
__global__ void __launch_bounds__(kRowThreads, 8) turn_rows_kernel(const __grid_constant__ TurnArgs a, const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b,
                                                                uint32_t* status) {
    constexpr int bytes = run_bytes(WIDE, sizeof(T), INTER), W = bytes / (int)sizeof(T), P = INTER ? W / 2 : W, U = WIDE && !INTER ? 2 : 4;        // components and pairs of a run; heads a lane has on their way
    extern __shared__ float2 turn_s[];                                          // [warps][pairs]
    if (PAGES) check_ranges(a, b, status);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const long long at = (long long)blockIdx.x * (kRowThreads / 32) + wid;
    const int i = (int)(at / a.shares), share = (int)(at - (long long)i * a.shares);
    if (i >= a.rows) return;
    int pos;
    int64_t row_to = kNowhere;
    if (PAGES) {
        if (!place_of(a, p, b, i, &pos, &row_to, status)) return;
    } else pos = a.pos[i];
    float2* turn = turn_s + wid * a.pairs;
    for (int k = lane; k < a.pairs; k += 32) turn[k] = turn_of(a, pos, k);
    __syncwarp();
    auto address = [&](int t, int h) -> uint8_t* {                              // of a head of set t where it goes; null: nowhere
        if (PAGES && t > 0) return row_to == kNowhere ? nullptr : p.base + (int64_t)a.layer * p.sl + (t == 2 ? p.skv : 0) + row_to + (int64_t)h * p.sh;
        return a.set[t].out + (int64_t)i * a.set[t].os_row + (int64_t)h * a.set[t].os_head;
    };
#pragma unroll 1
    for (int t = 0; t < a.sets; ++t) {
        const TurnSet& s = a.set[t];
        const int lo = s.heads * share / a.shares, hi = s.heads * (share + 1) / a.shares;
        if (lo == hi || (PAGES && t > 0 && row_to == kNowhere)) continue;
        const uint8_t* from = s.x + (int64_t)i * s.xs_row;
        const int turned = s.dim / W / (INTER ? 1 : 2), wide = min(s.per_head, 32), abreast = 32 / wide, h0 = lo + lane / wide;
        const int64_t half = (int64_t)s.dim / 2 * (int)sizeof(T);
#pragma unroll 1
        for (int e0 = 0; e0 < s.per_head; e0 += 32) {
            const int e = e0 + lane % wide;
            if (lane >= abreast * wide || e >= s.per_head) continue;
            const bool turns = e < turned;
            const int64_t off = turns ? (int64_t)e * bytes : (int64_t)s.dim * (int)sizeof(T) + (int64_t)(e - turned) * bytes;
            float2 cs[P];
            if (turns) {
#pragma unroll
                for (int k = 0; k < P; ++k) cs[k] = turn[e * P + k];
            }
#pragma unroll 1
            for (int h = h0; h < hi; h += U * abreast) {
                Run<T, W> x[U], y[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (h + u * abreast < hi) {
                        const uint8_t* src = from + (int64_t)(h + u * abreast) * s.xs_head + off;
                        x[u].load(src);
                        if (!INTER && turns) y[u].load(src + half);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (h + u * abreast < hi) {
                        uint8_t* dst = address(t, h + u * abreast) + off;
                        if (turns) {
#pragma unroll
                            for (int k = 0; k < P; ++k) {
                                T& a0 = x[u].v[INTER ? 2 * k : k];
                                T& b0 = INTER ? x[u].v[2 * k + 1 < W ? 2 * k + 1 : 0] : y[u].v[k];
                                const float xa = Wide<T>::get(a0), xb = Wide<T>::get(b0);
                                a0 = Wide<T>::put(xa * cs[k].x - xb * cs[k].y);
                                b0 = Wide<T>::put(xb * cs[k].x + xa * cs[k].y);
                            }
                            if (!INTER) y[u].store(dst + half);
                        }
                        x[u].store(dst);
                    }
            }
        }
    }
}

// The same for rows of few runs, several of which share a warp (a.lanes lanes each): the heads of all sets are taken as if they were one set's.  The blocks stay,
// and the next row's position is on its way while one is turned.
// A warp a row leaves most lanes without a load there.  Measured, rows of heads: 67732 of 2 + 2 of 32 in bf16 58 -> 12.5 us, 73352 of 2 + 2 of 128 (64 turned) in fp16
// 70 -> 43, 47345 of 2 + 2 of 80 in binary32 46 -> 27.
template <class T, bool INTER, bool WIDE>
__global__ void __launch_bounds__(kRowThreads, 8) turn_small_kernel(const __grid_constant__ TurnArgs a) {
    constexpr int bytes = run_bytes(WIDE, sizeof(T), INTER), W = bytes / (int)sizeof(T), P = INTER ? W / 2 : W, U = WIDE && !INTER ? 2 : 4;
    extern __shared__ float2 turn_s[];                                          // [rows of the block][pairs]
    const int lanes = a.lanes, log2 = __ffs(lanes) - 1, sub = (threadIdx.x & 31) >> log2, lane = threadIdx.x & (lanes - 1);
    const int rows_warp = 32 >> log2, wid = threadIdx.x >> 5, step = gridDim.x * (kRowThreads / 32);
    float2* turn = turn_s + (wid * rows_warp + sub) * a.pairs;
    const int dim = a.set[0].dim, per_head = a.set[0].per_head, turned = dim / W / (INTER ? 1 : 2), half = dim / 2 * (int)sizeof(T);
    const int wide = min(per_head, lanes), abreast = lanes / wide, heads = a.units / per_head;
    const int last = (a.rows - 1) / rows_warp;
    int at = blockIdx.x * (kRowThreads / 32) + wid, i = at * rows_warp + sub, next_pos = at <= last && i < a.rows ? a.pos[i] : 0;
    for (; at <= last; at += step) {
        i = at * rows_warp + sub;
        const int pos = next_pos;
        if (at + step <= last && i + step * rows_warp < a.rows) next_pos = a.pos[i + step * rows_warp];
        __syncwarp();                             // the row before has been turned
        for (int k = lane; k < a.pairs; k += lanes) turn[k] = turn_of(a, pos, k);
        __syncwarp();
        if (i >= a.rows) continue;
#pragma unroll 1
        for (int e0 = 0; e0 < per_head; e0 += lanes) {
            const int e = e0 + lane % wide;
            if (lane >= abreast * wide || e >= per_head) continue;
            const bool turns = e < turned;
            const int off = turns ? e * bytes : dim * (int)sizeof(T) + (e - turned) * bytes;
            float2 cs[P];
            if (turns) {
#pragma unroll
                for (int k = 0; k < P; ++k) cs[k] = turn[e * P + k];
            }
#pragma unroll 1
            for (int h0 = lane / wide; h0 < heads; h0 += U * abreast) {
                Run<T, W> x[U], y[U];
                uint8_t* to[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    int h = h0 + u * abreast, t = 0;
                    to[u] = nullptr;
                    if (h >= heads) continue;
#pragma unroll
                    for (int k = 0; k + 1 < kMostSets; ++k)
                        if (h >= a.set[t].heads) h -= a.set[t++].heads;
                    const TurnSet& s = a.set[t];
                    const uint8_t* from = s.x + (int64_t)i * s.xs_row + (int64_t)h * s.xs_head + off;
                    to[u] = s.out + (int64_t)i * s.os_row + (int64_t)h * s.os_head + off;
                    x[u].load(from);
                    if (!INTER && turns) y[u].load(from + half);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (to[u]) {
                        if (turns) {
#pragma unroll
                            for (int k = 0; k < P; ++k) {
                                T& a0 = x[u].v[INTER ? 2 * k : k];
                                T& b0 = INTER ? x[u].v[2 * k + 1 < W ? 2 * k + 1 : 0] : y[u].v[k];
                                const float xa = Wide<T>::get(a0), xb = Wide<T>::get(b0);
                                a0 = Wide<T>::put(xa * cs[k].x - xb * cs[k].y);
                                b0 = Wide<T>::put(xb * cs[k].x + xa * cs[k].y);
                            }
                            if (!INTER) y[u].store(to[u] + half);
                        }
                        x[u].store(to[u]);
                    }
            }
        }
    }
}

// Component by component, where addresses, strides or parts of a head allow no runs.  A block takes a few rows with all their heads.
template <class T, bool INTER, bool PAGES>
__global__ void __launch_bounds__(kTurnThreads) turn_parts_kernel(const __grid_constant__ TurnArgs a, const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b,
                                                                  uint32_t* status) {
    extern __shared__ float2 turn[];              // [rows of the block][pairs] cosine, sine
    __shared__ int64_t row_to[kMostRows];         // where a row's key goes, or kNowhere
    __shared__ int row_pos[kMostRows];            // its position; the row is in some range
    __shared__ bool row_in[kMostRows];
    const int tid = threadIdx.x, r0 = blockIdx.x * a.rows_block, rows = min(a.rows_block, a.rows - r0);
    if (PAGES) {
        check_ranges(a, b, status);
        const int w = tid >> 5;
        if (w < rows) {
            int pos = 0;
            int64_t to = kNowhere;
            const bool in = place_of(a, p, b, r0 + w, &pos, &to, status);
            if ((tid & 31) == 0) { row_to[w] = to; row_in[w] = in; row_pos[w] = pos; }
        }
    } else if (tid < rows) row_pos[tid] = a.pos[r0 + tid];
    __syncthreads();
    for (int i = tid; i < rows * a.pairs; i += kTurnThreads) turn[i] = turn_of(a, row_pos[i / a.pairs], i % a.pairs);
    __syncthreads();
    const int units = rows * a.units;
    for (int u = tid; u < units; u += kTurnThreads) {
        const int r = a.rows_block == 1 ? 0 : u / a.units, v = u - r * a.units;
        int t = 0;
#pragma unroll
        for (int i = 1; i < kMostSets; ++i) t += i < a.sets && v >= a.set[i].first;
        const TurnSet& s = a.set[t];
        const int w = v - s.first, h = w / s.per_head, e = w - h * s.per_head;
        if (PAGES && (t > 0 ? row_to[r] == kNowhere : !row_in[r])) continue;
        const T* from = reinterpret_cast<const T*>(s.x + (int64_t)(r0 + r) * s.xs_row + (int64_t)h * s.xs_head);
        T* to = reinterpret_cast<T*>(PAGES && t > 0 ? p.base + (int64_t)a.layer * p.sl + (t == 2 ? p.skv : 0) + row_to[r] + (int64_t)h * p.sh
                                                    : s.out + (int64_t)(r0 + r) * s.os_row + (int64_t)h * s.os_head);
        if (e < s.dim / 2) {
            const int ia = INTER ? 2 * e : e, ib = INTER ? 2 * e + 1 : e + s.dim / 2;
            const float2 cs = turn[r * a.pairs + e];
            const float xa = Wide<T>::get(from[ia]), xb = Wide<T>::get(from[ib]);
            to[ia] = Wide<T>::put(xa * cs.x - xb * cs.y);
            to[ib] = Wide<T>::put(xb * cs.x + xa * cs.y);
        } else to[e + s.dim / 2] = from[e + s.dim / 2];
    }
}

// Whether runs of so many bytes cover the turned part, its halves and the rest of every set, and start on their boundaries.
bool in_runs(const TurnArgs& a, bool inter, int esz, int bytes) {
    for (int i = 0; i < a.sets; ++i) {
        const TurnSet& s = a.set[i];
        if (s.heads == 0) continue;
        const uintptr_t bits = reinterpret_cast<uintptr_t>(s.x) | reinterpret_cast<uintptr_t>(s.out) | (uintptr_t)s.xs_row | (uintptr_t)s.xs_head | (uintptr_t)s.os_row |
                               (uintptr_t)s.os_head | (uintptr_t)((inter ? s.dim : s.dim / 2) * esz) | (uintptr_t)((a.d - s.dim) * esz);
        if (bits & (bytes - 1)) return false;
    }
    return true;
}

// Units of the sets, and the launch.
template <bool PAGES>
plc_status launch_turn(TurnArgs& a, const PoolDev& p, const BookDev& b, int dtype, bool inter, uint32_t* status, cudaStream_t st) {
    const int esz = dtype == PLC_OUT_F32 ? 4 : 2, sms = sm_count();
    const bool wide = in_runs(a, inter, esz, 16), runs = wide || in_runs(a, inter, esz, run_bytes(false, esz, inter));
    const int w = run_bytes(wide, esz, inter) / esz;
    int units = 0;
    for (int i = 0; i < a.sets; ++i) {
        TurnSet& s = a.set[i];
        s.per_head = runs ? (inter ? s.dim / w : s.dim / 2 / w) + (a.d - s.dim) / w : s.dim / 2 + a.d - s.dim;
        s.first = units;
        units += s.heads * s.per_head;
    }
    auto go = [&](auto* kern, unsigned grid, int threads, size_t smem) { return launch_kernel(kern, grid, threads, smem, st, false, 1, a, p, b, status); };
    cudaError_t e;
    if (runs) {
        // warps that share a row: so many that there are sixteen an SM, as long as each has the runs of a load for all of its lanes
        const long long want = (16ll * sms + a.rows - 1) / a.rows, most = (units + 127) / 128;
        a.shares = (int)(want < most ? want : most);
        a.units = units;
        // or, where rows are many and small, rows that share a warp: as few lanes as leave each two rounds of loads.  40000 rows of 4 + 4 heads of 128 in bf16: halves
        // 36.5 us (twice the loads a lane 41), neighbours 39 (half the loads 47)
        a.lanes = 32;
        const int loads = wide && !inter ? 4 : 8;
        if (!PAGES && a.shares == 1)
            while (a.lanes > 4 && units <= loads * a.lanes / 2) a.lanes /= 2;
        constexpr int warps = kRowThreads / 32;
        const bool small = a.lanes < 32;
        const long long full = ((long long)a.rows * a.shares * a.lanes / 32 + warps) / warps, stay = 8ll * sms;
        const unsigned grid = (unsigned)(small ? (full < stay ? full : stay) : ((long long)a.rows * a.shares + warps - 1) / warps);
        const size_t smem = (size_t)warps * (32 / a.lanes) * a.pairs * sizeof(float2);
        auto rows = [&](auto* wide_inter, auto* wide_half, auto* inter_kern, auto* half) { return wide ? (inter ? wide_inter : wide_half) : inter ? inter_kern : half; };
#define PLC_TURN(T) go(rows(turn_rows_kernel<T, true, PAGES, true>, turn_rows_kernel<T, false, PAGES, true>, turn_rows_kernel<T, true, PAGES, false>, turn_rows_kernel<T, false, PAGES, false>), grid, kRowThreads, smem)
#define PLC_TURN_SMALL(T) launch_kernel(rows(turn_small_kernel<T, true, true>, turn_small_kernel<T, false, true>, turn_small_kernel<T, true, false>, turn_small_kernel<T, false, false>), grid, kRowThreads, smem, st, false, 1, a)
        if (small) e = dtype == PLC_OUT_F32 ? PLC_TURN_SMALL(float) : dtype == PLC_OUT_F16 ? PLC_TURN_SMALL(__half) : PLC_TURN_SMALL(__nv_bfloat16);
        else e = dtype == PLC_OUT_F32 ? PLC_TURN(float) : dtype == PLC_OUT_F16 ? PLC_TURN(__half) : PLC_TURN(__nv_bfloat16);
#undef PLC_TURN_SMALL
#undef PLC_TURN
    } else {
        // rows of a block so that there are several blocks an SM
        const int per = a.rows / (4 * sms);
        a.units = units;
        a.rows_block = per < 1 ? 1 : per > kMostRows ? kMostRows : per;
        const unsigned grid = (unsigned)((a.rows + a.rows_block - 1) / a.rows_block);
        const size_t smem = (size_t)a.rows_block * a.pairs * sizeof(float2);
        auto parts = [&](auto* inter_kern, auto* half) { return go(inter ? inter_kern : half, grid, kTurnThreads, smem); };
#define PLC_TURN(T) parts(turn_parts_kernel<T, true, PAGES>, turn_parts_kernel<T, false, PAGES>)
        e = dtype == PLC_OUT_F32 ? PLC_TURN(float) : dtype == PLC_OUT_F16 ? PLC_TURN(__half) : PLC_TURN(__nv_bfloat16);
#undef PLC_TURN
    }
    if (e != cudaSuccess) return PLC_E_CUDA;
    count_launch(1);
    return PLC_OK;
}

plc_status check_rotary(const plc_rotary* r, int head_dim, TurnArgs* a) {
    if (!r || !r->turns_dev) return PLC_E_INVALID;
    if (r->dim < 2 || r->dim % 2 || r->dim > head_dim) return PLC_E_SHAPE;
    if (!isfinite(r->scale)) return PLC_E_INVALID;
    if (reinterpret_cast<uintptr_t>(r->turns_dev) & 7) return PLC_E_ALIGN;
    a->turns = r->turns_dev;
    a->pairs = r->dim / 2;
    a->scale = r->scale;
    return PLC_OK;
}
}  // namespace
}  // namespace plc

using namespace plc;

extern "C" {

plc_status plc_rotary_turns(const double* radians, int32_t n, uint64_t* turns) {
    if (!radians || !turns || n < 1) return PLC_E_INVALID;
    for (int i = 0; i < n; ++i) {
        const double f = radians[i];
        if (!(f >= 0.0) || f > 65536.0) return PLC_E_INVALID;
        // f = m 2^(e - 53); turns = m / (2 pi) 2^(e - 53 + 64).  1 / (2 pi) = 0x28BE60DB9391054A 7F09D5F47D4D3770 2^-128
        int e;
        const uint64_t m = (uint64_t)ldexp(frexp(f, &e), 53);
        const unsigned __int128 lo = (unsigned __int128)m * 0x7F09D5F47D4D3770ull, hi = (unsigned __int128)m * 0x28BE60DB9391054Aull + (uint64_t)(lo >> 64);
        // m / (2 pi) = (hi 2^64 + (low half of lo)) 2^-128; times 2^(e + 11), rounded
        const int shift = 53 - e;                 // of hi, to the right: at least 36
        if (shift > 126) { turns[i] = 0; continue; }
        turns[i] = (uint64_t)((hi + ((unsigned __int128)1 << (shift - 1))) >> shift);
    }
    return PLC_OK;
}

plc_status plc_rotary_apply(const plc_rotary* rotary, const plc_rotary_set* sets, int32_t n_sets, const int32_t* pos_dev, int32_t n_rows, int32_t head_dim,
                            int32_t dtype, int32_t back, void* stream) {
    TurnArgs a{};
    if (!sets || n_sets < 1 || !pos_dev || n_rows < 0 || head_dim < 2) return PLC_E_INVALID;
    if (dtype != PLC_OUT_F32 && dtype != PLC_OUT_F16 && dtype != PLC_OUT_BF16) return PLC_E_INVALID;
    if (n_sets > kMostSets || head_dim > kMostDim) return PLC_E_SHAPE;
    const plc_status rc = check_rotary(rotary, head_dim, &a);
    if (rc) return rc;
    const int esz = dtype == PLC_OUT_F32 ? 4 : 2;
    long long heads = 0;
    for (int i = 0; i < n_sets; ++i) {
        if (sets[i].heads < 1) return PLC_E_INVALID;
        heads += sets[i].heads;
    }
    if (heads > (1 << 12)) return PLC_E_SHAPE;
    for (int i = 0; i < n_sets; ++i) {
        const plc_rotary_set& s = sets[i];
        if (!s.x_dev || !s.out_dev) return PLC_E_INVALID;
        if ((reinterpret_cast<uintptr_t>(s.x_dev) | reinterpret_cast<uintptr_t>(s.out_dev)) & (esz - 1)) return PLC_E_ALIGN;
        if (s.x_dev == s.out_dev && ((n_rows > 1 && s.x_stride_row != s.out_stride_row) || (s.heads > 1 && s.x_stride_head != s.out_stride_head))) return PLC_E_INVALID;
        if (n_rows > 0 && !runs_apart(s.out_stride_row, n_rows, s.out_stride_head, s.heads, head_dim)) return PLC_E_INVALID;     // results on top of each other
        a.set[i] = TurnSet{static_cast<const uint8_t*>(s.x_dev), static_cast<uint8_t*>(s.out_dev), s.x_stride_row * esz, s.x_stride_head * esz, s.out_stride_row * esz,
                           s.out_stride_head * esz, s.heads, rotary->dim, 0, 0};
    }
    if (n_rows == 0) return PLC_OK;
    a.sets = n_sets; a.back = back != 0; a.pos = pos_dev; a.rows = n_rows; a.d = head_dim;
    return launch_turn<false>(a, PoolDev{}, BookDev{}, dtype, rotary->interleaved != 0, nullptr, static_cast<cudaStream_t>(stream));
}

plc_status plc_pages_append(const plc_page_pool* pool, int32_t layer, const plc_page_book* book, const plc_rotary* rotary, const plc_new_tokens* t,
                            uint32_t* status_dev, void* stream) {
    PoolDev p;
    BookDev b;
    TurnArgs a{};
    plc_status rc = check_pool(pool, &p);
    if (rc || (rc = check_book(book, &b))) return rc;
    if (!t || !t->k_dev || !t->v_dev || !t->begin_dev || t->n_rows < 0 || t->n_heads < 0 || !status_dev || layer < 0 || layer >= p.L) return PLC_E_INVALID;
    if (t->n_heads > 0 && (!t->q_dev || !t->out_dev)) return PLC_E_INVALID;
    if (rotary && (rc = check_rotary(rotary, p.d, &a))) return rc;
    if ((long long)t->n_heads + 2 * p.H > (1 << 14)) return PLC_E_SHAPE;
    const int esz = p.esz, dim = rotary ? rotary->dim : 0;
    const bool inter = rotary && rotary->interleaved;
    if ((reinterpret_cast<uintptr_t>(t->k_dev) | reinterpret_cast<uintptr_t>(t->v_dev) | reinterpret_cast<uintptr_t>(t->n_heads ? t->q_dev : nullptr) |
         reinterpret_cast<uintptr_t>(t->n_heads ? t->out_dev : nullptr)) & (esz - 1))
        return PLC_E_ALIGN;
    if (t->n_heads > 0 && t->q_dev == t->out_dev &&
        ((t->n_rows > 1 && t->q_stride_row != t->out_stride_row) || (t->n_heads > 1 && t->q_stride_head != t->out_stride_head)))
        return PLC_E_INVALID;
    if (t->n_heads > 0 && t->n_rows > 0 && !runs_apart(t->out_stride_row, t->n_rows, t->out_stride_head, t->n_heads, p.d)) return PLC_E_INVALID;
    if (t->n_rows == 0) return PLC_OK;
    a.set[0] = TurnSet{static_cast<const uint8_t*>(t->q_dev), static_cast<uint8_t*>(t->out_dev), t->q_stride_row * esz, t->q_stride_head * esz, t->out_stride_row * esz,
                       t->out_stride_head * esz, t->n_heads, dim, 0, 0};
    a.set[1] = TurnSet{static_cast<const uint8_t*>(t->k_dev), nullptr, t->k_stride_row * esz, t->k_stride_head * esz, 0, 0, p.H, dim, 0, 0};
    a.set[2] = TurnSet{static_cast<const uint8_t*>(t->v_dev), nullptr, t->v_stride_row * esz, t->v_stride_head * esz, 0, 0, p.H, 0, 0, 0};
    a.sets = 3; a.pos = t->pos_dev; a.rows = t->n_rows; a.d = p.d; a.begin = t->begin_dev; a.layer = layer;
    return launch_turn<true>(a, p, b, pool->dtype, inter, status_dev, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
