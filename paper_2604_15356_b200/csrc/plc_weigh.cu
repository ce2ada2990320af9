// Attention weights that cached positions receive (plc_pages_weigh), added up for eviction.
//
// weight[s][h][t] = decay weight[s][h][t] + sum over the session's newest rows i that see t, and over the query heads g of KV head h, of
// exp(scale q_ig . k_t - lse_ig), with the log-sum-exp that the attention has left: no maximum and no sum is carried, every tile of positions stands by itself.
//
// A warp takes tiles of 16 positions.  The product S = K Q^T has the positions as rows; the components may come in any order as long as K and Q have the same
// one, so a lane's 16 bytes of a key, as they come from the page, are its operands of two products: keys go from HBM to registers
// and never through shared memory, while the queries of a (session, head) stay in registers.  The exponentials of a tile's columns are summed in a fixed
// order by the lanes that share a position, and one lane adds the sum to the weight: the same call gives the same bits.
// All (session, head, tile) form one sequence, cut into equal ranges, one a warp.  A tile's keys are loaded while the one before is multiplied, its page is
// looked up a tile earlier still.  HBM bound: 64 sessions of up to 4096 positions, 8 x 4 heads of 128, one token each: 61 us on the device (355 MB, 5.8 TB/s); without the
// loads ahead 80 us.
// Products of this size are on the tensor cores' warp instructions, since nothing is to be gained by more: the tensor pipe is busy 8 % of the time.
#include <cuda_bf16.h>
#include <math.h>

#include "plc_weigh.cuh"

namespace plc {
namespace {

constexpr float kLog2e = 1.44269504088896f;

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <class T> __device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16816<__half>(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int kThreads = 128, kWarps = kThreads / 32, kTile = 16;
constexpr int64_t kNoKey = -1;                    // no offset: those are multiples of 16 bytes, of either sign

// NT: tiles of eight columns (a column: an entry's query head) that a warp has in registers.
// Blocks an SM: what the registers of the keys on their way, of the queries and of the rest leave.
template <int D, int NT> constexpr int kPerSm = D == 256 ? (NT == 1 ? 3 : 2) : D == 128 ? (NT == 1 ? 5 : 4) : NT == 1 ? 7 : 5;
template <class T, int D, int NT>
__global__ void __launch_bounds__(kThreads, kPerSm<D, NT>) weigh_kernel(const __grid_constant__ PoolDev p, const __grid_constant__ BookDev b, const __grid_constant__ WeighArgs a,
                                                         uint32_t* status) {
    constexpr int B = D / 32;                     // 32-component blocks of a vector
    __shared__ long long upto_s[kThreads];
    __shared__ long long warp_sum_s[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    // tiles of the sessions: a thread sums a run of them, the threads' sums are scanned
    const int run = (b.rows + kThreads - 1) / kThreads, first_s = min(b.rows, tid * run), last_s = min(b.rows, first_s + run);
    auto tiles_of = [&](int s, bool* bad) -> long long { return (long long)((newest_of(p, b, a, s, bad).len + kTile - 1) / kTile) * p.H; };
    long long mine = 0;
    bool any_bad = false;
    for (int s = first_s; s < last_s; ++s) {
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
    if (lane == 31) warp_sum_s[wid] = upto;
    __syncthreads();
    long long total = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < wid) upto += warp_sum_s[w];
        total += warp_sum_s[w];
    }
    upto_s[tid] = upto;
    __syncthreads();
    const long long workers = min((long long)gridDim.x * kWarps, total), me = (long long)blockIdx.x * kWarps + wid;
    if (me >= workers) return;
    const long long t0 = total * me / workers, t1 = total * (me + 1) / workers;
    int s = 0;
    long long rest = t0;
    {
        int j = 0;
        while (upto_s[j] <= t0) ++j;
        rest -= j ? upto_s[j - 1] : 0;
        s = j * run;
        bool bad;
        for (;; ++s) {
            const long long f = tiles_of(s, &bad);
            if (rest < f) break;
            rest -= f;
        }
    }
    long long left = t1 - t0;
    bool bad;
    Newest x = newest_of(p, b, a, s, &bad);
    int tiles = (x.len + kTile - 1) / kTile, h = (int)(rest / tiles), tile = (int)(rest - (long long)h * tiles);
    const int quad = lane >> 2, part = lane & 3;
    const float c2 = a.scale * kLog2e;
    // Where the vectors of tile i of the item stand, as far as this lane's position is concerned (kNoKey: it has none).  Looked up two tiles ahead, loaded one ahead.
    auto look_up = [&](int i) -> int64_t {
        const int t = i * kTile + (lane & 15);
        if (t >= x.len) return kNoKey;
        const int page = b.table[(int64_t)s * b.max_pages + t / p.page_pos];
        if (page < 0 || page >= p.n_pages) { atomicOr(status, kStRange); return kNoKey; }
        return (int64_t)a.layer * p.sl + (int64_t)page * p.spage + (int64_t)(t % p.page_pos) * p.sp + (int64_t)h * p.sh;
    };
    auto fetch = [&](int64_t off, uint4 (&k0)[B], uint4 (&k1)[B]) {
        const int64_t off0 = __shfl_sync(kFull, off, quad), off1 = __shfl_sync(kFull, off, quad + 8);
#pragma unroll
        for (int e = 0; e < B; ++e) {
            k0[e] = off0 == kNoKey ? make_uint4(0, 0, 0, 0) : __ldcs(reinterpret_cast<const uint4*>(p.base + off0 + e * 64 + part * 16));
            k1[e] = off1 == kNoKey ? make_uint4(0, 0, 0, 0) : __ldcs(reinterpret_cast<const uint4*>(p.base + off1 + e * 64 + part * 16));
        }
    };
    while (left > 0) {
        const int todo = (int)min(left, (long long)(tiles - tile)), cols = x.n * a.group;
        int64_t off = look_up(tile), next = todo > 1 ? look_up(tile + 1) : kNoKey;
        uint4 k0[B], k1[B];
        fetch(off, k0, k1);
        // the queries, a lane its column's run of components and log-sum-exp
        uint4 q[NT][B];
        float l_mine[NT];
        int entry[NT];
        auto queries = [&](int col0) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int col = col0 + n * 8 + quad;
                entry[n] = col / a.group;
                int row = -1;
                if (col < cols) row = a.rows ? a.rows[x.first + entry[n]] : x.first + entry[n];
                if (row < -1 || row >= a.n_rows) { atomicOr(status, kStRange); row = -1; }
                const int head = h * a.group + col - entry[n] * a.group;
                l_mine[n] = row < 0 ? INFINITY : a.lse[(int64_t)row * a.heads + head] * kLog2e;
                const uint16_t* from = a.q + (int64_t)max(row, 0) * a.qs_row + (int64_t)(row < 0 ? 0 : head) * a.qs_head + part * 8;
#pragma unroll
                for (int e = 0; e < B; ++e) q[n][e] = row < 0 ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(from + e * 32);
            }
        };
        queries(0);
        for (int i = 0; i < todo; ++i) {
            const int base = (tile + i) * kTile;
            const bool have0 = __shfl_sync(kFull, off, quad) != kNoKey, have1 = __shfl_sync(kFull, off, quad + 8) != kNoKey;
            float sum0 = 0.f, sum1 = 0.f;
            const int seen0 = base + quad - (x.len - x.n), seen1 = seen0 + 8;             // entries from this one on see the position
            // sessions of more columns than the call's mean take them in turns
            for (int col0 = 0; col0 < cols; col0 += 8 * NT) {
                if (cols > 8 * NT && (i > 0 || col0 > 0)) queries(col0);
                float acc[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[n][j] = 0.f;
#pragma unroll
                    for (int e = 0; e < B; ++e) {
                        mma16816<T>(acc[n], k0[e].x, k1[e].x, k0[e].y, k1[e].y, q[n][e].x, q[n][e].y);
                        mma16816<T>(acc[n], k0[e].z, k1[e].z, k0[e].w, k1[e].w, q[n][e].z, q[n][e].w);
                    }
                }
                if (col0 + 8 * NT >= cols) {      // the keys are not needed any more
                    off = next;
                    if (i + 1 < todo) fetch(off, k0, k1);
                    next = i + 2 < todo ? look_up(tile + i + 2) : kNoKey;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) { // columns 2 part + j
                        const float l = __shfl_sync(kFull, l_mine[n], (2 * part + j) * 4);
                        const int en = __shfl_sync(kFull, entry[n], (2 * part + j) * 4);
                        const bool dead = isinf(l);
                        sum0 += dead || en < seen0 ? 0.f : exp2_approx(fmaf(acc[n][j], c2, -l));
                        sum1 += dead || en < seen1 ? 0.f : exp2_approx(fmaf(acc[n][2 + j], c2, -l));
                    }
            }
            sum0 += __shfl_xor_sync(kFull, sum0, 1);
            sum1 += __shfl_xor_sync(kFull, sum1, 1);
            sum0 += __shfl_xor_sync(kFull, sum0, 2);
            sum1 += __shfl_xor_sync(kFull, sum1, 2);
            const int t = base + quad + 8 * part;
            if (part < 2 && t < x.len) put_weight(a, x, s, h, t, part ? sum1 : sum0, part ? have1 : have0, status);
        }
        left -= todo;
        tile = 0;
        if (left > 0 && ++h == p.H) {
            h = 0;
            do x = newest_of(p, b, a, ++s, &bad);
            while (x.len == 0);
            tiles = (x.len + kTile - 1) / kTile;
        }
    }
}

template <class T, int D>
cudaError_t launch(const PoolDev& p, const BookDev& b, const WeighArgs& a, uint32_t* status, cudaStream_t st) {
    const unsigned sms = sm_count();
    return (long long)a.n_list * a.group <= 8ll * b.rows ? launch_kernel(weigh_kernel<T, D, 1>, kPerSm<D, 1> * sms, kThreads, 0, st, false, 1, p, b, a, status)
                                                         : launch_kernel(weigh_kernel<T, D, 2>, kPerSm<D, 2> * sms, kThreads, 0, st, false, 1, p, b, a, status);
}
template <class T>
cudaError_t launch_weigh(const PoolDev& p, const BookDev& b, const WeighArgs& a, uint32_t* status, cudaStream_t st) {
    switch (p.d) {
        case 32: return launch<T, 32>(p, b, a, status, st);
        case 64: return launch<T, 64>(p, b, a, status, st);
        case 128: return launch<T, 128>(p, b, a, status, st);
        default: return launch<T, 256>(p, b, a, status, st);
    }
}

// Columns (entries times the query heads of a group) a session beyond which the other kernel takes the call, by the mean, which is what the host knows.  Half as many sessions as
// above, us a call, here and there: 16 columns 37 and 54 (before its boxes had a warp of their own; now 44), 32 columns 65 and 44; with queries in shared memory 32 columns took 64 here, 64
// columns 137.
constexpr int kFewColumns = 16;
bool many_columns(const PoolDev& p, int sessions, int heads, int n_list) { return (long long)n_list * (heads / p.H) > (long long)kFewColumns * sessions; }

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" {

plc_status plc_pages_weigh_workspace(const plc_page_pool* pool, int32_t sessions, int32_t n_heads, int32_t n_list, uint64_t* bytes) {
    PoolDev p;
    const plc_status rc = check_pool(pool, &p);
    if (rc) return rc;
    if (n_heads < 1 || sessions < 1 || n_list < 0 || !bytes) return PLC_E_INVALID;
    if (n_heads % p.H || n_heads > (1 << 16)) return PLC_E_SHAPE;
    *bytes = many_columns(p, sessions, n_heads, n_list) ? weigh_many_bytes() : 0;
    return PLC_OK;
}

plc_status plc_pages_weigh(const plc_page_pool* pool, int32_t layer, const plc_page_book* book, const plc_weigh_queries* t, float scale, float decay,
                           const plc_weights* weights, void* workspace_dev, uint64_t workspace_bytes, uint32_t* status_dev, void* stream) {
    PoolDev p;
    BookDev b;
    plc_status rc = check_pool(pool, &p);
    if (rc || (rc = check_book(book, &b))) return rc;
    if (!t || !t->q_dev || !t->lse_dev || !t->begin_dev || t->n_rows < 0 || t->n_list < 0 || !weights || !weights->base_dev || !status_dev) return PLC_E_INVALID;
    if (layer < 0 || layer >= p.L || pool->dtype == PLC_OUT_F32 || !(scale > 0.f) || isinf(scale) || !isfinite(decay) || decay < 0.f) return PLC_E_INVALID;
    if (t->n_heads < 1 || weights->n_pos < 1) return PLC_E_INVALID;
    if (!runs_apart(weights->stride_row, b.rows, weights->stride_head, p.H, weights->n_pos) || (p.L > 1 && weights->stride_layer == 0)) return PLC_E_INVALID;
    if (t->n_heads % p.H || t->n_heads > (1 << 16) || (!t->rows_dev && t->n_list > t->n_rows)) return PLC_E_SHAPE;
    const int group = t->n_heads / p.H;
    if ((long long)t->n_list * group > (1 << 30)) return PLC_E_SHAPE;
    const bool many = many_columns(p, b.rows, t->n_heads, t->n_list);
    if (many && !workspace_dev) return PLC_E_INVALID;
    if (!plc_aligned16(workspace_dev) || !plc_aligned16(t->q_dev) || t->q_stride_row % 8 || t->q_stride_head % 8 || (reinterpret_cast<uintptr_t>(weights->base_dev) & 3)) return PLC_E_ALIGN;
    if (workspace_bytes < (many ? weigh_many_bytes() : 0)) return PLC_E_CAPACITY;
    if (t->n_list == 0) return PLC_OK;
    const WeighArgs a{static_cast<const uint16_t*>(t->q_dev), t->q_stride_row, t->q_stride_head, t->lse_dev, t->rows_dev, t->begin_dev, t->n_list, t->n_rows, t->n_heads,
                      group, layer, weights->base_dev + (int64_t)layer * weights->stride_layer, weights->stride_row, weights->stride_head, weights->n_pos, decay, scale, nullptr, nullptr, 0, {}, 0};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (many) {
        if (launch_weigh_many(p, b, a, workspace_dev, pool->dtype == PLC_OUT_BF16, status_dev, st) != cudaSuccess) return PLC_E_CUDA;
        count_launch(2);
        return PLC_OK;
    }
    if ((pool->dtype == PLC_OUT_F16 ? launch_weigh<__half>(p, b, a, status_dev, st) : launch_weigh<__nv_bfloat16>(p, b, a, status_dev, st)) != cudaSuccess) return PLC_E_CUDA;
    count_launch(1);
    return PLC_OK;
}

}  // extern "C"
