// Attention of drafted tokens over their session's pages (plc_tree_attention).
#include <cuda_bf16.h>

#include "plc_pages.cuh"

namespace plc {
namespace {

struct AttendArgs {
    const void* q; int64_t qs_row, qs_head;       // elements
    void* out; int64_t os_row, os_head;
    float* lse;
    const int32_t* begin; const uint32_t* mask;
    int rows, heads, group, mask_words, layer;
    float scale;
};

template <class T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ __half narrow(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }

// The plain form: a warp a (query row, head), 32 positions at a time with a running maximum and sum.
template <class T, int D>
__global__ void __launch_bounds__(128) attend_kernel(PoolDev p, BookDev b, AttendArgs a, uint32_t* status) {
    __shared__ float qs[4][D];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int row = blockIdx.x, head = blockIdx.y * 4 + wid;
    if (head >= a.heads) return;
    if (row == 0 && head == 0) {
        bool bad = false;
        for (int i = lane; i < b.rows; i += 32) bad |= a.begin[i] < 0 || a.begin[i + 1] < a.begin[i] || a.begin[i + 1] > a.rows;
        if (bad) atomicOr(status, kStRange);
    }
    int s = 0;
    {
        int lo = 0, hi = b.rows;                  // the last session that begins at or before the row
        while (hi - lo > 1) { const int m = (lo + hi) / 2; if (a.begin[m] <= row) lo = m; else hi = m; }
        s = lo;
    }
    const int first = max(a.begin[s], 0), end = a.begin[s + 1];
    if (row < first || row >= end) return;
    const int most = most_positions(b, p);
    int len = b.len[s], n = min(end, a.rows) - first;
    if (len < 0 || len > most || n > most - len) {
        if (lane == 0) atomicOr(status, kStRange);
        len = min(max(len, 0), most);
        n = min(n, most - len);
    }
    const int i = row - first, kh = head / a.group;
    const T* q = static_cast<const T*>(a.q) + row * a.qs_row + head * a.qs_head;
    for (int c = lane; c < D; c += 32) qs[wid][c] = widen(q[c]);
    __syncwarp();
    const uint8_t* kb = p.base + a.layer * p.sl + kh * p.sh;
    float m = -INFINITY, sum = 0.f, o[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; ++c) o[c] = 0.f;
    for (int t0 = 0; t0 < len + n; t0 += 32) {
        const int t = t0 + lane, j = t - len;
        bool sees = t < len + n && (j < 0 || (a.mask ? j < a.mask_words * 32 && (a.mask[(int64_t)row * a.mask_words + j / 32] >> (j & 31) & 1) : j <= i));
        int64_t at = 0;
        if (sees) {
            const int page = b.table[(int64_t)s * b.max_pages + t / p.page_pos];
            at = (int64_t)page * p.spage + (int64_t)(t % p.page_pos) * p.sp;
            if (page < 0 || page >= p.n_pages) { atomicOr(status, kStRange); sees = false; at = 0; }
        }
        float x = -INFINITY;
        if (sees) {
            const T* k = reinterpret_cast<const T*>(kb + at);
            x = 0.f;
            for (int c = 0; c < D; c += 8) {
                const uint4 r = *reinterpret_cast<const uint4*>(k + c);
                const T* h = reinterpret_cast<const T*>(&r);
#pragma unroll
                for (int e = 0; e < 8; ++e) x = fmaf(qs[wid][c + e], widen(h[e]), x);
            }
            x *= a.scale;
        }
        float top = x;
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, w));
        top = fmaxf(top, m);
        if (top == -INFINITY) continue;
        const float w = sees ? __expf(x - top) : 0.f, old = __expf(m - top);
        m = top;
        sum = sum * old + warp_sum(w);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) o[c] *= old;
        const uint32_t who = __ballot_sync(kFull, sees);
        for (int e = 0; e < 32; ++e) {
            if (!(who >> e & 1)) continue;
            const int64_t from = __shfl_sync(kFull, at, e);
            const float we = __shfl_sync(kFull, w, e);
            const T* v = reinterpret_cast<const T*>(kb + p.skv + from);
#pragma unroll
            for (int c = 0; c < D / 32; ++c) o[c] = fmaf(we, widen(v[c * 32 + lane]), o[c]);
        }
    }
    T* out = static_cast<T*>(a.out) + row * a.os_row + head * a.os_head;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) out[c * 32 + lane] = narrow<T>(sum == 0.f ? 0.f : o[c] / sum);
    if (a.lse && lane == 0) a.lse[(int64_t)row * a.heads + head] = sum == 0.f ? -INFINITY : m + logf(sum);
}

template <class T>
cudaError_t launch_attend(const PoolDev& p, const BookDev& b, const AttendArgs& a, uint32_t* status, cudaStream_t st) {
    const dim3 grid(a.rows, (a.heads + 3) / 4);
    switch (p.d) {
        case 32: attend_kernel<T, 32><<<grid, 128, 0, st>>>(p, b, a, status); break;
        case 64: attend_kernel<T, 64><<<grid, 128, 0, st>>>(p, b, a, status); break;
        case 128: attend_kernel<T, 128><<<grid, 128, 0, st>>>(p, b, a, status); break;
        default: attend_kernel<T, 256><<<grid, 128, 0, st>>>(p, b, a, status); break;
    }
    return cudaGetLastError();
}

plc_status check_heads(const PoolDev& p, int32_t n_heads) {
    if (n_heads < 1) return PLC_E_INVALID;
    return n_heads % p.H || n_heads > (1 << 16) ? PLC_E_SHAPE : PLC_OK;
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" {

plc_status plc_tree_attention_workspace(const plc_page_pool* pool, int32_t n_heads, uint64_t* bytes) {
    PoolDev p;
    plc_status rc = check_pool(pool, &p);
    if (rc || (rc = check_heads(p, n_heads))) return rc;
    if (!bytes) return PLC_E_INVALID;
    *bytes = 16;
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
    if (!plc_aligned16(t->q_dev) || !plc_aligned16(t->out_dev) || !plc_aligned16(workspace_dev) || t->q_stride_row % 8 || t->q_stride_head % 8 ||
        t->out_stride_row % 8 || t->out_stride_head % 8)
        return PLC_E_ALIGN;
    uint64_t need = 0;
    plc_tree_attention_workspace(pool, t->n_heads, &need);
    if (workspace_bytes < need) return PLC_E_CAPACITY;
    if (t->n_rows == 0) return PLC_OK;
    const AttendArgs a{t->q_dev, t->q_stride_row, t->q_stride_head, t->out_dev, t->out_stride_row, t->out_stride_head, t->lse_dev, t->begin_dev,
                       t->mask_dev, t->n_rows, t->n_heads, t->n_heads / p.H, t->mask_dev ? t->mask_words : 0, layer, scale};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = pool->dtype == PLC_OUT_F16 ? launch_attend<__half>(p, b, a, status_dev, st) : launch_attend<__nv_bfloat16>(p, b, a, status_dev, st);
    if (e != cudaSuccess) return PLC_E_CUDA;
    count_launch();
    return PLC_OK;
}

}  // extern "C"
