// Beam search: selection over beams and vocabulary, and states that follow their beams.
//
// Of a session's beams*V continuations the n_out best are among each row's n_out best, and in a row the order is that of
// the logits.  So one pass over the logits gives, for each part of a row, the maximum, the sum of exp(x - maximum) and
// the n_out largest logits; a second, small launch joins the parts: the row's log-sum-exp, and a merge of the
// sorted lists by score.  HBM bound: each logit is read once.
//
// Exactness: continuations of different rows are compared by score + x - lse in binary64.  Exponentials are binary32 (x - maximum
// is subtracted before it is scaled, so that the largest terms, which carry the sum, have the smallest errors); groups of eight are added in
// binary32 and the groups in binary64, in an order that depends on the column alone and not on the row's alignment:
// equal rows have equal sums, so that their ties go to the lower row.
#include <cuda_bf16.h>
#include <float.h>

#include "plc_common.cuh"

namespace plc {
namespace {

constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;
constexpr int kMostOut = 128;                     // n_out, beams
constexpr int kBuffer = 512;                      // a warp's candidates: cut to n_out when a step of 256 more might not fit
constexpr int kMostListed = 16384;                // entries of a session's lists (the merge holds them in shared memory)

struct SelectArgs {
    const void* logits; int64_t row_stride;
    int rows, V, k, parts, part_len;              // k: entries of a list, min(n_out, V); part_len: a multiple of 8
    const float* score; const uint8_t* done; int beams, eos, n_out;
    unsigned long long* list;                     // [rows][parts][k] keys, best first
    double* sum;                                  // [rows][parts] sum of exp(x - maximum)
    float* top;                                   // [rows][parts] maximum
    float* out_score; int32_t* out_parent; int32_t* out_token;
};

// A key orders by (value, lower column first): the value's order-preserving bits above the complement of the column.
__device__ __forceinline__ uint32_t order_bits(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);                       // -0 becomes +0
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }

template <class T> struct Octet;                  // eight logits
template <> struct Octet<float> {
    static __device__ __forceinline__ void load(const float* p, bool vec, int n, float* x) {
        if (vec && n >= 8) {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < n ? p[i] : -INFINITY;
        }
    }
};
template <class H> __device__ __forceinline__ float widen(H v);
template <> __device__ __forceinline__ float widen(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class H> struct Octet {
    static __device__ __forceinline__ void load(const H* p, bool vec, int n, float* x) {
        if (vec && n >= 8) {
            const uint4 r = *reinterpret_cast<const uint4*>(p);
            const H* h = reinterpret_cast<const H*>(&r);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = widen(h[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < n ? widen(p[i]) : -INFINITY;
        }
    }
};

// Cuts a warp's buffer of n keys (n <= kBuffer) to its k largest, in no particular order; returns the k-th largest's value bits.
// Bisection over the value bits, then ties by column: few calls, so it is kept small.
__device__ __forceinline__ uint32_t cut(unsigned long long* buf, int n, int k, int lane) {
    unsigned long long key[kBuffer / 32];
#pragma unroll
    for (int i = 0; i < kBuffer / 32; ++i) key[i] = i * 32 + lane < n ? buf[i * 32 + lane] : 0ull;
    unsigned long long lo = 0;                    // the largest t with at least k keys >= t
    for (int bit = 63; bit >= 0; --bit) {
        const unsigned long long t = lo | (1ull << bit);
        int c = 0;
#pragma unroll
        for (int i = 0; i < kBuffer / 32; ++i) c += key[i] >= t;
        if (__reduce_add_sync(kFull, c) >= k) lo = t;
    }
    __syncwarp();
    int at = 0;
    const uint32_t lt = lanemask_lt();
#pragma unroll
    for (int i = 0; i < kBuffer / 32; ++i) {
        const bool take = key[i] >= lo && key[i] != 0;
        const uint32_t m = __ballot_sync(kFull, take);
        if (take) buf[at + __popc(m & lt)] = key[i];
        at += __popc(m);
    }
    __syncwarp();
    return (uint32_t)(lo >> 32);
}

template <class T>
__global__ void __launch_bounds__(kRowThreads) beam_rows_kernel(SelectArgs a) {
    __shared__ unsigned long long buf[kRowWarps][kBuffer];
    __shared__ int held[kRowWarps];
    __shared__ float wtop[kRowWarps];
    __shared__ double wsum[kRowWarps];
    chain_next();
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    if (a.done && a.done[row]) return;            // one continuation, at the beam's own score: the logits are not needed
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const T* x0 = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride;
    const bool vec = (reinterpret_cast<uintptr_t>(x0) & 15) == 0;
    const int c0 = part * a.part_len, c1 = min(a.V, c0 + a.part_len);
    float m = -FLT_MAX;                           // not -inf: exp(-inf - m) stays 0
    double s = 0.0;
    int n = 0;
    uint32_t least = 0;                           // value bits that a candidate has to reach
    unsigned long long* mine = buf[wid];
    const uint32_t lt = lanemask_lt();
    for (int base = c0 + wid * 256; base < c1; base += kRowThreads * 8) {
        const int c = base + lane * 8, left = c1 - c;
        float x[8];
        Octet<T>::load(x0 + c, vec, left, x);
        float t = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) t = fmaxf(t, x[i]);
        if (t > m) { s *= (double)__expf(m - t); m = t; }
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = exp2f((x[i] - m) * 1.44269504088896f);
        s += (double)(((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
        if (__any_sync(kFull, left > 0 && order_bits(t) >= least)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t o = order_bits(x[i]);
                const bool take = i < left && o >= least;
                const uint32_t b = __ballot_sync(kFull, take);
                if (take) mine[n + __popc(b & lt)] = ((unsigned long long)o << 32) | (uint32_t)~(c + i);
                n += __popc(b);
            }
            __syncwarp();
            if (n > kBuffer - 256) { least = cut(mine, n, a.k, lane); n = min(n, a.k); }
        }
    }
    if (n > a.k) { cut(mine, n, a.k, lane); n = a.k; }
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
    s *= (double)exp2f((m - top) * 1.44269504088896f);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    if (lane == 0) { held[wid] = n; wtop[wid] = top; wsum[wid] = s; }
    __syncthreads();
    const long long slot = (long long)row * a.parts + part;
    if (tid == 0) {
        float all = wtop[0];
        for (int w = 1; w < kRowWarps; ++w) all = fmaxf(all, wtop[w]);
        double sum = 0.0;
        for (int w = 0; w < kRowWarps; ++w) sum += wsum[w] * (double)exp2f((wtop[w] - all) * 1.44269504088896f);
        a.sum[slot] = sum;
        a.top[slot] = all;
    }
    // each key's place is the number of larger ones
    unsigned long long* out = a.list + slot * a.k;
    int total = 0;
    for (int w = 0; w < kRowWarps; ++w) total += held[w];
    for (int i = total + tid; i < a.k; i += kRowThreads) out[i] = 0ull;
    for (int i = lane; i < n; i += 32) {
        const unsigned long long key = mine[i];
        int place = 0;
        for (int w = 0; w < kRowWarps; ++w)
            for (int j = 0; j < held[w]; ++j) place += buf[w][j] > key;
        if (place < a.k) out[place] = key;
    }
}

// Better of two continuations: the larger score, then the lower place (row in the session, column).
struct Best { double score; unsigned long long place; int list; };
__device__ __forceinline__ bool better(double s, unsigned long long p, const Best& b) { return s > b.score || (s == b.score && p < b.place); }
__device__ __forceinline__ Best warp_best(Best b) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const double s = __shfl_xor_sync(kFull, b.score, o);
        const unsigned long long p = __shfl_xor_sync(kFull, b.place, o);
        const int l = __shfl_xor_sync(kFull, b.list, o);
        if (better(s, p, b)) { b.score = s; b.place = p; b.list = l; }
    }
    return b;
}

// A block a session: its lists are merged by taking the best head n_out times; the lists of a warp first, then the warps'.
constexpr int kMergeThreads = 256, kMergeWarps = kMergeThreads / 32;
__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(SelectArgs a) {
    extern __shared__ unsigned long long keys[];             // [beams][parts][k]
    __shared__ double offset[kMostOut];                      // score - lse
    __shared__ int done[kMostOut];
    __shared__ Best won[kMergeWarps][kMostOut];
    __shared__ int n_won[kMergeWarps];
    chain_wait();
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, lists = a.beams * a.parts;
    for (int w = tid; w < a.beams; w += kMergeThreads) {
        const long long row = (long long)b * a.beams + w;
        const double own = (double)a.score[row];
        done[w] = a.done && a.done[row];
        double o = own;
        if (!done[w]) {
            float top = -FLT_MAX;
            for (int p = 0; p < a.parts; ++p) top = fmaxf(top, a.top[row * a.parts + p]);
            double sum = 0.0;
            for (int p = 0; p < a.parts; ++p) sum += a.sum[row * a.parts + p] * (double)exp2f((a.top[row * a.parts + p] - top) * 1.44269504088896f);
            o = own - ((double)top + log(sum));
        }
        offset[w] = isfinite(own) && isfinite(o) ? o : -INFINITY;
    }
    const unsigned long long* from = a.list + (long long)b * lists * a.k;
    for (int i = tid; i < lists * a.k; i += kMergeThreads) keys[i] = from[i];
    __syncthreads();
    // a list's head as a continuation; `at` entries of it have been taken
    auto head = [&](int l, int at) -> Best {
        const int w = l / a.parts;
        const Best none{-INFINITY, ~0ull, -1};
        if (offset[w] == -INFINITY) return none;
        if (done[w]) return l % a.parts == 0 && at == 0 ? Best{offset[w], (unsigned long long)w * a.V + a.eos, l} : none;
        if (at >= a.k) return none;
        const unsigned long long key = keys[l * a.k + at];
        if (key == 0) return none;
        const double s = (double)value_of((uint32_t)(key >> 32)) + offset[w];
        return s > -INFINITY ? Best{s, (unsigned long long)w * a.V + (uint32_t)~(uint32_t)key, l} : none;
    };
    // a warp has the lists wid, wid + 8, ...; a lane every 32nd of those: at most beams*parts / 256, whose heads it keeps
    constexpr int kMine = 8;
    int at[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) at[i] = 0;
    int n = 0;
    for (; n < a.n_out; ++n) {
        Best m{-INFINITY, ~0ull, -1};
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int l = (i * 32 + lane) * kMergeWarps + wid;
            if (l < lists) { const Best h = head(l, at[i]); if (better(h.score, h.place, m)) m = h; }
        }
        m = warp_best(m);
        if (m.list < 0) break;
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if ((i * 32 + lane) * kMergeWarps + wid == m.list) ++at[i];
        if (lane == 0) won[wid][n] = m;
    }
    if (lane == 0) n_won[wid] = n;
    __syncthreads();
    if (wid) return;
    int pos = 0;
    for (n = 0; n < a.n_out; ++n) {
        Best m{-INFINITY, ~0ull, -1};
        if (lane < kMergeWarps && pos < n_won[lane]) { m = won[lane][pos]; m.list = lane; }
        m = warp_best(m);
        if (lane == m.list) ++pos;
        if (lane == 0) {
            const long long o = (long long)b * a.n_out + n;
            a.out_score[o] = (float)m.score;
            a.out_parent[o] = m.list < 0 ? -1 : (int)(b * a.beams + m.place / a.V);
            a.out_token[o] = m.list < 0 ? -1 : (int)(m.place % a.V);
        }
    }
}

// dst row r = src row parent[r], zeros without one.  A block takes pieces of one row of one set at a time.
constexpr int kMostSets = 16, kCopyThreads = 256, kPiece = 16384;
struct ReorderArgs {
    const uint8_t* src[kMostSets]; uint8_t* dst[kMostSets];
    int64_t ss[kMostSets], ds[kMostSets], bytes[kMostSets];
    long long ends[kMostSets];                    // pieces of the sets up to this one
    int sets, rows_in, rows_out;
};
template <class V>
__device__ __forceinline__ void copy_piece(const uint8_t* src, uint8_t* dst, int bytes) {
    const int n = bytes / (int)sizeof(V);
    V zero{};
    for (int i = threadIdx.x; i < n; i += 4 * kCopyThreads) {
        V x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k * kCopyThreads < n) x[k] = src ? reinterpret_cast<const V*>(src)[i + k * kCopyThreads] : zero;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k * kCopyThreads < n) reinterpret_cast<V*>(dst)[i + k * kCopyThreads] = x[k];
    }
}
__global__ void __launch_bounds__(kCopyThreads) beam_reorder_kernel(const __grid_constant__ ReorderArgs a, const int32_t* parent, uint32_t* status) {
    for (long long item = blockIdx.x; item < a.ends[a.sets - 1]; item += gridDim.x) {
        int t = 0;
        while (item >= a.ends[t]) ++t;
        const long long i = item - (t ? a.ends[t - 1] : 0), pieces = (a.bytes[t] + kPiece - 1) / kPiece;
        const int r = (int)(i / pieces);
        const long long at = (i - r * pieces) * kPiece;
        const int bytes = (int)min((long long)kPiece, a.bytes[t] - at);
        int from = parent[r];
        if (from < -1 || from >= a.rows_in) {
            if (status && threadIdx.x == 0) atomicOr(status, kStRange);
            from = -1;
        }
        const uint8_t* src = from < 0 ? nullptr : a.src[t] + from * a.ss[t] + at;
        uint8_t* dst = a.dst[t] + r * a.ds[t] + at;
        const uintptr_t bits = reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | (uintptr_t)bytes;
        if ((bits & 15) == 0) copy_piece<uint4>(src, dst, bytes);
        else if ((bits & 3) == 0) copy_piece<uint32_t>(src, dst, bytes);
        else copy_piece<uint8_t>(src, dst, bytes);
    }
}

// Parts of a row: enough for the GPU where rows are few, as long as a part has 4096 logits and the session's lists fit the merge.
int row_parts(long long rows, int beams, int V, int k) {
    const long long most = (V + 4095) / 4096, fill = (8LL * sm_count() + rows - 1) / rows, fit = kMostListed / ((long long)beams * k);
    const long long lists = 2048 / beams;         // a merging lane keeps at most 8 heads
    long long p = fill < most ? fill : most;
    p = p < fit ? p : fit;
    p = p < lists ? p : lists;
    return (int)(p < 1 ? 1 : p);
}
uint64_t beam_bytes(long long rows, int beams, int V, int n_out, int* parts, int* k) {
    *k = n_out < V ? n_out : V;
    *parts = row_parts(rows, beams, V, *k);
    return (uint64_t)rows * *parts * (8ull * *k + 12);
}
plc_status check_beams(int32_t sessions, int32_t beams, int32_t vocab, int32_t n_out) {
    if (sessions < 1 || beams < 1 || vocab < 1 || n_out < 1) return PLC_E_INVALID;
    if (beams > kMostOut || n_out > kMostOut || sessions > (1 << 20) || (long long)sessions * beams > (1 << 24)) return PLC_E_SHAPE;
    return PLC_OK;
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" {

plc_status plc_beam_workspace(int32_t sessions, int32_t beams, int32_t vocab, int32_t n_out, uint64_t* bytes) {
    const plc_status rc = check_beams(sessions, beams, vocab, n_out);
    if (rc) return rc;
    if (!bytes) return PLC_E_INVALID;
    int parts, k;
    *bytes = beam_bytes((long long)sessions * beams, beams, vocab, n_out, &parts, &k);
    return PLC_OK;
}

plc_status plc_beam_select(const void* logits_dev, int32_t dtype, int64_t row_stride, int32_t sessions, int32_t beams, int32_t vocab,
                           const float* score_dev, const uint8_t* done_dev, int32_t eos, int32_t n_out, float* out_score_dev,
                           int32_t* out_parent_dev, int32_t* out_token_dev, void* workspace_dev, uint64_t workspace_bytes, void* stream) {
    const plc_status rc = check_beams(sessions, beams, vocab, n_out);
    if (rc) return rc;
    if (!logits_dev || !score_dev || !out_score_dev || !out_parent_dev || !out_token_dev || !workspace_dev) return PLC_E_INVALID;
    if (dtype != PLC_OUT_F32 && dtype != PLC_OUT_F16 && dtype != PLC_OUT_BF16) return PLC_E_INVALID;
    if (done_dev && (eos < 0 || eos >= vocab)) return PLC_E_INVALID;
    const int esz = dtype == PLC_OUT_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(logits_dev) & (esz - 1)) || (reinterpret_cast<uintptr_t>(workspace_dev) & 15)) return PLC_E_ALIGN;
    SelectArgs a{};
    const long long rows = (long long)sessions * beams;
    const uint64_t need = beam_bytes(rows, beams, vocab, n_out, &a.parts, &a.k);
    if (workspace_bytes < need) return PLC_E_CAPACITY;
    a.logits = logits_dev; a.row_stride = row_stride; a.rows = (int)rows; a.V = vocab;
    a.part_len = ((vocab + a.parts - 1) / a.parts + 7) & ~7;
    a.score = score_dev; a.done = done_dev; a.beams = beams; a.eos = eos; a.n_out = n_out;
    a.list = static_cast<unsigned long long*>(workspace_dev);
    a.sum = reinterpret_cast<double*>(a.list + rows * a.parts * a.k);
    a.top = reinterpret_cast<float*>(a.sum + rows * a.parts);
    a.out_score = out_score_dev; a.out_parent = out_parent_dev; a.out_token = out_token_dev;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto kern = dtype == PLC_OUT_F32 ? beam_rows_kernel<float> : dtype == PLC_OUT_F16 ? beam_rows_kernel<__half> : beam_rows_kernel<__nv_bfloat16>;
    if (launch_kernel(kern, (unsigned)(rows * a.parts), kRowThreads, 0, st, false, 1, a) != cudaSuccess) return PLC_E_CUDA;
    const size_t smem = (size_t)beams * a.parts * a.k * 8;
    if (cudaFuncSetAttribute(beam_merge_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostListed * 8) != cudaSuccess) return PLC_E_CUDA;
    if (launch_kernel(beam_merge_kernel, (unsigned)sessions, kMergeThreads, smem, st, true, 1, a) != cudaSuccess) return PLC_E_CUDA;
    count_launch(2);
    return PLC_OK;
}

plc_status plc_beam_reorder(const plc_row_set* sets, int32_t n_sets, const int32_t* parent_dev, int32_t rows_in, int32_t rows_out,
                            uint32_t* status_dev, void* stream) {
    if (!sets || !parent_dev || n_sets < 1 || rows_in < 1 || rows_out < 1) return PLC_E_INVALID;
    if (n_sets > kMostSets) return PLC_E_SHAPE;
    ReorderArgs a{};
    long long pieces = 0;
    for (int i = 0; i < n_sets; ++i)
        if (!sets[i].src_dev || !sets[i].dst_dev || sets[i].row_bytes < 1 || sets[i].src_stride < 0 || sets[i].dst_stride < 0) return PLC_E_INVALID;
    for (int i = 0; i < n_sets; ++i) {
        if (rows_out > 1 && sets[i].dst_stride < sets[i].row_bytes) return PLC_E_INVALID;
        const uintptr_t d0 = reinterpret_cast<uintptr_t>(sets[i].dst_dev), d1 = d0 + (rows_out - 1) * sets[i].dst_stride + sets[i].row_bytes;
        for (int j = 0; j < n_sets; ++j) {
            const uintptr_t s0 = reinterpret_cast<uintptr_t>(sets[j].src_dev), s1 = s0 + (rows_in - 1) * sets[j].src_stride + sets[j].row_bytes;
            if (d0 < s1 && s0 < d1) return PLC_E_INVALID;
        }
        a.src[i] = static_cast<const uint8_t*>(sets[i].src_dev);
        a.dst[i] = static_cast<uint8_t*>(sets[i].dst_dev);
        a.ss[i] = sets[i].src_stride;
        a.ds[i] = sets[i].dst_stride;
        a.bytes[i] = sets[i].row_bytes;
        pieces += (sets[i].row_bytes + kPiece - 1) / kPiece * rows_out;
        a.ends[i] = pieces;
    }
    a.sets = n_sets; a.rows_in = rows_in; a.rows_out = rows_out;
    const long long most = 8LL * sm_count();
    if (launch_kernel(beam_reorder_kernel, (unsigned)(pieces < most ? pieces : most), kCopyThreads, 0, static_cast<cudaStream_t>(stream), false, 1, a,
                      parent_dev, status_dev) != cudaSuccess)
        return PLC_E_CUDA;
    count_launch(1);
    return PLC_OK;
}

}  // extern "C"
