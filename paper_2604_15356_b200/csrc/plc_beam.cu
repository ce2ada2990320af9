// Beam search: selection over beams and vocabulary, and states that follow their beams.
//
// Of a session's beams*V continuations the n_out best are among each row's n_out best, and in a row the order is that of
// the logits.  So one pass over the logits gives, for each part of a row, the maximum, the sum of exp(x - maximum) and
// the n_out largest logits; a second, small launch joins the parts: the row's log-sum-exp, and a merge of the
// sorted lists by score.  HBM bound: each logit is read once.
// Measured: 512 rows of 128256 logits in bf16, 8 beams a session and 8 of their continuations: rows 38 us (131 MB, 3.4 TB/s; the exponentials' unit 0.49 busy,
// 21 warps an SM), merge 8 us, the states' rows 10 us; 49 us together.  With a list a warp that every logit was held against: 229 us.  Where fewer lanes than
// n_out hold a logit above the lowest of the row (ten tokens of 128256 that are not masked) the bound is that lowest one, all logits reach it, and one warp looks
// through them: 865 us instead of 48.
//
// Exactness: continuations of different rows are compared by (x - maximum) + (score - log sum) in binary64, the maximum taken off first: at the
// type's lowest values (a row that is masked with them as a whole) nothing else would be left of the sum.  Exponentials are binary32 (x - maximum
// is subtracted before it is scaled, so that the largest terms, which carry the sum, have the smallest errors); 32 of them are added in
// binary32 and the groups in binary64, in an order that depends on the column alone and not on the row's alignment:
// equal rows have equal sums, so that their ties go to the lower row.
#include <cuda_bf16.h>
#include <float.h>

#include "plc_common.cuh"

namespace plc {
namespace {

constexpr int kRowThreads = 128, kRowWarps = kRowThreads / 32, kResident = 7;   // blocks an SM
constexpr int kMostOut = 128;                     // n_out, beams
constexpr int kChunks = 32;                       // pieces of a lane's logits whose maxima are kept
constexpr int kRoom = 1024;                       // candidates of a part that are ranked as they are
constexpr int kBuffer = 512;                      // and, where there are more (equal logits), at a time
constexpr int kMostVocab = 0x7fff0000;             // a column is an int, with up to 5000 more where a block's last step begins
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

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.44269504088896f;

// Eight logits as they stand in memory; -inf behind the n-th.
template <class T> struct Octet;
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> struct Octet<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const float* p, bool vec, int n) {
        if (n >= 8) {
            if (vec) { a = reinterpret_cast<const uint4*>(p)[0]; b = reinterpret_cast<const uint4*>(p)[1]; return; }
            const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
            a = make_uint4(q[0], q[1], q[2], q[3]);
            b = make_uint4(q[4], q[5], q[6], q[7]);
            return;
        }
        uint32_t* w = reinterpret_cast<uint32_t*>(this);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = i < n ? __float_as_uint(p[i]) : 0xff800000u;
    }
    __device__ __forceinline__ float top() const {
        float x[8];
        widen(x);
        return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    }
    __device__ __forceinline__ void widen(float* x) const {
        x[0] = __uint_as_float(a.x); x[1] = __uint_as_float(a.y); x[2] = __uint_as_float(a.z); x[3] = __uint_as_float(a.w);
        x[4] = __uint_as_float(b.x); x[5] = __uint_as_float(b.y); x[6] = __uint_as_float(b.z); x[7] = __uint_as_float(b.w);
    }
};
template <class H> struct Half8 {
    uint4 a;
    __device__ __forceinline__ void load(const H* p, bool vec, int n, uint32_t none) {
        if (n >= 8) {
            if (vec) { a = *reinterpret_cast<const uint4*>(p); return; }
            // rows that start off 16-byte boundaries: the aligned words that hold the eight, put together
            const bool odd = reinterpret_cast<uintptr_t>(p) & 2;
            const uint32_t* q = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)3);
            uint32_t w[5];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = q[i];
            w[4] = odd ? q[4] : 0u;
            a = odd ? make_uint4(__funnelshift_r(w[0], w[1], 16), __funnelshift_r(w[1], w[2], 16), __funnelshift_r(w[2], w[3], 16), __funnelshift_r(w[3], w[4], 16))
                    : make_uint4(w[0], w[1], w[2], w[3]);
            return;
        }
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = i < n ? q[i] : none;
        a = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
};
template <> struct Octet<__half> : Half8<__half> {
    __device__ __forceinline__ void load(const __half* p, bool vec, int n) { Half8<__half>::load(p, vec, n, 0xfc00u); }
    __device__ __forceinline__ float top() const {
        const __half2* h = reinterpret_cast<const __half2*>(&a);
        const float2 f = __half22float2(__hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
        return fmaxf(f.x, f.y);
    }
    __device__ __forceinline__ void widen(float* x) const {
        const __half2* h = reinterpret_cast<const __half2*>(&a);
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(h[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
    }
};
template <> struct Octet<__nv_bfloat16> : Half8<__nv_bfloat16> {
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool vec, int n) { Half8<__nv_bfloat16>::load(p, vec, n, 0xff80u); }
    __device__ __forceinline__ float top() const {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&a);
        const float2 f = __bfloat1622float2(__hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
        return fmaxf(f.x, f.y);
    }
    __device__ __forceinline__ void widen(float* x) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
};

// The largest t such that at least k of the warp's values (keys of which `n` lanes' slots hold one each, invalid ones 0) are >= t.
template <int M> __device__ __forceinline__ uint32_t kth_largest(const uint32_t* v, int k) {
    uint32_t lo = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t t = lo | (1u << bit);
        int c = 0;
#pragma unroll
        for (int i = 0; i < M; ++i) c += v[i] >= t;
        if (__reduce_add_sync(kFull, c) >= k) lo = t;
    }
    return lo;
}

// Cuts a warp's buffer of n > k keys to its k largest, in no particular order; returns the smallest of their value bits.  Bisection over the
// values, then over the columns of those that equal the last one.
__device__ __noinline__ uint32_t cut(unsigned long long* buf, int n, int k, int lane) {
    constexpr int M = kBuffer / 32;
    unsigned long long key[M];
    uint32_t v[M];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < M; ++i) {
        key[i] = i * 32 + lane < n ? buf[i * 32 + lane] : 0ull;
        v[i] = (uint32_t)(key[i] >> 32);
    }
    const uint32_t least = kth_largest<M>(v, k);
    int above = 0, equal = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) { above += v[i] > least; equal += key[i] != 0 && v[i] == least; }
    above = __reduce_add_sync(kFull, above);
    equal = __reduce_add_sync(kFull, equal);
    uint32_t column = 0;                          // lowest complement of a column that is taken at the border
    if (above + equal > k) {
#pragma unroll
        for (int i = 0; i < M; ++i) v[i] = key[i] != 0 && v[i] == least ? (uint32_t)key[i] : 0u;
        column = kth_largest<M>(v, k - above);
    }
    __syncwarp();
    int at = 0;
    const uint32_t lt = lanemask_lt();
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const uint32_t hi = (uint32_t)(key[i] >> 32);
        const bool take = key[i] != 0 && (hi > least || (hi == least && (uint32_t)key[i] >= column));
        const uint32_t m = __ballot_sync(kFull, take);
        if (take) buf[at + __popc(m & lt)] = key[i];
        at += __popc(m);
    }
    __syncwarp();
    return least;
}

// A block takes a part of a row in two passes.  The first streams: a warp takes 32 lanes times kGroups times eight logits a step, the next step's loads on
// their way, forms the sum and keeps the maximum of each lane's chunks of steps.  The k-th largest of the lanes' maxima is a bound that k logits reach and
// few others do, so the second pass looks at the chunks that reach it alone: about k of them, from L2.
template <class T> struct Step { static constexpr int groups = 4; };                  // 64 bytes a lane
template <> struct Step<float> { static constexpr int groups = 2; };
template <class T>
__global__ void __launch_bounds__(kRowThreads, kResident) beam_rows_kernel(SelectArgs a) {
    constexpr int groups = Step<T>::groups, step = 256 * groups;
    __shared__ float tops[kChunks][kRowThreads];
    __shared__ unsigned long long found[kRoom];
    __shared__ float wtop[kRowWarps];
    __shared__ double wsum[kRowWarps];
    __shared__ __align__(16) uint32_t order[kRowThreads];
    __shared__ float bound;
    __shared__ int count;
    chain_next();
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    if (a.done && a.done[row]) return;            // one continuation, at the beam's own score: the logits are not needed
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const T* x0 = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride;
    const bool vec = (reinterpret_cast<uintptr_t>(x0) & 15) == 0;
    const int c0 = part * a.part_len, c1 = min(a.V, c0 + a.part_len);
    const int steps = (c1 - c0 + kRowWarps * step - 1) / (kRowWarps * step), per_chunk = (steps + kChunks - 1) / kChunks;
    // the i-th step of this warp begins at column
    auto column = [&](int w, int i) { return c0 + (i * kRowWarps + w) * step; };
    float m = -FLT_MAX;                           // not -inf: exp(-inf - m) stays 0
    float top = -INFINITY, chunk_top = -INFINITY;
    double s = 0.0;
    Octet<T> o[groups];
    auto fetch = [&](int base) {
        const T* x = x0 + base + lane * 8;
        if (vec && base + step <= c1) {
#pragma unroll
            for (int g = 0; g < groups; ++g) o[g].load(x + g * 256, true, 8);
        } else {
#pragma unroll
            for (int g = 0; g < groups; ++g) o[g].load(x + g * 256, vec, c1 - (base + g * 256 + lane * 8));
        }
    };
    fetch(column(wid, 0));
    int left = per_chunk, chunk = 0;
    for (int i = 0; i < steps; ++i) {
        Octet<T> now[groups];
#pragma unroll
        for (int g = 0; g < groups; ++g) now[g] = o[g];
        if (i + 1 < steps) fetch(column(wid, i + 1));
        float t = now[0].top();
#pragma unroll
        for (int g = 1; g < groups; ++g) t = fmaxf(t, now[g].top());
        chunk_top = fmaxf(chunk_top, t);
        if (t > m) { s *= (double)exp2_approx((m - t) * kLog2e); m = t; }
        float part_sum = 0.f;
        const unsigned long long neg = pack2(-m, -m), scale = pack2(kLog2e, kLog2e);
#pragma unroll
        for (int g = 0; g < groups; ++g) {
            float x[8];
            now[g].widen(x);
            unsigned long long e[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float lo, hi;
                unpack2(fma2(add2(pack2(x[2 * k], x[2 * k + 1]), neg), scale, 0ull), lo, hi);
                e[k] = pack2(exp2_approx(lo), exp2_approx(hi));
            }
            float lo, hi;
            unpack2(add2(add2(e[0], e[1]), add2(e[2], e[3])), lo, hi);
            part_sum += lo + hi;
        }
        s += (double)part_sum;
        if (--left == 0 || i + 1 == steps) {
            tops[chunk++][tid] = chunk_top;
            top = fmaxf(top, chunk_top);
            chunk_top = -INFINITY;
            left = per_chunk;
        }
    }
    order[tid] = order_bits(top);
    if (tid == 0) count = 0;
    float warp_top = m;
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) warp_top = fmaxf(warp_top, __shfl_xor_sync(kFull, warp_top, w));
    s *= (double)exp2_approx((m - warp_top) * kLog2e);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(kFull, s, w);
    if (lane == 0) { wtop[wid] = warp_top; wsum[wid] = s; }
    __syncthreads();
    const long long slot = (long long)row * a.parts + part;
    {
        int rank = 0;                             // of the lane's maximum among all
        const uint32_t mine = order[tid];
#pragma unroll 4
        for (int i = 0; i < kRowThreads; i += 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(order + i);
            rank += (v.x > mine || (v.x == mine && i < tid)) + (v.y > mine || (v.y == mine && i + 1 < tid)) + (v.z > mine || (v.z == mine && i + 2 < tid)) +
                    (v.w > mine || (v.w == mine && i + 3 < tid));
        }
        if (rank == a.k - 1) bound = top;
        if (tid == 0) {
            float all = wtop[0];
            for (int w = 1; w < kRowWarps; ++w) all = fmaxf(all, wtop[w]);
            double sum = 0.0;
            for (int w = 0; w < kRowWarps; ++w) sum += wsum[w] * (double)exp2_approx((wtop[w] - all) * kLog2e);
            a.sum[slot] = sum;
            a.top[slot] = all;
        }
    }
    __syncthreads();
    const uint32_t lt = lanemask_lt();
    // what lane l of warp w took in its i-th step, a logit a lane (0: none)
    auto look = [&](int w, int l, int i) -> unsigned long long {
        const int at = column(w, i) + (lane >> 3) * 256 + l * 8 + (lane & 7);
        return lane < 8 * groups && at < c1 ? ((unsigned long long)order_bits(widen(x0[at])) << 32) | (uint32_t)~at : 0ull;
    };
    {
        const float limit = bound;
        const uint32_t least = order_bits(limit);
        for (int c = 0; c < chunk; ++c) {
            uint32_t who = __ballot_sync(kFull, tops[c][tid] >= limit);
            while (who) {
                const int l = __ffs(who) - 1;
                who &= who - 1;
                for (int i = c * per_chunk; i < min(steps, (c + 1) * per_chunk); ++i) {
                    const unsigned long long key = look(wid, l, i);
                    const bool take = (uint32_t)(key >> 32) >= least && key != 0;
                    const uint32_t b = __ballot_sync(kFull, take);
                    if (!b) continue;
                    int at = 0;
                    if (lane == 0) at = atomicAdd(&count, __popc(b));
                    at = __shfl_sync(kFull, at, 0) + __popc(b & lt);
                    if (take && at < kRoom) found[at] = key;
                }
            }
        }
    }
    __syncthreads();
    int n = count;
    if (n > kRoom) {                              // many equal logits: one warp looks through them, in no more than kBuffer places
        __syncthreads();
        if (wid == 0) {
            n = 0;
            unsigned long long worst = 0ull;      // what a candidate has to pass, once k have been found
            for (int w = 0; w < kRowWarps; ++w)
                for (int c = 0; c < chunk; ++c) {
                    uint32_t who = __ballot_sync(kFull, order_bits(tops[c][w * 32 + lane]) >= max((uint32_t)(worst >> 32), order_bits(bound)));
                    while (who) {
                        const int l = __ffs(who) - 1;
                        who &= who - 1;
                        for (int i = c * per_chunk; i < min(steps, (c + 1) * per_chunk); ++i) {
                            const unsigned long long key = look(w, l, i);
                            const bool take = key > worst;
                            const uint32_t b = __ballot_sync(kFull, take);
                            if (take) found[n + __popc(b & lt)] = key;
                            n += __popc(b);
                            if (n <= kBuffer - 32) continue;
                            cut(found, n, a.k, lane);
                            n = a.k;
                            worst = ~0ull;
                            for (int k = lane; k < n; k += 32) worst = min(worst, found[k]);
#pragma unroll
                            for (int k = 16; k > 0; k >>= 1) worst = min(worst, __shfl_xor_sync(kFull, worst, k));
                        }
                    }
                }
            __syncwarp();
            if (lane == 0) count = n;
        }
        __syncthreads();
        n = count;
    }
    // each candidate's place is the number of better ones
    unsigned long long* out = a.list + slot * a.k;
    for (int i = n + tid; i < a.k; i += kRowThreads) out[i] = 0ull;
    for (int i = tid; i < n; i += kRowThreads) {
        const unsigned long long key = found[i];
        int place = 0;
        for (int j = 0; j < n; ++j) place += found[j] > key;
        if (place < a.k) out[place] = key;
    }
}

// A continuation: its score's order-preserving bits (0: none), and its place (row in the session, column) as one number.
struct Cont { unsigned long long score; uint32_t place; };
__device__ __forceinline__ bool better(const Cont& a, const Cont& b) { return a.score > b.score || (a.score == b.score && a.place < b.place); }
__device__ __forceinline__ Cont shuffle(const Cont& c, int lane) { return Cont{__shfl_sync(kFull, c.score, lane), __shfl_sync(kFull, c.place, lane)}; }
__device__ __forceinline__ Cont exchange(const Cont& x, int lane, int stride, bool larger) {
    const Cont y = shuffle(x, lane ^ stride);
    return better(y, x) == larger ? y : x;
}
__device__ __forceinline__ Cont sort32(Cont x, int lane) {
#pragma unroll 1
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll 1
        for (int stride = size >> 1; stride > 0; stride >>= 1) x = exchange(x, lane, stride, ((lane & stride) == 0) == ((lane & size) == 0 || size == 32));
    return x;
}
__device__ __forceinline__ Cont merge32(Cont x, const Cont& y, int lane) {
    const Cont r = shuffle(y, 31 - lane);
    if (better(r, x)) x = r;
#pragma unroll 1
    for (int stride = 16; stride > 0; stride >>= 1) x = exchange(x, lane, stride, (lane & stride) == 0);
    return x;
}
__device__ __forceinline__ unsigned long long order_bits(double x) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(x);
    return b ^ ((unsigned long long)((long long)b >> 63) | (1ull << 63));
}
__device__ __forceinline__ double double_of(unsigned long long o) {
    return __longlong_as_double((long long)(o >> 63 ? o ^ (1ull << 63) : ~o));
}

// A block a session: the 32 best of its lists' entries, then the 32 behind those, and so on.  The lists' first entries come first, so that
// soon only few of the others pass the 32nd best so far; 32 at a time are sorted and merged into the warp's 32, and the warps' in the end.
constexpr int kMergeThreads = 256, kMergeWarps = kMergeThreads / 32;
__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(SelectArgs a) {
    extern __shared__ unsigned long long keys[];             // [beams][parts][k]
    __shared__ double offset[kMostOut];                      // score - log of the sum of exp(x - top); -inf: no continuation
    __shared__ float row_top[kMostOut];                      // the row's largest logit
    __shared__ Cont best[kMergeWarps][32];
    __shared__ Cont border;
    chain_wait();
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, lists = a.beams * a.parts, entries = lists * a.k;
    const unsigned long long* from = a.list + (long long)b * entries;
    for (int i = tid; i < entries; i += kMergeThreads) keys[i] = from[i];
    for (int w = tid; w < a.beams; w += kMergeThreads) {
        const long long row = (long long)b * a.beams + w;
        const double own = (double)a.score[row];
        double o = own;
        float top = -FLT_MAX;
        if (a.done && a.done[row]) {                         // its one continuation stands first in its first list
            o = 0.0;
            if (!isfinite(own)) o = -INFINITY;
        } else {
            for (int p = 0; p < a.parts; ++p) top = fmaxf(top, a.top[row * a.parts + p]);
            double sum = 0.0;
            for (int p = 0; p < a.parts; ++p) sum += a.sum[row * a.parts + p] * (double)exp2_approx((a.top[row * a.parts + p] - top) * kLog2e);
            o = own - log(sum);
        }
        row_top[w] = top;
        offset[w] = isfinite(own) && isfinite(o) ? o : -INFINITY;
    }
    __syncthreads();
    for (int done = 0; done < a.n_out; done += 32) {
        const int want = min(32, a.n_out - done);
        Cont mine{0ull, ~0u};
        const Cont above = done ? border : Cont{~0ull, 0u};  // the last one taken
        int l = tid % lists, j = tid / lists;
        const int dl = kMergeThreads % lists, dj = kMergeThreads / lists;
        for (int i0 = wid * 32; i0 < entries; i0 += kMergeThreads) {
            Cont c{0ull, ~0u};
            if (i0 + lane < entries) {
                const int w = l / a.parts;
                const double o = offset[w];
                if (a.done && a.done[(long long)b * a.beams + w]) {
                    if (l % a.parts == 0 && j == 0 && o > -INFINITY)
                        c = Cont{order_bits((double)a.score[(long long)b * a.beams + w]), (uint32_t)w * (uint32_t)a.V + (uint32_t)a.eos};
                } else {
                    const unsigned long long key = keys[l * a.k + j];
                    const double s = ((double)value_of((uint32_t)(key >> 32)) - (double)row_top[w]) + o;
                    if (key != 0 && s > -INFINITY) c = Cont{order_bits(s), (uint32_t)w * (uint32_t)a.V + ~(uint32_t)key};
                }
            }
            l += dl;
            j += dj;
            if (l >= lists) { l -= lists; ++j; }
            const Cont last = shuffle(mine, want - 1);
            const bool take = c.score != 0 && better(c, last) && better(above, c);
            if (!__any_sync(kFull, take)) continue;
            if (!take) c = Cont{0ull, ~0u};
            mine = merge32(mine, sort32(c, lane), lane);
        }
        best[wid][lane] = mine;
        __syncthreads();
        if (wid == 0) {
            for (int w = 1; w < kMergeWarps && w * 32 < entries; ++w) mine = merge32(mine, best[w][lane], lane);
            if (lane == 31) border = mine;
            if (lane < want) {
                const long long o = (long long)b * a.n_out + done + lane;
                const bool some = mine.score != 0;
                a.out_score[o] = some ? (float)double_of(mine.score) : -INFINITY;
                a.out_parent[o] = some ? (int)(b * a.beams + mine.place / (uint32_t)a.V) : -1;
                a.out_token[o] = some ? (int)(mine.place % (uint32_t)a.V) : -1;
            }
        }
        __syncthreads();
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

// Parts of a row: of those that leave a part 4096 logits and fit the merge, the one with the least rounds of blocks times (a warp's logits plus kSetUp, what
// its first candidates and the joining of the warps cost, in logits).
constexpr int kSetUp = 1500;
int row_parts(long long rows, int beams, int V, int k) {
    const long long most = (V + 4095) / 4096, fit = kMostListed / ((long long)beams * k), slots = (long long)kResident * sm_count();
    long long best = 1, least = 0;
    for (long long p = 1; p <= most && p <= fit && p <= 64; ++p) {
        const long long cost = (rows * p + slots - 1) / slots * ((V + p - 1) / p / kRowWarps + kSetUp);
        if (p == 1 || cost < least) { best = p; least = cost; }
    }
    return (int)best;
}
uint64_t beam_bytes(long long rows, int beams, int V, int n_out, int* parts, int* k) {
    *k = n_out < V ? n_out : V;
    *parts = row_parts(rows, beams, V, *k);
    return (uint64_t)rows * *parts * (8ull * *k + 12);
}
plc_status check_beams(int32_t sessions, int32_t beams, int32_t vocab, int32_t n_out) {
    if (sessions < 1 || beams < 1 || vocab < 1 || n_out < 1) return PLC_E_INVALID;
    if (beams > kMostOut || n_out > kMostOut || vocab > kMostVocab || sessions > (1 << 20) || (long long)sessions * beams > (1 << 24) || (long long)beams * vocab >= (1ll << 32))
        return PLC_E_SHAPE;
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
