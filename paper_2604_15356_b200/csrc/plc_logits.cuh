// Rows of logits: one pass that forms a row's maximum, the sum of its exponentials and the sorted list of its largest logits (beam selection, log
// probabilities).
#pragma once
#include <cuda_bf16.h>
#include <float.h>

#include "plc_common.cuh"

namespace plc {
namespace {

constexpr int kRowThreads = 128, kRowWarps = kRowThreads / 32, kResident = 7;   // blocks an SM
constexpr int kChunks = 32;                       // pieces of a lane's logits whose maxima are kept
constexpr int kRoom = 1024;                       // candidates of a part that are ranked as they are
constexpr int kBuffer = 512;                      // and, where there are more (equal logits), at a time
constexpr int kMostVocab = 0x7fff0000;             // a column is an int, with up to 5000 more where a block's last step begins

struct RowArgs {
    const void* logits; int64_t row_stride;
    int rows, V, k, parts, part_len;              // k: entries of a list (0: none); part_len: a multiple of 8
    const uint8_t* done;                          // rows that are left out, or null
    unsigned long long* list;                     // [rows][parts][k] keys, best first
    double* sum;                                  // [rows][parts] sum of exp(x - maximum)
    double* spread;                               // [rows][parts] sum of exp(x - maximum) (maximum - x), where it is asked for
    float* top;                                   // [rows][parts] maximum
};

// A key orders by (value, lower column first): the value's order-preserving bits above the complement of the column.
__device__ __forceinline__ uint32_t order_bits(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);                       // -0 becomes +0, NaN of either sign the positive one, which stands above all: its row has its places filled
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

// groups: 64 bytes a lane.  last_bit: the bits of order_bits below it are alike in all values of the type of one sign.
template <class T> struct Step;
template <> struct Step<__nv_bfloat16> { static constexpr int groups = 4, last_bit = 16; };
template <> struct Step<__half> { static constexpr int groups = 4, last_bit = 13; };
template <> struct Step<float> { static constexpr int groups = 2, last_bit = 0; };

// A block takes a part of a row in two passes.  The first streams: a warp takes 32 lanes times kGroups times eight logits a step, the next step's loads on
// their way, forms the sum and keeps the maximum of each lane's chunks of steps.  The k-th largest of the lanes' maxima is a bound that k logits reach and
// few others do, so the second pass looks at the chunks that reach it alone: about k of them, from L2.
// SPREAD: also the sum that the entropy is made of.
template <class T, bool SPREAD>
__device__ __forceinline__ void row_part(const RowArgs& a, int row, int part) {
    constexpr int groups = Step<T>::groups, step = 256 * groups;
    __shared__ float tops[kChunks][kRowThreads];
    __shared__ unsigned long long found[kRoom];
    __shared__ float wtop[kRowWarps];
    __shared__ double wsum[kRowWarps], wspread[SPREAD ? kRowWarps : 1];
    __shared__ __align__(16) uint32_t order[kRowThreads];
    __shared__ float bound;
    __shared__ int reach[2][kRowWarps];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const T* x0 = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride;
    const bool vec = (reinterpret_cast<uintptr_t>(x0) & 15) == 0;
    const int c0 = part * a.part_len, c1 = min(a.V, c0 + a.part_len);
    const int steps = (c1 - c0 + kRowWarps * step - 1) / (kRowWarps * step), per_chunk = (steps + kChunks - 1) / kChunks;
    // the i-th step of this warp begins at column
    auto column = [&](int w, int i) { return c0 + (i * kRowWarps + w) * step; };
    float m = -FLT_MAX;                           // not -inf: exp(-inf - m) stays 0
    float top = -INFINITY, chunk_top = -INFINITY;
    double s = 0.0, spread = 0.0;                 // spread: in steps of a factor of two
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
        if (t > m) {
            const double f = (double)exp2_approx((m - t) * kLog2e);
            if (SPREAD && s != 0.0) spread = f * (spread + s * ((double)t - (double)m) * (double)kLog2e);
            s *= f;
            m = t;
        }
        float part_sum = 0.f;
        const unsigned long long neg = pack2(-m, -m), scale = pack2(kLog2e, kLog2e);
        if constexpr (SPREAD) {
            unsigned long long sums[2] = {0ull, 0ull}, far[2] = {0ull, 0ull};
#pragma unroll
            for (int g = 0; g < groups; ++g) {
                float x[8];
                now[g].widen(x);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float lo, hi;
                    unpack2(fma2(add2(pack2(x[2 * k], x[2 * k + 1]), neg), scale, 0ull), lo, hi);
                    const unsigned long long e = pack2(exp2_approx(lo), exp2_approx(hi));
                    // a logit of -inf has the exponential 0, and adds nothing, not 0 times infinity
                    const unsigned long long d = pack2(fmaxf(lo, -1e4f), fmaxf(hi, -1e4f));
                    sums[k & 1] = add2(sums[k & 1], e);
                    far[k & 1] = fma2(e, d, far[k & 1]);
                }
            }
            float lo, hi;
            unpack2(add2(sums[0], sums[1]), lo, hi);
            part_sum = lo + hi;
            unpack2(add2(far[0], far[1]), lo, hi);
            spread -= (double)(lo + hi);
        } else {
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
    const double down = (double)exp2_approx((m - warp_top) * kLog2e);
    if (SPREAD) spread = s != 0.0 ? down * (spread + s * ((double)warp_top - (double)m) * (double)kLog2e) : 0.0;
    s *= down;
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) {
        s += __shfl_xor_sync(kFull, s, w);
        if (SPREAD) spread += __shfl_xor_sync(kFull, spread, w);
    }
    if (lane == 0) {
        wtop[wid] = warp_top;
        wsum[wid] = s;
        if (SPREAD) wspread[wid] = spread;
    }
    __syncthreads();
    const long long slot = (long long)row * a.parts + part;
    if (wid == 0 && a.k > 0) {
        // The k-th largest of the lanes' maxima, by the upper half of their bits; what is just below it will do as a bound, as long as hardly any more maxima reach it than are asked
        // for.  Logits far from 0 lie closer together than half of their bits tell, and take the others that differ too, a microsecond a block (by all of them always: one row of 32000 in binary32 8.4 -> 9.2 us; 512 rows of 128256 in binary32 around
        // 1000, beams: 893 us by the upper half alone, 61 so).
        uint32_t v[kRowWarps], least = 0;
        int reaching = kRowThreads;               // maxima that are not below `least`
#pragma unroll
        for (int i = 0; i < kRowWarps; ++i) v[i] = order[i * 32 + lane];
#pragma unroll 1
        for (int bit = 31; bit >= Step<T>::last_bit && (bit >= 16 || reaching > a.k + 8); --bit) {
            const uint32_t t = least | (1u << bit);
            int c = 0;
#pragma unroll
            for (int i = 0; i < kRowWarps; ++i) c += v[i] >= t;
            c = __reduce_add_sync(kFull, c);
            if (c >= a.k) { least = t; reaching = c; }
        }
        if (lane == 0) bound = value_of(max(least, order_bits(-INFINITY)));
    } else if (wid == 1) {                        // a lane a warp's sums, added in the warps' order
        const int w = min(lane, kRowWarps - 1);
        float all = wtop[w];
#pragma unroll
        for (int o = kRowWarps / 2; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor_sync(kFull, all, o));
        const double f = (double)exp2_approx((wtop[w] - all) * kLog2e), s_here = wsum[w] * f;
        double far_here = 0.0, sum = 0.0, far = 0.0;
        if (SPREAD && wsum[w] != 0.0) far_here = f * (wspread[w] + wsum[w] * ((double)all - (double)wtop[w]) * (double)kLog2e);
#pragma unroll
        for (int v = 0; v < kRowWarps; ++v) {
            sum += __shfl_sync(kFull, s_here, v);
            if (SPREAD) far += __shfl_sync(kFull, far_here, v);
        }
        if (lane == 0) {
            a.sum[slot] = sum;
            if (SPREAD) a.spread[slot] = far * 0.693147180559945309;
            a.top[slot] = all;
        }
    }
    if (a.k == 0) return;
    __syncthreads();
    const uint32_t lt = lanemask_lt();
    // what lane l of warp w took in its i-th step, a logit a lane (0: none)
    auto look = [&](int w, int l, int i) -> unsigned long long {
        const int at = column(w, i) + (lane >> 3) * 256 + l * 8 + (lane & 7);
        return lane < 8 * groups && at < c1 ? ((unsigned long long)order_bits(widen(x0[at])) << 32) | (uint32_t)~at : 0ull;
    };
    if (a.k > kRowThreads / 2 && chunk > 1) {     // (with one chunk a lane it is the same bound)
        // With as many places as lanes the least of the lanes' maxima is the bound, and five times as many logits reach it as are wanted, now and then more than there is room
        // for (1024 rows of 128256, 128 of each: 555 us).  One that goes by the lanes' chunks is nearer to the k-th largest (119 us; for 64 of each it was 100 instead of 89, 85 by now).
        float* list = reinterpret_cast<float*>(found);
        const float limit = bound;
        for (int c = 0; c < chunk; ++c) {
            const bool take = tops[c][tid] >= limit;
            const uint32_t b = __ballot_sync(kFull, take);
            int at = 0;
            if (lane == 0 && b) at = atomicAdd(&count, __popc(b));
            at = __shfl_sync(kFull, at, 0) + __popc(b & lt);
            if (take && at < 2 * kRoom) list[at] = tops[c][tid];
        }
        __syncthreads();
        const int listed = count;
        __syncthreads();                          // all have read it: the branch, which has barriers, is taken by all or none, and the counter begins anew behind it
        if (listed <= 2 * kRoom) {
            uint32_t least = 0;
            for (int bit = 31; bit >= 0; --bit) {
                const uint32_t t = least | (1u << bit);
                int c = 0;
                for (int i = tid; i < listed; i += kRowThreads) c += order_bits(list[i]) >= t;
                c = __reduce_add_sync(kFull, c);
                if (lane == 0) reach[bit & 1][wid] = c;
                __syncthreads();
                if (reach[bit & 1][0] + reach[bit & 1][1] + reach[bit & 1][2] + reach[bit & 1][3] >= a.k) least = t;
            }
            if (tid == 0) bound = value_of(least);
        }
        if (tid == 0) count = 0;
        __syncthreads();
    }
    {
        const float limit = bound;
        const uint32_t least = order_bits(limit);
        for (int c = 0; c < chunk; ++c) {
            uint32_t who = __ballot_sync(kFull, tops[c][tid] >= limit);
            while (who) {                         // four lanes' chunks at a time, so that their loads are on their way together
                int l[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    l[k] = __ffs(who) - 1;
                    who &= who - 1;
                }
                for (int i = c * per_chunk; i < min(steps, (c + 1) * per_chunk); ++i) {
                    unsigned long long key[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) key[k] = l[k] >= 0 ? look(wid, l[k], i) : 0ull;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const bool take = (uint32_t)(key[k] >> 32) >= least && key[k] != 0;
                        const uint32_t b = __ballot_sync(kFull, take);
                        if (!b) continue;
                        int at = 0;
                        if (lane == 0) at = atomicAdd(&count, __popc(b));
                        at = __shfl_sync(kFull, at, 0) + __popc(b & lt);
                        if (take && at < kRoom) found[at] = key[k];
                    }
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

}  // namespace
}  // namespace plc
