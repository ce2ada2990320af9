// Log probabilities of given tokens, the entropy of their rows and the likeliest alternatives (plc_token_logprobs).
//
// With y = x - max x and Z = sum exp y:  log p_v = y_v - ln Z,  H = ln Z + (sum exp(y) (-y)) / Z.  One pass over the logits (the rows of beam selection, with the
// second sum beside the first) leaves maximum, sums and the n largest of each part of a row; a second, small launch joins the parts and
// looks the given tokens up, where not a block or a cluster has the whole row and does so itself.  HBM bound: each logit is read once.
// Measured on the device: 1024 rows of 128256 in bf16, 8 alternatives 61 us (263 MB, 4.3 TB/s; issue slots 0.63, the exponentials' unit 0.57 busy; of 65 us then
// without exponentials 57, without the maxima 60); 64 alternatives 85, 128 119; one row of 32000 8 us.
//
// Exponentials and the sums of 32 of them are binary32, what is added up beyond binary64.  The largest term of Z is exactly 1 and -y >= 0, so that neither a
// log probability near 0 nor a small entropy is the difference of larger numbers (terms below 2^-24 of their group are rounded to it).
#include "plc_logits.cuh"

namespace plc {
namespace {

constexpr int kMostTop = 128, kMostTokens = 1 << 20;
constexpr int kMostListed = 1024;                 // entries of a row's lists

struct LogprobArgs : RowArgs {
    const int32_t* tokens; int n_tokens, n_top, esz_log2, bf16;
    float* logp; float* entropy; float* top_logp; int32_t* top_token;
    uint32_t* status;
};

// ln of a row's sum of exponentials, not less than 1: e ln 2 in binary64 and, of what is left between 3/4 and 3/2, log1p in binary32, which is off by 2^-24 of at most 0.41 (and
// of the whole where the sum is near 1).  The sum of a row that is no distribution (NaN, or nothing but -inf) has none.
__device__ __forceinline__ double log_of(double sum) {
    if (!(sum > 0.0) || isinf(sum)) return (double)NAN;
    const long long bits = __double_as_longlong(sum);
    const int e = (int)((bits + (1ll << 51)) >> 52) - 1023;
    const double m = __longlong_as_double(bits - ((long long)e << 52));
    return (double)e * 0.693147180559945309 + (double)log1pf((float)(m - 1.0));
}

// A row's results from its parts: a block, of the same threads as a part.  LISTED: entries of its lists at most.
template <int LISTED>
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int row) {
    __shared__ unsigned long long keys[LISTED];
    __shared__ double log_sum;
    __shared__ float row_top;
    const int tid = threadIdx.x, lane = tid & 31;
    const long long slot = (long long)row * a.parts;
    const int entries = a.parts * a.k;
    auto logit_of = [&](int i, int* v) -> float { // of the i-th given token, and which it is
        *v = a.tokens[(long long)row * a.n_tokens + i];
        if (*v < 0 || *v >= a.V) return 0.f;
        const uint8_t* x = static_cast<const uint8_t*>(a.logits) + (((int64_t)row * a.row_stride + *v) << a.esz_log2);
        return a.esz_log2 == 2 ? *reinterpret_cast<const float*>(x)
               : a.bf16 ? widen(*reinterpret_cast<const __nv_bfloat16*>(x)) : widen(*reinterpret_cast<const __half*>(x));
    };
    // The first warp joins the sums; meanwhile the others have the lists and the first tokens' logits come.
    const int seat = (tid + kRowThreads - 32) % kRowThreads;
    int first_token = -1;
    float first_logit = 0.f;
    double spread = 0.0, sum = 0.0;
    if (tid < 32) {
        const int upto = min(a.parts, 32);        // at most 64 parts, two a lane
        float t[2];
        double s[2], w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int q = lane + 32 * e;
            const bool some = q < a.parts;
            t[e] = some ? __ldcg(a.top + slot + q) : -FLT_MAX;
            s[e] = some ? __ldcg(a.sum + slot + q) : 0.0;
            w[e] = some ? __ldcg(a.spread + slot + q) : 0.0;
        }
        float top = fmaxf(t[0], t[1]);
        for (int o = 1; o < upto; o <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (s[e] == 0.0) continue;
            const double f = (double)exp2_approx((t[e] - top) * kLog2e);
            sum += f * s[e];
            spread += f * (w[e] + s[e] * ((double)top - (double)t[e]));
        }
        for (int o = 1; o < upto; o <<= 1) {
            sum += __shfl_xor_sync(kFull, sum, o);
            spread += __shfl_xor_sync(kFull, spread, o);
        }
        if (lane == 0) {
            log_sum = log_of(sum);
            row_top = top;
        }
    } else {
        for (int i = tid - 32; i < entries; i += kRowThreads - 32) keys[i] = __ldcg(a.list + slot * a.k + i);
        if (seat < a.n_tokens) first_logit = logit_of(seat, &first_token);
    }
    __syncthreads();
    const double l = log_sum;
    const float top = row_top;
    if (tid == 0 && a.entropy) a.entropy[row] = (float)(l + spread / sum);
    for (int i = seat; i < a.n_tokens; i += kRowThreads) {
        int v = first_token;
        const float z = i == seat && tid >= 32 ? first_logit : logit_of(i, &v);
        const bool inside = v >= 0 && v < a.V;
        if (!inside && v != -1 && a.status) atomicOr(a.status, kStRange);
        a.logp[(long long)row * a.n_tokens + i] = inside ? (float)(((double)z - (double)top) - l) : 0.f;
    }
    // an entry's place is the number of better ones: those before it in its own list, and in each other list as many as a bisection finds
    for (int i = tid; i < entries; i += kRowThreads) {
        const unsigned long long key = keys[i];
        const int mine = i / a.k;
        int place = i - mine * a.k;
        for (int q = 0; q < a.parts && place < a.n_top; ++q) {
            if (q == mine) continue;
            int lo = 0, hi = a.k;                 // keys[lo - 1] > key >= keys[hi]
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (keys[q * a.k + mid] > key) lo = mid + 1;
                else hi = mid;
            }
            place += lo;
        }
        if (key != 0 && place < a.n_top) {
            const float z = value_of((uint32_t)(key >> 32));
            const double y = ((double)z - (double)top) - l;
            const bool some = isfinite(y);
            a.top_logp[(long long)row * a.n_top + place] = some ? (float)y : -INFINITY;
            a.top_token[(long long)row * a.n_top + place] = some ? (int)~(uint32_t)key : -1;
        }
    }
    for (int i = min(a.n_top, a.V) + tid; i < a.n_top; i += kRowThreads) {
        a.top_logp[(long long)row * a.n_top + i] = -INFINITY;
        a.top_token[(long long)row * a.n_top + i] = -1;
    }
}

// How the parts of a row come together: a block has a row; a cluster has it, whose first block finishes it behind the cluster's barrier; or a second launch does.
enum Way { kBlock, kCluster, kJoin };
template <class T, int WAY>
__global__ void __launch_bounds__(kRowThreads, kResident) logprob_rows_kernel(const __grid_constant__ LogprobArgs a) {
    if (WAY == kJoin) chain_next();
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    row_part<T, true>(a, row, part);
    if (WAY == kJoin) return;
    if (WAY == kBlock) __syncthreads();
    else {
        asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
        if (part > 0) return;
    }
    finish_row<WAY == kBlock ? kMostTop : kMostListed>(a, row);
}
__global__ void __launch_bounds__(kRowThreads) logprob_join_kernel(const __grid_constant__ LogprobArgs a) {
    chain_wait();
    finish_row<kMostListed>(a, blockIdx.x);
}

// Rows that are few enough for a cluster each take one launch; with vocabularies beyond kMostClustered
// more blocks a row are worth the second one.  Else as many parts as for beams: the least rounds of blocks times (a warp's logits plus what is done once).
constexpr int kSetUp = 1500, kMostClustered = 1 << 18;
struct RowPlan { Way way; int parts; };
RowPlan row_plan(long long rows, int V, int k) {
    const long long slots = (long long)kResident * sm_count();
    if (rows * 8 <= slots && V <= kMostClustered) {
        int parts = 1;
        while (parts < 8 && V > 4096 * parts) parts *= 2;
        return RowPlan{parts == 1 ? kBlock : kCluster, parts};
    }
    const long long most = (V + 4095) / 4096, fit = k ? kMostListed / k : 64;
    long long best = 1, least = 0;
    for (long long q = 1; q <= most && q <= fit && q <= 64; ++q) {
        const long long cost = (rows * q + slots - 1) / slots * ((V + q - 1) / q / kRowWarps + kSetUp);
        if (q == 1 || cost < least) { best = q; least = cost; }
    }
    return RowPlan{best == 1 ? kBlock : kJoin, (int)best};
}
uint64_t logprob_bytes(long long rows, int V, int n_top, RowPlan* plan, int* k) {
    *k = n_top < V ? n_top : V;
    *plan = row_plan(rows, V, *k);
    return (uint64_t)rows * plan->parts * (8ull * *k + 20);
}
plc_status check_rows(int32_t rows, int32_t vocab, int32_t n_tokens, int32_t n_top) {
    if (rows < 1 || vocab < 1 || n_tokens < 0 || n_top < 0) return PLC_E_INVALID;
    return rows > (1 << 24) || vocab > kMostVocab || n_tokens > kMostTokens || n_top > kMostTop ? PLC_E_SHAPE : PLC_OK;
}

}  // namespace
}  // namespace plc

using namespace plc;

extern "C" {

plc_status plc_token_logprobs_workspace(int32_t rows, int32_t vocab, int32_t n_top, uint64_t* bytes) {
    const plc_status rc = check_rows(rows, vocab, 0, n_top);
    if (rc) return rc;
    if (!bytes) return PLC_E_INVALID;
    RowPlan plan;
    int k;
    *bytes = logprob_bytes(rows, vocab, n_top, &plan, &k);
    return PLC_OK;
}

plc_status plc_token_logprobs(const void* logits_dev, int32_t dtype, int64_t row_stride, int32_t rows, int32_t vocab, const int32_t* tokens_dev, int32_t n_tokens,
                              int32_t n_top, float* logp_dev, float* entropy_dev, float* top_logp_dev, int32_t* top_token_dev, void* workspace_dev,
                              uint64_t workspace_bytes, uint32_t* status_dev, void* stream) {
    const plc_status rc = check_rows(rows, vocab, n_tokens, n_top);
    if (rc) return rc;
    if (!logits_dev || !workspace_dev || (n_tokens > 0 && (!tokens_dev || !logp_dev)) || (n_top > 0 && (!top_logp_dev || !top_token_dev))) return PLC_E_INVALID;
    if (dtype != PLC_OUT_F32 && dtype != PLC_OUT_F16 && dtype != PLC_OUT_BF16) return PLC_E_INVALID;
    const int esz = dtype == PLC_OUT_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(logits_dev) & (esz - 1)) || (reinterpret_cast<uintptr_t>(workspace_dev) & 15)) return PLC_E_ALIGN;
    LogprobArgs a{};
    RowPlan plan;
    const uint64_t need = logprob_bytes(rows, vocab, n_top, &plan, &a.k);
    a.parts = plan.parts;
    if (workspace_bytes < need) return PLC_E_CAPACITY;
    if ((long long)rows * a.parts > 0x7fffffffll) return PLC_E_SHAPE;
    a.logits = logits_dev; a.row_stride = row_stride; a.rows = rows; a.V = vocab;
    a.part_len = ((vocab + a.parts - 1) / a.parts + 7) & ~7;
    a.list = static_cast<unsigned long long*>(workspace_dev);
    a.sum = reinterpret_cast<double*>(a.list + (int64_t)rows * a.parts * a.k);
    a.spread = a.sum + (int64_t)rows * a.parts;
    a.top = reinterpret_cast<float*>(a.spread + (int64_t)rows * a.parts);
    a.tokens = tokens_dev; a.n_tokens = n_tokens; a.n_top = n_top; a.esz_log2 = esz == 4 ? 2 : 1; a.bf16 = dtype == PLC_OUT_BF16;
    a.logp = logp_dev; a.entropy = entropy_dev; a.top_logp = top_logp_dev; a.top_token = top_token_dev; a.status = status_dev;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto go = [&](auto* block, auto* cluster, auto* join) {
        return launch_kernel(plan.way == kBlock ? block : plan.way == kCluster ? cluster : join, (unsigned)(rows * a.parts), kRowThreads, 0, st, false,
                             plan.way == kCluster ? (unsigned)a.parts : 1u, a);
    };
#define PLC_ROWS(T) go(logprob_rows_kernel<T, kBlock>, logprob_rows_kernel<T, kCluster>, logprob_rows_kernel<T, kJoin>)
    if ((dtype == PLC_OUT_F32 ? PLC_ROWS(float) : dtype == PLC_OUT_F16 ? PLC_ROWS(__half) : PLC_ROWS(__nv_bfloat16)) != cudaSuccess) return PLC_E_CUDA;
#undef PLC_ROWS
    if (plan.way == kJoin && launch_kernel(logprob_join_kernel, (unsigned)rows, kRowThreads, 0, st, true, 1, a) != cudaSuccess) return PLC_E_CUDA;
    count_launch(plan.way == kJoin ? 2 : 1);
    return PLC_OK;
}

}  // extern "C"
