// Attention of drafted tokens over their session's pages (plc_tree_attention): argument checks, and which kernel a call takes.
//
// For a session's KV head the rows are its drafted tokens times the query heads of the group.  Both kernels take K and V in tiles of positions:
// scores S, weights P = exp2(c S - m) with a running maximum m and sum l in binary32, O += P V; out = O / l at the end.  Where a session has few rows
// (plc_attend_few.cuh) HBM is the bound, where it has many (plc_attend_many.cuh) the products and exponentials.
//
// Work.  All (session, head, row tile, position tile) form one sequence, cut into equal ranges, one a CTA: lengths that differ, and one long context,
// fill the GPU alike.  A CTA's first and last piece may be parts of an item (session, head, row tile); those leave O, m and l in the
// workspace and a second, small launch joins them in a fixed order.
//
// The copies are boxes of a page (TMA) where pages are multiples of eight positions, else cp.async position by position, since a page may be any
// size and lie anywhere.
//
// The weights are rounded to the type of V because the product takes both operands in one type; l sums them unrounded.  For f16 they are formed as
// 2^12 times themselves, so that weights down to 2^-26 of the largest keep all their bits.  A row's maximum is raised only when it would grow by
// more than 2^3 (a weight is at most 2^15 then), which spares most passes over O.
#include "plc_attend.cuh"

namespace plc {
namespace {

AttendPlan plan_of(int row_tile, int per_sm, long long rows, int d) {
    AttendPlan x;
    x.row_tile = row_tile;
    x.grid = per_sm * sm_count();                 // at most: the kernel may take fewer
    x.part_rows = (int)(rows < row_tile ? rows : row_tile);
    x.bytes = (uint64_t)x.grid * 16 + 2ull * x.grid * x.part_rows * (8 + 4 * d);
    return x;
}
// Up to kFewRows rows a session and KV head (32 of 256 components) take the layout for few rows; beyond, two row tiles share K and V where a
// session has more rows than one holds.  By the mean, since a session's rows are known on the device only; where sessions are alike or have about the
// mean that is right, where they are not it costs: a chunk of 2048 among 255 single tokens (8 x 4 heads of 128, 512 positions) 626 us, in calls
// of their own 198 + 120; four trees of 26 rows among 60 sessions without any 91 us, by themselves 75.
constexpr int kFewRows = 64;
AttendPlan plan(const PoolDev& p, int heads, int sessions, int n_rows) {
    const long long rows = (long long)n_rows * (heads / p.H);
    const int few = p.d == 256 ? kFewRows / 2 : kFewRows;
    if (rows <= (long long)few * sessions) {
        const int tile = rows <= 16LL * sessions ? 16 : rows <= 32LL * sessions ? 32 : few;
        return plan_of(tile, tile <= 32 && p.d != 256 ? 2 : 1, rows, p.d);
    }
    const bool two = rows > 128LL * sessions && p.d != 256;
    return plan_of(two ? 256 : 128, two || p.d == 256 ? 1 : 2, rows, p.d);
}

// How many items a call has at most, if they are no more than SMs and short: then a CTA takes one whole, and there is no second launch to join them.  A tile
// after the other costs 1.6 us each, the second launch 2.4 us on the device and 2 us of the caller's time.  One token of 32 heads of 128, split and whole:
//   positions   calls in a row (the caller's time)   each waited for   in a graph
//      128            18.9   16.7                     32.3   31.0      10.8    9.5
//      256            19.0   16.7                     34.9   33.5      12.8   12.1
//      384            18.9   16.7                     34.7   36.1      12.8   14.4
// Beyond 256 the call costs its caller less and the device more; the border stands where a fourth tile begins.  It goes by what a row of the book can hold, which
// is what the host knows.
constexpr int kWholePositions = 384;
int whole_items(const PoolDev& p, const BookDev& b, long long rows, int n_rows, int row_tile) {
    const long long items = p.H * (rows / row_tile + (n_rows < b.rows ? n_rows : b.rows));
    return (long long)b.max_pages * p.page_pos <= kWholePositions && items <= sm_count() ? (int)items : 0;
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
                 t->mask_dev, t->n_rows, t->n_heads, group, t->mask_dev ? t->mask_words : 0, layer, scale, nullptr, nullptr, nullptr, x.part_rows, 0, 0, 0, {}, 0};
    a.first = static_cast<int4*>(workspace_dev);
    a.part_o = reinterpret_cast<float*>(a.first + x.grid);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + 2ll * x.grid * x.part_rows * p.d);
    a.whole = whole_items(p, b, (long long)t->n_rows * group, t->n_rows, x.row_tile);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool half = pool->dtype == PLC_OUT_F16;
    const cudaError_t e = x.row_tile <= kFewRows ? (half ? launch_attend_few_f16(p, b, a, x, status_dev, st) : launch_attend_few_bf16(p, b, a, x, status_dev, st))
                                                 : (half ? launch_attend_many_f16(p, b, a, x, status_dev, st) : launch_attend_many_bf16(p, b, a, x, status_dev, st));
    if (e != cudaSuccess) return PLC_E_CUDA;
    count_launch(a.whole ? 1 : 2);
    return PLC_OK;
}

}  // extern "C"
