// Attention weights of positions: what the two kernels share.
#pragma once
#include "plc_pages.cuh"

namespace plc {

struct WeighArgs {
    const uint16_t* q; int64_t qs_row, qs_head;   // elements
    const float* lse; const int32_t* rows; const int32_t* begin;
    int n_list, n_rows, heads, group, layer;
    float* weight; int64_t ws_row, ws_head; int n_pos;
    float decay, scale;
    int4* first;                                  // [grid]: session, head, position tile of a CTA's range (-1: none), row tiles of that item before it
    float* part;                                  // [2 * grid][positions of a tile] sums of items that more than one CTA has
    int box_pos, box_dim[4];                      // keys come in boxes of so many positions (0: in pieces of 16 bytes); what dimensions 1 .. 4 of their map are
    int q_boxes;                                  // the queries of a row tile are one box
};

uint64_t weigh_many_bytes();
cudaError_t launch_weigh_many(const PoolDev& p, const BookDev& b, const WeighArgs& a, void* workspace, bool bf16, uint32_t* status, cudaStream_t st);

#ifdef __CUDACC__
namespace {

// A session as the call gives it, cut to what there is: entries first .. first + n - 1 of the list stand at its last n positions.
struct Newest { int first, n, len; };
__device__ __forceinline__ Newest newest_of(const PoolDev& p, const BookDev& b, const WeighArgs& a, int s, bool* bad) {
    const int b0 = a.begin[s], b1 = a.begin[s + 1], len = b.len[s], most = most_positions(b, p);
    Newest x;
    x.first = min(max(b0, 0), a.n_list);
    x.n = min(max(b1, x.first), a.n_list) - x.first;
    x.len = x.n > 0 ? min(max(len, 0), most) : 0;
    *bad = b0 < 0 || b1 < b0 || b1 > a.n_list || len < 0 || len > most || x.n > len;
    return x;
}

// A position's weight: `sum` is what it receives; there: it has a page.
__device__ __forceinline__ void put_weight(const WeighArgs& a, const Newest& x, int s, int h, int t, float sum, bool there, uint32_t* status) {
    if (t >= a.n_pos) { atomicOr(status, kStCapacity); return; }
    float* w = a.weight + (int64_t)s * a.ws_row + (int64_t)h * a.ws_head + t;
    const float old = t < x.len - x.n && a.decay != 0.f ? *w * a.decay : 0.f;
    *w = there ? old + sum : old;
}

}  // namespace
#endif

}  // namespace plc
