// Paged cache: what the calls on page pools and page books share (argument checks, device-side views).
#pragma once
#include "plc_common.cuh"

namespace plc {

constexpr int kMostPositions = 0x7fff0000;        // of a row

// A pool as the kernels see it: strides in bytes.
struct PoolDev {
    uint8_t* base;
    int64_t sl, skv, spage, sh, sp;
    int L, H, d, n_pages, page_pos, esz;
};
struct BookDev {
    int32_t* table; int32_t* len; int32_t* ref;
    int rows, max_pages;
};

inline bool plc_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline plc_status check_pool(const plc_page_pool* p, PoolDev* out) {
    if (!p || !p->view.base_dev || p->n_layers < 1 || p->n_kv_heads < 1 || p->n_pages < 1 || p->page_pos < 1) return PLC_E_INVALID;
    if (p->dtype != PLC_OUT_F32 && p->dtype != PLC_OUT_F16 && p->dtype != PLC_OUT_BF16) return PLC_E_INVALID;
    if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return PLC_E_SHAPE;
    if (p->n_pages > (1 << 28) || p->n_layers > (1 << 14) || p->n_kv_heads > (1 << 14) || p->page_pos > (1 << 14)) return PLC_E_SHAPE;
    const int esz = p->dtype == PLC_OUT_F32 ? 4 : 2;
    const int64_t st[5] = {p->view.stride_layer, p->view.stride_kv, p->view.stride_session, p->view.stride_head, p->view.stride_pos};
    if (!plc_aligned16(p->view.base_dev)) return PLC_E_ALIGN;
    for (int64_t s : st)
        if (s * esz % 16) return PLC_E_ALIGN;
    *out = PoolDev{static_cast<uint8_t*>(p->view.base_dev), st[0] * esz, st[1] * esz, st[2] * esz, st[3] * esz, st[4] * esz,
                   p->n_layers, p->n_kv_heads, p->head_dim, p->n_pages, p->page_pos, esz};
    return PLC_OK;
}

inline plc_status check_book(const plc_page_book* b, BookDev* out) {
    if (!b || !b->table_dev || !b->len_dev || !b->ref_dev || b->rows < 1 || b->max_pages < 1) return PLC_E_INVALID;
    if (b->rows > (1 << 20)) return PLC_E_SHAPE;
    *out = BookDev{b->table_dev, b->len_dev, b->ref_dev, b->rows, b->max_pages};
    return PLC_OK;
}

#ifdef __CUDACC__
// Positions that `max_pages` pages hold, as far as an int counts them with a tile's positions to spare.
__device__ __forceinline__ int most_positions(const BookDev& b, const PoolDev& p) {
    return (int)min((long long)b.max_pages * p.page_pos, (long long)kMostPositions);
}
#endif

}  // namespace plc
