// A KV cache as the append and tree-attention entry points see it: contiguous, or in pages with a table per
// (sequence, KV head).
#pragma once
#include "common.cuh"

namespace lvlm {

constexpr int kMinPage = 16;

struct CacheGeom {
    int32_t Hkv, cap;
    int32_t page, shift, n_pages, max_pages;   // page 0 = contiguous; page = 1 << shift
    int64_t sb, sh;                            // elements between sequences and heads; paged: sh = between pages, sb unused
};

// Host: the geometry of (Kc, Vc, table), or why it cannot be.
inline lvlm_status cache_geom(const lvlm_dims* d, const int32_t* table, CacheGeom* c) {
    c->Hkv = d->Hkv;
    if (!table) {
        if (d->page != 0 || d->cap <= 0) return LVLM_ERR_INVALID_ARG;
        c->cap = d->cap;
        c->page = c->shift = c->n_pages = c->max_pages = 0;
        c->sh = d->kv_stride_h ? d->kv_stride_h : (int64_t)d->cap * kHeadDim;
        c->sb = d->kv_stride_b ? d->kv_stride_b : (int64_t)d->Hkv * c->sh;
    } else {
        if (d->page <= 0 || d->n_pages <= 0 || d->max_pages <= 0) return LVLM_ERR_INVALID_ARG;
        if (d->page < kMinPage || (d->page & (d->page - 1))) return LVLM_ERR_UNSUPPORTED;
        const int64_t cap = (int64_t)d->page * d->max_pages;
        if (cap > 0x7FFFFF00ll) return LVLM_ERR_UNSUPPORTED;
        c->cap = (int32_t)cap;
        c->page = d->page; c->n_pages = d->n_pages; c->max_pages = d->max_pages;
        c->shift = 0;
        while ((1 << c->shift) < d->page) ++c->shift;
        c->sh = d->page_stride ? d->page_stride : (int64_t)d->page * kHeadDim;
        c->sb = 0;
        if (c->sh < (int64_t)d->page * kHeadDim) return LVLM_ERR_INVALID_ARG;
    }
    return c->sh % 8 || c->sb % 8 ? LVLM_ERR_ALIGNMENT : LVLM_OK;
}

// Host: whether the np bytes from p and the nq bytes from q share some.
inline bool overlap(const void* p, int64_t np, const void* q, int64_t nq) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + (uintptr_t)nq && b < a + (uintptr_t)np;
}

// Device: element offset of row `row` (0 <= row < cap) of head hd = b * Hkv + g, or -1: its page number is not one of the pool.
__device__ __forceinline__ int64_t cache_row(const CacheGeom& c, const int32_t* table, int b, int g, int row) {
    if (!c.page) return (int64_t)b * c.sb + (int64_t)g * c.sh + (int64_t)row * kHeadDim;
    const int id = *(table + ((int64_t)b * c.Hkv + g) * c.max_pages + (row >> c.shift));
    return id < 0 || id >= c.n_pages ? -1 : (int64_t)id * c.sh + (int64_t)(row & (c.page - 1)) * kHeadDim;
}

}  // namespace lvlm
