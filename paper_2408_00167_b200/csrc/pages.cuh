// The paged 8-bit cache: device view, metadata of one request, addresses.
//
// Tokens of a request live in pages of kPage tokens, listed in its row of the page table.  A full page holds e4m3 codes with one
// scale for each KV head, separately for K and V; the tokens behind the last full page wait in the request's open rows, in the
// type of the model, so that a page is quantised once and from unrounded values however the tokens arrived.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "finch_internal.cuh"

namespace finch {

constexpr int kPage = FINCH_PAGE_TOKENS;
constexpr float kE4m3Max = 448.f;

struct PagesView {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    char *open_k, *open_v;
    const int *table, *open_slot;
    int n_pages, table_width, n_open;

    __device__ __forceinline__ int64_t page_head(const ModelView &mv, int l, int page, int h) const {
        return ((int64_t)l * n_pages + page) * mv.Hkv + h;
    }
    // first open row of a request, in rows of head_dim elements
    __device__ __forceinline__ int64_t open_row(const ModelView &mv, int l, int slot, int h) const {
        return (((int64_t)l * n_open + slot) * mv.Hkv + h) * kPage;
    }
};

struct PagedView {
    int batch;
    const int *q_off, *new_off, *len;
    int total_q, total_new, max_q, max_new, max_len;
};

struct PagedInfo {
    int b, len, slot;  // tokens that are there, open rows' slot
    int row0, n;       // query rows (attention) or new rows (append)
    bool ok;
};

__device__ __forceinline__ PagedInfo paged_info(const PagesView &pg, const PagedView &bv, int b, bool append) {
    PagedInfo u;
    const int *off = append ? bv.new_off : bv.q_off;
    const int most = append ? bv.max_new : bv.max_q, total = append ? bv.total_new : bv.total_q;
    u.b = b;
    u.len = bv.len[b];
    u.slot = pg.open_slot ? pg.open_slot[b] : b;
    u.row0 = off[b];
    u.n = off[b + 1] - u.row0;
    u.ok = u.len >= 0 && u.len <= bv.max_len && u.slot >= 0 && u.slot < pg.n_open && u.n >= 0 && u.n <= most && u.row0 >= 0 &&
           u.row0 <= total - u.n;
    return u;
}

inline PagesView view_of(const finch_pages *p) {
    return PagesView{(uint8_t *)p->k, (uint8_t *)p->v, p->k_scale, p->v_scale, (char *)p->open_k, (char *)p->open_v, p->table,
                     p->open_slot, p->n_pages, p->table_width, p->n_open};
}
inline PagedView view_of(const finch_paged_batch *b) {
    return PagedView{b->batch, b->q_off, b->new_off, b->len, b->total_q, b->total_new, b->max_q, b->max_new, b->max_len};
}

}  // namespace finch
