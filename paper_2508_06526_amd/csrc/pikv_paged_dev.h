// A paged cache: where a slot of a shard lies.
#pragma once

#include "pikv_common.h"

namespace pikv {

// What the calls on paged shards check of their descriptor (its strides mean nothing there) and of the pages.
inline int check_paged(const pikv_desc *d, const pikv_pages *pages) {
    if (!d || !pages) return PIKV_ERR_INVALID;
    pikv_desc whole = *d;
    whole.stride_s = d->rank > 0 ? d->rank : d->D;
    whole.stride_h = (int64_t)(d->S > 0 ? d->S : 1) * whole.stride_s;
    if (d->Hq > kPagedRows) return PIKV_ERR_UNSUPPORTED;
    const int rc = check_slots(&whole, false);
    if (rc != PIKV_OK) return rc;
    if (d->rank != 0 || d->D < 32 || d->S > (1 << 30)) return PIKV_ERR_UNSUPPORTED;
    if (pages->n_pages < 1) return PIKV_ERR_INVALID;
    if (pages->page != 16 && pages->page != 32 && pages->page != 64 && pages->page != 128 && pages->page != 256) return PIKV_ERR_INVALID;
    const int64_t es = elem_bytes(d->dtype), D = d->D, sp = pages->stride_page, sh = pages->stride_h, ss = pages->stride_s;
    if (sp <= 0 || sh < 0 || ss < D) return PIKV_ERR_INVALID;
    if (ss > (1 << 24) / es || sh > ((int64_t)1 << 40) || sp > ((int64_t)1 << 40)) return PIKV_ERR_UNSUPPORTED;
    if (sp * es % 16 != 0 || sh * es % 16 != 0 || ss * es % 16 != 0) return PIKV_ERR_INVALID;
    // no two rows overlap: the rows of a head one behind the other, or the heads of a slot
    const int64_t rows = (int64_t)(pages->page - 1) * ss + D, heads = (int64_t)(d->Hkv - 1) * sh + D;
    if (d->Hkv > 1 && sh < rows && (sh < D || ss < heads)) return PIKV_ERR_INVALID;
    if (pages->n_pages > 1 && sp < rows + heads - D) return PIKV_ERR_INVALID;
    return PIKV_OK;
}

// Geometry of the pages in bytes, as the kernels take it.
struct PageGeometry {
    const int32_t *table;       // [B*E][per_shard]
    int64_t stride_page, stride_h, stride_s;
    int n_pages, bits, per_shard;
};
inline PageGeometry page_geometry(const pikv_desc *d, const pikv_pages *pages, const int32_t *table) {
    const int64_t es = elem_bytes(d->dtype);
    return PageGeometry{table, pages->stride_page * es, pages->stride_h * es, pages->stride_s * es, pages->n_pages,
                        __builtin_ctz(pages->page), (d->S - 1) / pages->page + 1};
}

// The byte offset of slot `slot` (0 .. S-1) of shard `be` in a pool, before its head; -1 where it has no page.
__device__ __forceinline__ int64_t slot_offset(const PageGeometry &g, int64_t be, int slot) {
    const int page = g.table[be * g.per_shard + (slot >> g.bits)];
    return page >= 0 && page < g.n_pages ? page * g.stride_page + (slot & ((1 << g.bits) - 1)) * g.stride_s : -1;
}

}  // namespace pikv
