// Host-side argument checks that the attention-layer calls share (treewy_attn.h, treewy_prompt.h).
#pragma once

#include "attn_common.cuh"

namespace treewy {

inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool bad_ptr(const void *p) { return p == nullptr || misaligned(p); }
inline bool bad_dtype(int d) { return d != TREEWY_F32 && d != TREEWY_BF16; }
inline int elem_size(treewy_dtype_t t) { return t == TREEWY_BF16 ? 2 : 4; }
// a distance between rows: whole 16-byte vectors, rows that do not overlap
inline bool bad_stride(int64_t ld, int64_t least, int elem) { return ld < least || ld % (16 / elem) != 0; }
// rows whose elements 32 bits do not count (the kernels take offsets within a row in 32 bits)
inline bool wide_row(int64_t heads, int d) { return heads * d > INT32_MAX; }
inline treewy_status_t launched(cudaError_t e) { return e == cudaSuccess ? TREEWY_OK : TREEWY_ERR_CUDA; }

inline treewy_status_t check_cache(const treewy_kv_cache_t *c, int B, treewy_dtype_t io, CacheView *out)
{
    if (!c || bad_dtype(io)) return c ? TREEWY_ERR_UNSUPPORTED : TREEWY_ERR_INVALID_ARG;
    if (c->n_pages < 0 || c->page_size < 1 || c->max_pages < 0 || c->H_kv < 1 || c->d_head < 1) return TREEWY_ERR_INVALID_ARG;
    if (c->d_head % 8 != 0 || c->d_head > 256 || wide_row(c->H_kv, c->d_head)) return TREEWY_ERR_UNSUPPORTED;
    if ((int64_t)c->max_pages * c->page_size > INT32_MAX - TREEWY_MAX_NODES) return TREEWY_ERR_UNSUPPORTED;  // tokens are int32
    const int vec = 16 / elem_size(io);
    if (c->stride_page < 0 || c->stride_slot < 0 || c->stride_head < 0 || c->stride_page % vec || c->stride_slot % vec ||
        c->stride_head % vec)
        return TREEWY_ERR_INVALID_ARG;
    if (B > 0 && bad_ptr(c->context_len)) return TREEWY_ERR_INVALID_ARG;
    if (B > 0 && c->max_pages > 0 && (bad_ptr(c->page_table) || (c->n_pages > 0 && (bad_ptr(c->k) || bad_ptr(c->v)))))
        return TREEWY_ERR_INVALID_ARG;
    *out = {c->k, c->v, c->stride_page, c->stride_slot, c->stride_head, c->page_table, c->context_len,
            c->n_pages, c->page_size, c->max_pages, c->H_kv, c->d_head};
    return TREEWY_OK;
}

inline treewy_status_t check_rope(const treewy_rope_t *r, int T, int d, int inverse, RopeView *out)
{
    if (!r) return TREEWY_ERR_INVALID_ARG;
    if (r->n_axes < 1 || r->max_positions < 1 || r->rot_dim < 2) return TREEWY_ERR_INVALID_ARG;
    if (r->rot_dim % 2 != 0 || r->rot_dim > d || r->n_axes > 32) return TREEWY_ERR_UNSUPPORTED;
    if (T > 0 && (bad_ptr(r->cos_sin) || bad_ptr(r->positions) || (r->pair_axis && misaligned(r->pair_axis))))
        return TREEWY_ERR_INVALID_ARG;
    *out = {r->cos_sin, r->positions, r->pair_axis, r->n_axes, r->max_positions, r->rot_dim, r->interleaved ? 1 : 0,
            inverse ? 1 : 0};
    return TREEWY_OK;
}

}  // namespace treewy
