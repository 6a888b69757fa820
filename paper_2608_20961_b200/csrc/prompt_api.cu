// C ABI of the calls that take new rows through the attention layers (treewy_prompt.h): argument checks and kernel
// dispatch.  No allocation, no host synchronisation, no state kept between calls.
#include <float.h>

#include "attn_checks.cuh"
#include "treewy_kernels.cuh"

using namespace treewy;

namespace {

// norm NULL: none
treewy_status_t check_norm(const treewy_head_norm_t *n, NormView *out)
{
    *out = {};
    if (!n) return TREEWY_OK;
    if (bad_dtype(n->weight_dtype)) return TREEWY_ERR_UNSUPPORTED;
    if (bad_ptr(n->weight) || !(n->eps > 0.f) || n->eps > FLT_MAX) return TREEWY_ERR_INVALID_ARG;
    *out = {n->weight, n->weight_dtype == TREEWY_BF16, n->plus_one ? 1 : 0, n->eps};
    return TREEWY_OK;
}

// what forward and backward share
treewy_status_t norm_common(const treewy_head_norm_t *norm, const treewy_rope_t *rope, int32_t T, int32_t H, int32_t d, int inverse,
                            treewy_dtype_t io, NormView *n, RopeView *r)
{
    if (!norm || T < 0 || H < 1 || d < 2) return TREEWY_ERR_INVALID_ARG;
    if (bad_dtype(io) || d % 2 != 0 || d > 256 || wide_row(H, d)) return TREEWY_ERR_UNSUPPORTED;
    const treewy_status_t st = check_norm(norm, n);
    if (st != TREEWY_OK) return st;
    *r = {};
    return rope ? check_rope(rope, T, d, inverse, r) : TREEWY_OK;
}

treewy_status_t chunk_args(const treewy_kv_cache_t *cache, int32_t B, int32_t T, int32_t H_q, int32_t window, int32_t sinks,
                           treewy_dtype_t io, ChunkArgs *a)
{
    *a = {};
    if (B < 0 || T < 0) return TREEWY_ERR_INVALID_ARG;
    const treewy_status_t st = check_cache(cache, B, io, &a->c);
    if (st != TREEWY_OK) return st;
    if (H_q < 1 || H_q % cache->H_kv != 0 || window < 0 || sinks < 0) return TREEWY_ERR_INVALID_ARG;
    if (wide_row(H_q, cache->d_head)) return TREEWY_ERR_UNSUPPORTED;
    a->B = B, a->T = T, a->H_q = H_q, a->G = H_q / cache->H_kv;
    a->window = window == 0 ? INT32_MAX : window, a->sinks = sinks;
    return TREEWY_OK;
}

treewy_status_t chunk_common(bool force_generic, const treewy_kv_cache_t *cache, int32_t B, int32_t T, const int32_t *row_offsets,
                             const void *q, int64_t ld_q, int32_t H_q, float scale, int32_t window, int32_t sinks, treewy_dtype_t io,
                             void *O, void *workspace, size_t workspace_bytes, int32_t *seq_status, void *cuda_stream)
{
    ChunkArgs a;
    const treewy_status_t st = chunk_args(cache, B, T, H_q, window, sinks, io, &a);
    if (st != TREEWY_OK) return st;
    if (seq_status && misaligned(seq_status)) return TREEWY_ERR_INVALID_ARG;
    if (!(scale > 0.f) || scale > FLT_MAX) return TREEWY_ERR_INVALID_ARG;
    if (B == 0) return TREEWY_OK;
    if (T == 0) {              // (ranges that claim rows are flagged all the same)
        if (!seq_status) return TREEWY_OK;
        if (bad_ptr(row_offsets)) return TREEWY_ERR_INVALID_ARG;
        return launched(launch_no_rows(row_offsets, a.c.context_len, B, (int64_t)a.c.max_pages * a.c.page_size, seq_status, static_cast<cudaStream_t>(cuda_stream)));
    }
    if (bad_ptr(row_offsets) || bad_ptr(q) || bad_ptr(O) || bad_stride(ld_q, (int64_t)H_q * cache->d_head, elem_size(io)))
        return TREEWY_ERR_INVALID_ARG;
    const bool tc = !force_generic && chunk_tc_applies(a, io);
    const size_t need = tc ? chunk_tc_workspace(a) : chunk_generic_workspace(a);
    if (workspace_bytes < need || (need > 0 && bad_ptr(workspace))) return TREEWY_ERR_INVALID_ARG;
    a.row_offsets = row_offsets, a.q = q, a.ld_q = ld_q, a.O = O, a.scale = scale;
    a.ws = static_cast<float *>(workspace), a.seq_status = seq_status;
    a.wait_cycles = debug_inject().wait_cycles, a.skip_item = debug_inject().skip_item;
    if (tc) return launched(launch_chunk_tc(a, static_cast<cudaStream_t>(cuda_stream)));
    return launched(launch_chunk_generic(a, io, static_cast<cudaStream_t>(cuda_stream)));
}

treewy_status_t check_pool(const treewy_page_pool_t *p, int32_t B, PagesArgs *a)
{
    *a = {};
    if (!p || B < 0 || p->n_pages < 0 || p->page_size < 1 || p->max_pages < 0) return TREEWY_ERR_INVALID_ARG;
    if ((int64_t)p->max_pages * p->page_size > INT32_MAX || (int64_t)B * p->max_pages > INT32_MAX) return TREEWY_ERR_UNSUPPORTED;
    if (B > 0 && (bad_ptr(p->free_count) || (p->n_pages > 0 && bad_ptr(p->free_pages)) || (p->max_pages > 0 && bad_ptr(p->page_table))))
        return TREEWY_ERR_INVALID_ARG;
    a->page_table = p->page_table, a->free_pages = p->free_pages, a->free_count = p->free_count;
    a->n_pages = p->n_pages, a->page_size = p->page_size, a->max_pages = p->max_pages, a->B = B;
    return TREEWY_OK;
}

}  // namespace

extern "C" {

treewy_status_t treewy_norm_rope(const treewy_head_norm_t *norm, const treewy_rope_t *rope, int32_t B, int32_t T,
                                 const int32_t *row_offsets, const void *x, int64_t ld_x, void *y, int64_t ld_y, int32_t H,
                                 int32_t d_head, treewy_dtype_t io_dtype, int32_t *seq_status, void *cuda_stream)
{
    if (B < 0) return TREEWY_ERR_INVALID_ARG;
    NormRowsArgs a = {};
    const treewy_status_t st = norm_common(norm, rope, T, H, d_head, 0, io_dtype, &a.q, &a.rows.r);
    if (st != TREEWY_OK) return st;
    if (seq_status && misaligned(seq_status)) return TREEWY_ERR_INVALID_ARG;
    if (T == 0) return TREEWY_OK;
    const int e = elem_size(io_dtype);
    const int64_t row = (int64_t)H * d_head;
    if ((row_offsets && misaligned(row_offsets)) || (B > 0 && !row_offsets)) return TREEWY_ERR_INVALID_ARG;
    if (bad_ptr(x) || bad_ptr(y) || bad_stride(ld_x, row, e) || bad_stride(ld_y, row, e)) return TREEWY_ERR_INVALID_ARG;
    if (row_offsets && B == 0) return TREEWY_OK;       // rows of no sequence
    RowsArgs &r = a.rows;
    r.q = x, r.ld_q = ld_x, r.q_out = y, r.ld_qo = ld_y, r.row_offsets = row_offsets;
    r.B = B, r.T = T, r.H_q = H, r.d = d_head, r.status = seq_status;
    return launched(launch_norm_rows(a, io_dtype, static_cast<cudaStream_t>(cuda_stream)));
}

size_t treewy_norm_rope_workspace(int32_t T, int32_t H, int32_t d_head, treewy_dtype_t io_dtype)
{
    if (T < 0 || H < 1 || d_head < 2 || d_head > 256 || bad_dtype(io_dtype)) return 0;
    return norm_backward_workspace(d_head);
}

treewy_status_t treewy_norm_rope_backward(const treewy_head_norm_t *norm, const treewy_rope_t *rope, const void *x, int64_t ld_x,
                                          const void *dy, int64_t ld_dy, void *dx, int64_t ld_dx, float *dweight, int32_t T,
                                          int32_t H, int32_t d_head, treewy_dtype_t io_dtype, void *workspace,
                                          size_t workspace_bytes, int32_t *row_status, void *cuda_stream)
{
    NormBackwardArgs a = {};
    const treewy_status_t st = norm_common(norm, rope, T, H, d_head, 1, io_dtype, &a.norm, &a.rows.r);
    if (st != TREEWY_OK) return st;
    if (row_status && misaligned(row_status)) return TREEWY_ERR_INVALID_ARG;
    const int e = elem_size(io_dtype);
    const int64_t row = (int64_t)H * d_head;
    if (T > 0 && (bad_ptr(x) || bad_ptr(dy) || bad_ptr(dx) || bad_stride(ld_x, row, e) || bad_stride(ld_dy, row, e) || bad_stride(ld_dx, row, e)))
        return TREEWY_ERR_INVALID_ARG;
    if (bad_ptr(dweight) || bad_ptr(workspace) || workspace_bytes < norm_backward_workspace(d_head)) return TREEWY_ERR_INVALID_ARG;
    RowsArgs &r = a.rows;
    r.q = x, r.ld_q = ld_x, r.q_out = dx, r.ld_qo = ld_dx, r.T = T, r.H_q = H, r.d = d_head, r.status = row_status;
    a.dy = dy, a.ld_dy = ld_dy, a.dweight = dweight, a.parts = static_cast<float *>(workspace);
    // (no rows: dweight is still written)
    return launched(launch_norm_backward(a, io_dtype, static_cast<cudaStream_t>(cuda_stream)));
}

treewy_status_t treewy_kv_append_norm(const treewy_kv_cache_t *cache, const treewy_rope_t *rope, const treewy_head_norm_t *q_norm,
                                      const treewy_head_norm_t *k_norm, int32_t B, int32_t T, const int32_t *row_offsets,
                                      const void *k, int64_t ld_k, const void *v, int64_t ld_v, int32_t H_q, const void *q,
                                      int64_t ld_q, void *q_out, int64_t ld_qo, treewy_dtype_t io_dtype, int32_t *seq_status,
                                      void *cuda_stream)
{
    if (B < 0 || T < 0 || H_q < 0) return TREEWY_ERR_INVALID_ARG;
    NormRowsArgs na = {};
    RowsArgs &a = na.rows;
    treewy_status_t st = check_cache(cache, B, io_dtype, &a.c);
    if (st != TREEWY_OK) return st;
    if (wide_row(H_q, cache->d_head)) return TREEWY_ERR_UNSUPPORTED;
    if (rope) {
        st = check_rope(rope, T, cache->d_head, 0, &a.r);
        if (st != TREEWY_OK) return st;
    }
    if ((st = check_norm(q_norm, &na.q)) != TREEWY_OK || (st = check_norm(k_norm, &na.k)) != TREEWY_OK) return st;
    if (seq_status && misaligned(seq_status)) return TREEWY_ERR_INVALID_ARG;
    if (B == 0) return TREEWY_OK;
    if (T == 0) {              // (ranges that claim rows are flagged all the same)
        if (!seq_status) return TREEWY_OK;
        if (bad_ptr(row_offsets)) return TREEWY_ERR_INVALID_ARG;
        return launched(launch_no_rows(row_offsets, nullptr, B, 0, seq_status, static_cast<cudaStream_t>(cuda_stream)));
    }
    const int e = elem_size(io_dtype);
    const int64_t kv_row = (int64_t)cache->H_kv * cache->d_head, q_row = (int64_t)H_q * cache->d_head;
    if (bad_ptr(row_offsets) || bad_ptr(k) || bad_ptr(v) || bad_stride(ld_k, kv_row, e) || bad_stride(ld_v, kv_row, e))
        return TREEWY_ERR_INVALID_ARG;
    if (H_q > 0 && (bad_ptr(q) || bad_ptr(q_out) || bad_stride(ld_q, q_row, e) || bad_stride(ld_qo, q_row, e)))
        return TREEWY_ERR_INVALID_ARG;
    a.row_offsets = row_offsets, a.q = q, a.k = k, a.v = v, a.q_out = q_out;
    a.ld_q = ld_q, a.ld_k = ld_k, a.ld_v = ld_v, a.ld_qo = ld_qo;
    a.B = B, a.T = T, a.H_q = H_q, a.d = cache->d_head, a.status = seq_status;
    if (!q_norm && !k_norm) return launched(launch_rows(a, io_dtype, static_cast<cudaStream_t>(cuda_stream)));
    return launched(launch_norm_rows(na, io_dtype, static_cast<cudaStream_t>(cuda_stream)));
}

size_t treewy_attn_chunk_workspace(const treewy_kv_cache_t *cache, int32_t B, int32_t T, int32_t H_q, int32_t window, int32_t sinks,
                                   treewy_dtype_t io_dtype)
{
    ChunkArgs a;
    if (chunk_args(cache, B, T, H_q, window, sinks, io_dtype, &a) != TREEWY_OK || B == 0 || T == 0) return 0;
    const size_t g = chunk_generic_workspace_most(a), t = io_dtype == TREEWY_BF16 ? chunk_tc_workspace(a) : 0;
    return g > t ? g : t;
}

treewy_status_t treewy_attn_chunk(const treewy_kv_cache_t *cache, int32_t B, int32_t T, const int32_t *row_offsets, const void *q,
                                  int64_t ld_q, int32_t H_q, float scale, int32_t window, int32_t sinks, treewy_dtype_t io_dtype,
                                  void *O, void *workspace, size_t workspace_bytes, int32_t *seq_status, void *cuda_stream)
{
    return chunk_common(false, cache, B, T, row_offsets, q, ld_q, H_q, scale, window, sinks, io_dtype, O, workspace, workspace_bytes, seq_status,
                        cuda_stream);
}

treewy_status_t treewy_attn_chunk_generic(const treewy_kv_cache_t *cache, int32_t B, int32_t T, const int32_t *row_offsets,
                                          const void *q, int64_t ld_q, int32_t H_q, float scale, int32_t window, int32_t sinks,
                                          treewy_dtype_t io_dtype, void *O, void *workspace, size_t workspace_bytes,
                                          int32_t *seq_status, void *cuda_stream)
{
    return chunk_common(true, cache, B, T, row_offsets, q, ld_q, H_q, scale, window, sinks, io_dtype, O, workspace, workspace_bytes, seq_status,
                        cuda_stream);
}

treewy_status_t treewy_pages_reserve(const treewy_page_pool_t *pool, int32_t B, int32_t T, const int32_t *context_len,
                                     const int32_t *row_offsets, int32_t *positions, int64_t *slots, int32_t *seq_status,
                                     void *cuda_stream)
{
    PagesArgs a;
    if (T < 0) return TREEWY_ERR_INVALID_ARG;
    const treewy_status_t st = check_pool(pool, B, &a);
    if (st != TREEWY_OK) return st;
    if (misaligned(seq_status) || misaligned(positions) || misaligned(slots)) return TREEWY_ERR_INVALID_ARG;
    if (B == 0) return TREEWY_OK;
    if (bad_ptr(context_len) || bad_ptr(row_offsets)) return TREEWY_ERR_INVALID_ARG;
    a.T = T, a.context_len = context_len, a.row_offsets = row_offsets, a.positions = positions, a.slots = slots, a.seq_status = seq_status;
    return launched(launch_pages_reserve(a, static_cast<cudaStream_t>(cuda_stream)));
}

treewy_status_t treewy_pages_release(const treewy_page_pool_t *pool, int32_t B, const int32_t *first, const int32_t *end,
                                     int32_t *seq_status, void *cuda_stream)
{
    PagesArgs a;
    const treewy_status_t st = check_pool(pool, B, &a);
    if (st != TREEWY_OK) return st;
    if (misaligned(seq_status)) return TREEWY_ERR_INVALID_ARG;
    if (B == 0) return TREEWY_OK;
    if (bad_ptr(first) || bad_ptr(end)) return TREEWY_ERR_INVALID_ARG;
    a.first = first, a.end = end, a.seq_status = seq_status;
    return launched(launch_pages_release(a, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
