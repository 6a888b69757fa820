// C ABI of the attention-layer calls (treewy_attn.h): argument checks and kernel dispatch.  No allocation, no
// host synchronisation, no state kept between calls.
#include <float.h>

#include "attn_common.cuh"
#include "treewy_kernels.cuh"

using namespace treewy;

namespace {

inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool bad_ptr(const void *p) { return p == nullptr || misaligned(p); }
inline bool bad_dtype(int d) { return d != TREEWY_F32 && d != TREEWY_BF16; }
inline int elem_size(treewy_dtype_t t) { return t == TREEWY_BF16 ? 2 : 4; }
// a distance between rows: whole 16-byte vectors, rows that do not overlap
inline bool bad_stride(int64_t ld, int64_t least, int elem) { return ld < least || ld % (16 / elem) != 0; }
// rows whose elements 32 bits do not count (the kernels take offsets within a row in 32 bits)
inline bool wide_row(int64_t heads, int d) { return heads * d > INT32_MAX; }
inline treewy_status_t launched(cudaError_t e) { return e == cudaSuccess ? TREEWY_OK : TREEWY_ERR_CUDA; }

treewy_status_t check_cache(const treewy_kv_cache_t *c, int B, treewy_dtype_t io, CacheView *out)
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

treewy_status_t check_rope(const treewy_rope_t *r, int T, int d, int inverse, RopeView *out)
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

// the part of a tree that the attention calls read
treewy_status_t check_nodes(const treewy_tree_t *t, int *max_nodes)
{
    if (!t) return TREEWY_ERR_INVALID_ARG;
    if (t->B < 0 || t->T < 0 || t->max_nodes < 0) return TREEWY_ERR_INVALID_ARG;
    if (t->max_nodes > TREEWY_MAX_NODES) return TREEWY_ERR_UNSUPPORTED;
    *max_nodes = t->max_nodes == 0 ? TREEWY_MAX_NODES : t->max_nodes;
    if (t->B == 0) return TREEWY_OK;
    if (bad_ptr(t->node_offsets) || (t->T > 0 && bad_ptr(t->anc_mask))) return TREEWY_ERR_INVALID_ARG;
    return TREEWY_OK;
}

treewy_status_t attn_args(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, int32_t H_q, int32_t shared_len,
                          treewy_dtype_t io, AttnArgs *a)
{
    *a = {};
    int max_nodes = 0;
    treewy_status_t st = check_nodes(tree, &max_nodes);
    if (st != TREEWY_OK) return st;
    st = check_cache(cache, tree->B, io, &a->c);
    if (st != TREEWY_OK) return st;
    if (H_q < 1 || H_q % cache->H_kv != 0) return TREEWY_ERR_INVALID_ARG;
    if (wide_row(H_q, cache->d_head)) return TREEWY_ERR_UNSUPPORTED;
    if (shared_len < 0 || shared_len % cache->page_size != 0) return TREEWY_ERR_INVALID_ARG;
    a->node_offsets = tree->node_offsets, a->anc_mask = tree->anc_mask;
    a->B = tree->B, a->T = tree->T, a->max_nodes = max_nodes, a->H_q = H_q, a->G = H_q / cache->H_kv;
    a->shared_len = shared_len;
    return TREEWY_OK;
}

size_t workspace_of(const AttnArgs &a, treewy_dtype_t io)
{
    return attn_tc_applies(a, io) ? attn_tc_workspace(a) : attn_generic_workspace(a);
}

treewy_status_t attn_common(bool force_generic, const treewy_kv_cache_t *cache, const treewy_tree_t *tree, const void *q,
                            int64_t ld_q, const void *k, int64_t ld_k, const void *v, int64_t ld_v, int32_t H_q, float scale,
                            const int32_t *shared_pages, int32_t shared_len, treewy_dtype_t io, void *O, void *workspace,
                            size_t workspace_bytes, int32_t *seq_status, void *cuda_stream)
{
    AttnArgs a;
    treewy_status_t st = attn_args(cache, tree, H_q, shared_len, io, &a);
    if (st != TREEWY_OK) return st;
    if (seq_status && misaligned(seq_status)) return TREEWY_ERR_INVALID_ARG;
    if (!(scale > 0.f) || scale > FLT_MAX) return TREEWY_ERR_INVALID_ARG;
    if (tree->B == 0 || tree->T == 0) return TREEWY_OK;
    const int64_t kv_row = (int64_t)cache->H_kv * cache->d_head, q_row = (int64_t)H_q * cache->d_head;
    const int e = elem_size(io);
    if (bad_ptr(q) || bad_ptr(k) || bad_ptr(v) || bad_ptr(O) || bad_stride(ld_q, q_row, e) || bad_stride(ld_k, kv_row, e) ||
        bad_stride(ld_v, kv_row, e))
        return TREEWY_ERR_INVALID_ARG;
    if (shared_len > 0 && bad_ptr(shared_pages)) return TREEWY_ERR_INVALID_ARG;
    const size_t need = force_generic ? attn_generic_workspace(a) : workspace_of(a, io);
    if (workspace_bytes < need || (need > 0 && bad_ptr(workspace))) return TREEWY_ERR_INVALID_ARG;
    a.q = q, a.k = k, a.v = v, a.ld_q = ld_q, a.ld_k = ld_k, a.ld_v = ld_v, a.O = O;
    a.shared_pages = shared_pages, a.scale = scale, a.ws = static_cast<float *>(workspace), a.seq_status = seq_status;
    a.wait_cycles = debug_inject().wait_cycles, a.skip_item = debug_inject().skip_item;
    if (!force_generic && attn_tc_applies(a, io)) return launched(launch_attn_tc(a, static_cast<cudaStream_t>(cuda_stream)));
    return launched(launch_attn_generic(a, io, static_cast<cudaStream_t>(cuda_stream)));
}

// row_offsets NULL: one status word for all rows
treewy_status_t rope_common(const treewy_rope_t *rope, int32_t B, int32_t T, const int32_t *row_offsets, const void *x,
                            int64_t ld_x, void *y, int64_t ld_y, int32_t H, int32_t d_head, int32_t inverse,
                            treewy_dtype_t io_dtype, int32_t *status, void *cuda_stream)
{
    if (T < 0 || H < 1 || d_head < 2) return TREEWY_ERR_INVALID_ARG;
    if (bad_dtype(io_dtype) || d_head % 2 != 0 || wide_row(H, d_head)) return TREEWY_ERR_UNSUPPORTED;
    RowsArgs a = {};
    treewy_status_t st = check_rope(rope, T, d_head, inverse, &a.r);
    if (st != TREEWY_OK) return st;
    if (status && misaligned(status)) return TREEWY_ERR_INVALID_ARG;
    if (T == 0) return TREEWY_OK;
    const int e = elem_size(io_dtype);
    const int64_t row = (int64_t)H * d_head;
    if (bad_ptr(x) || bad_ptr(y) || bad_stride(ld_x, row, e) || bad_stride(ld_y, row, e)) return TREEWY_ERR_INVALID_ARG;
    a.q = x, a.ld_q = ld_x, a.q_out = y, a.ld_qo = ld_y;
    a.row_offsets = row_offsets, a.B = B, a.T = T, a.H_q = H, a.d = d_head, a.status = status;
    return launched(launch_rows(a, io_dtype, static_cast<cudaStream_t>(cuda_stream)));
}

}  // namespace

extern "C" {

treewy_status_t treewy_rope(const treewy_rope_t *rope, const void *x, int64_t ld_x, void *y, int64_t ld_y, int32_t T,
                            int32_t H, int32_t d_head, int32_t inverse, treewy_dtype_t io_dtype, int32_t *row_status,
                            void *cuda_stream)
{
    return rope_common(rope, 0, T, nullptr, x, ld_x, y, ld_y, H, d_head, inverse, io_dtype, row_status, cuda_stream);
}

treewy_status_t treewy_rope_rows(const treewy_rope_t *rope, int32_t B, int32_t T, const int32_t *row_offsets, const void *x,
                                 int64_t ld_x, void *y, int64_t ld_y, int32_t H, int32_t d_head, int32_t inverse,
                                 treewy_dtype_t io_dtype, int32_t *seq_status, void *cuda_stream)
{
    if (B < 0) return TREEWY_ERR_INVALID_ARG;
    if (B > 0 && T > 0 && bad_ptr(row_offsets)) return TREEWY_ERR_INVALID_ARG;
    return rope_common(rope, B, B > 0 ? T : 0, row_offsets, x, ld_x, y, ld_y, H, d_head, inverse, io_dtype, seq_status, cuda_stream);
}

treewy_status_t treewy_kv_append(const treewy_kv_cache_t *cache, const treewy_rope_t *rope, int32_t B, int32_t T,
                                 const int32_t *row_offsets, const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                                 int32_t H_q, const void *q, int64_t ld_q, void *q_out, int64_t ld_qo,
                                 treewy_dtype_t io_dtype, int32_t *seq_status, void *cuda_stream)
{
    if (B < 0 || T < 0 || H_q < 0) return TREEWY_ERR_INVALID_ARG;
    RowsArgs a = {};
    treewy_status_t st = check_cache(cache, B, io_dtype, &a.c);
    if (st != TREEWY_OK) return st;
    if (wide_row(H_q, cache->d_head)) return TREEWY_ERR_UNSUPPORTED;
    if (rope) {
        st = check_rope(rope, T, cache->d_head, 0, &a.r);
        if (st != TREEWY_OK) return st;
    }
    if (seq_status && misaligned(seq_status)) return TREEWY_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return TREEWY_OK;
    const int e = elem_size(io_dtype);
    const int64_t kv_row = (int64_t)cache->H_kv * cache->d_head, q_row = (int64_t)H_q * cache->d_head;
    if (bad_ptr(row_offsets) || bad_ptr(k) || bad_ptr(v) || bad_stride(ld_k, kv_row, e) || bad_stride(ld_v, kv_row, e))
        return TREEWY_ERR_INVALID_ARG;
    if (H_q > 0 && (bad_ptr(q) || bad_ptr(q_out) || bad_stride(ld_q, q_row, e) || bad_stride(ld_qo, q_row, e)))
        return TREEWY_ERR_INVALID_ARG;
    a.row_offsets = row_offsets, a.q = q, a.k = k, a.v = v, a.q_out = q_out;
    a.ld_q = ld_q, a.ld_k = ld_k, a.ld_v = ld_v, a.ld_qo = ld_qo;
    a.B = B, a.T = T, a.H_q = H_q, a.d = cache->d_head, a.status = seq_status;
    return launched(launch_rows(a, io_dtype, static_cast<cudaStream_t>(cuda_stream)));
}

size_t treewy_attn_workspace(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, int32_t H_q, int32_t shared_len,
                             treewy_dtype_t io_dtype)
{
    AttnArgs a;
    if (attn_args(cache, tree, H_q, shared_len, io_dtype, &a) != TREEWY_OK || a.B == 0 || a.T == 0) return 0;
    const size_t g = attn_generic_workspace(a), w = workspace_of(a, io_dtype);
    return g > w ? g : w;
}

treewy_status_t treewy_attn_verify(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, const void *q,
                                   int64_t ld_q, const void *k, int64_t ld_k, const void *v, int64_t ld_v, int32_t H_q,
                                   float scale, const int32_t *shared_pages, int32_t shared_len,
                                   treewy_dtype_t io_dtype, void *O, void *workspace, size_t workspace_bytes,
                                   int32_t *seq_status, void *cuda_stream)
{
    return attn_common(false, cache, tree, q, ld_q, k, ld_k, v, ld_v, H_q, scale, shared_pages, shared_len, io_dtype, O,
                       workspace, workspace_bytes, seq_status, cuda_stream);
}

treewy_status_t treewy_attn_verify_generic(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, const void *q,
                                           int64_t ld_q, const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                                           int32_t H_q, float scale, const int32_t *shared_pages, int32_t shared_len,
                                           treewy_dtype_t io_dtype, void *O, void *workspace, size_t workspace_bytes,
                                           int32_t *seq_status, void *cuda_stream)
{
    return attn_common(true, cache, tree, q, ld_q, k, ld_k, v, ld_v, H_q, scale, shared_pages, shared_len, io_dtype, O,
                       workspace, workspace_bytes, seq_status, cuda_stream);
}

treewy_status_t treewy_kv_commit(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, const void *k, int64_t ld_k,
                                 const void *v, int64_t ld_v, const int32_t *accepted, treewy_dtype_t io_dtype,
                                 int32_t *new_context_len, int32_t *seq_status, void *cuda_stream)
{
    int max_nodes = 0;
    KvCommitArgs a = {};
    treewy_status_t st = check_nodes(tree, &max_nodes);
    if (st != TREEWY_OK) return st;
    st = check_cache(cache, tree->B, io_dtype, &a.c);
    if (st != TREEWY_OK) return st;
    if (seq_status && misaligned(seq_status)) return TREEWY_ERR_INVALID_ARG;
    if (new_context_len && (misaligned(new_context_len) || new_context_len == cache->context_len)) return TREEWY_ERR_INVALID_ARG;
    if (tree->B == 0) return TREEWY_OK;
    const int64_t kv_row = (int64_t)cache->H_kv * cache->d_head;
    const int e = elem_size(io_dtype);
    if (bad_ptr(accepted)) return TREEWY_ERR_INVALID_ARG;
    // (no rows at all: the kernel flags every sequence, as it does an empty one among others)
    if (tree->T > 0 && (bad_ptr(k) || bad_ptr(v) || bad_stride(ld_k, kv_row, e) || bad_stride(ld_v, kv_row, e)))
        return TREEWY_ERR_INVALID_ARG;
    a.node_offsets = tree->node_offsets, a.anc_mask = tree->anc_mask;
    a.k = k, a.v = v, a.ld_k = ld_k, a.ld_v = ld_v, a.accepted = accepted;
    a.new_len = new_context_len, a.seq_status = seq_status;
    a.B = tree->B, a.T = tree->T, a.max_nodes = max_nodes;
    return launched(launch_kv_commit(a, io_dtype, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
