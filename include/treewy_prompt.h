/*
 * treewy_prompt.h -- what takes a prompt, or any run of new tokens, through the attention layers of a hybrid, beside the
 * draft-tree calls of treewy_attn.h.  A step of such a layer is
 *       treewy_pages_reserve     once for all layers: pages for the new rows, their positions and slots,
 *       treewy_kv_append_norm    (or treewy_kv_append) queries and keys normalised and rotated, keys and values written
 *                                to the cache,
 *       treewy_attn_chunk        every new row attends to the cached tokens up to its own, or to a window of them;
 * single tokens are runs of one.  treewy_norm_rope normalises and rotates rows that stay packed (a draft tree's), and
 * treewy_norm_rope_backward is its gradient.
 *
 * Conventions are those of treewy_attn.h.  Packed rows are those of treewy_kv_append: sequence b owns rows row_offsets[b] ..
 * row_offsets[b+1]-1 of T (none is legal), and row i of them is its token context_len[b] + i.
 */
#ifndef TREEWY_PROMPT_H
#define TREEWY_PROMPT_H

#include "treewy_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* a further per-sequence status bit */
enum {
    TREEWY_SEQ_NO_PAGES = 512 /* the free list has run out before the sequence had its pages */
};

/*
 * Root-mean-square norm of one head's d_head elements ahead of the rotation,
 *       y = rotate(w x / sqrt(mean_c x_c^2 + eps)) ,   w = weight, or 1 + weight (plus_one),
 * in fp32 and rounded once (the sum of squares too: a head whose elements reach some 2^60 leaves its range and becomes 0).  weight
 * [d_head] is the same for all heads; weight_dtype may differ from the data's.
 */
typedef struct {
    const void *weight; /* device */
    treewy_dtype_t weight_dtype;
    float eps; /* positive and finite */
    int32_t plus_one;
} treewy_head_norm_t;

/*
 * y[t, h, :] from x[t, h, :], t < T, h < H; y may be x.  rope NULL: the norm alone.  row_offsets [B+1] NULL (B = 0): one
 * status word receives TREEWY_SEQ_BAD_POSITION, else it flags the row's sequence, as in treewy_rope and
 * treewy_rope_rows.  d_head is even, up to 256.
 */
treewy_status_t treewy_norm_rope(const treewy_head_norm_t *norm, const treewy_rope_t *rope, int32_t B, int32_t T,
                                 const int32_t *row_offsets, const void *x, int64_t ld_x, void *y, int64_t ld_y, int32_t H,
                                 int32_t d_head, treewy_dtype_t io_dtype, int32_t *seq_status, void *cuda_stream);
/*
 * Its backward pass.  With g = the rotation's transpose of dy, r = 1 / sqrt(mean x^2 + eps):
 *       dx = r (w g - x r mean_c(w g x r)) ,      dweight = sum over rows and heads of g x r   (fp32, overwritten) .
 * dx may be x or dy.  Rows whose position is out of range are flagged in the one row_status word (may be NULL), their dx is
 * not written, and they do not count in dweight.  Sums are taken in an order that the sizes alone decide.  workspace:
 * treewy_norm_rope_workspace bytes, no initial contents, one for each call in flight.
 */
size_t treewy_norm_rope_workspace(int32_t T, int32_t H, int32_t d_head, treewy_dtype_t io_dtype);
treewy_status_t treewy_norm_rope_backward(const treewy_head_norm_t *norm, const treewy_rope_t *rope, const void *x, int64_t ld_x,
                                          const void *dy, int64_t ld_dy, void *dx, int64_t ld_dx, float *dweight, int32_t T,
                                          int32_t H, int32_t d_head, treewy_dtype_t io_dtype, void *workspace,
                                          size_t workspace_bytes, int32_t *row_status, void *cuda_stream);
/* treewy_kv_append with norms: q_norm for the queries, k_norm for the keys (NULL: only rotated). */
treewy_status_t treewy_kv_append_norm(const treewy_kv_cache_t *cache, const treewy_rope_t *rope,
                                      const treewy_head_norm_t *q_norm, const treewy_head_norm_t *k_norm, int32_t B, int32_t T,
                                      const int32_t *row_offsets, const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                                      int32_t H_q, const void *q, int64_t ld_q, void *q_out, int64_t ld_qo,
                                      treewy_dtype_t io_dtype, int32_t *seq_status, void *cuda_stream);

/*
 * Attention of new rows over the cache.  Row i of sequence b stands at p = context_len[b] + i; its own key and value and those
 * of the rows before it are in the cache already (treewy_kv_append with the same row_offsets).  Query head h reads
 * key/value head g = h / (H_q / H_kv):
 *       o = sum_x softmax_x(scale * q . k_x) v_x ,   over the tokens x <= p with x > p - window or x < sinks .
 * window 0: all x <= p.  scale is positive and finite.  What a row may not see is never multiplied; page table entries
 * whose tokens no row sees are not read (a window's old pages may be gone).
 *   q [T,H_q,d]   rotated already;  O [T,H_q,d] contiguous, io_dtype.  Rows of no sequence are left as they are.
 *   workspace     treewy_attn_chunk_workspace bytes, which are enough for calls of fewer rows too; no initial contents,
 *                 nothing kept between calls; calls that may overlap in time need one each
 * d_head is a multiple of 8, up to 256.  BF16 with d_head 64, 128 or 256, page_size a power of two from 8 and at most
 * 128 query heads to a key/value head takes the tensor-core kernel; everything else an fp32 SIMT kernel.  Scores, softmax
 * statistics and accumulators are fp32; the tensor-core kernel rounds the softmax weights to bf16 (at most 2^-8 of
 * each) for the product with v.
 * A sequence whose range leaves the packed rows or runs backwards is flagged TREEWY_SEQ_BAD_OFFSETS, one whose rows do not fit
 * max_pages pages TREEWY_SEQ_BAD_LENGTH, one that sees a page out of range TREEWY_SEQ_BAD_PAGE, one with rows left
 * unwritten because a bounded wait gave up TREEWY_SEQ_TIMEOUT; the rows of O of a flagged sequence mean nothing.  (As in
 * treewy_kv_append a row that two sequences claim, beside one that runs backwards, is computed for one of them.)
 */
size_t treewy_attn_chunk_workspace(const treewy_kv_cache_t *cache, int32_t B, int32_t T, int32_t H_q, int32_t window,
                                   int32_t sinks, treewy_dtype_t io_dtype);
treewy_status_t treewy_attn_chunk(const treewy_kv_cache_t *cache, int32_t B, int32_t T, const int32_t *row_offsets, const void *q,
                                  int64_t ld_q, int32_t H_q, float scale, int32_t window, int32_t sinks,
                                  treewy_dtype_t io_dtype, void *O, void *workspace, size_t workspace_bytes, int32_t *seq_status,
                                  void *cuda_stream);
/* The same contract, always through the SIMT kernel: a cross-check for the tensor-core kernel. */
treewy_status_t treewy_attn_chunk_generic(const treewy_kv_cache_t *cache, int32_t B, int32_t T, const int32_t *row_offsets,
                                          const void *q, int64_t ld_q, int32_t H_q, float scale, int32_t window, int32_t sinks,
                                          treewy_dtype_t io_dtype, void *O, void *workspace, size_t workspace_bytes,
                                          int32_t *seq_status, void *cuda_stream);

/*
 * A page table kept on the GPU, and the pages that nobody holds.  Entry e of sequence b is page_table[b * max_pages + e]; a
 * negative entry holds no page.  free_pages [n_pages] is a stack of *free_count pages, the top last.  The caches of all
 * layers of a model go with one pool.  Calls on one pool are ordered by the caller (one stream).
 */
typedef struct {
    int32_t *page_table;             /* [B, max_pages] device */
    int32_t *free_pages, *free_count; /* device */
    int32_t n_pages, page_size, max_pages;
} treewy_page_pool_t;

/*
 * Reserve: every entry that the tokens context_len[b] .. context_len[b] + n_b - 1 fall into, n_b = row_offsets[b+1] -
 * row_offsets[b], and that holds no page gets one: in the order of sequences and entries, from the top of the stack
 * down.  Also, where not NULL, of each packed row: positions [T] int32 = its token's number, slots [T] int64 =
 * page * page_size + slot of its token, -1 where that has no page.  Rows of no sequence are left, and those of one whose
 * range or length is flagged.
 * Flags: TREEWY_SEQ_BAD_OFFSETS; TREEWY_SEQ_BAD_LENGTH when the rows do not fit max_pages; TREEWY_SEQ_NO_PAGES when the
 * stack has fewer pages left than the sequence and all before it want (it gets none, and neither does any after it that
 * wants some); TREEWY_SEQ_BAD_PAGE when its last token's page, only part of it in use, is not held, when a held entry is
 * out of range, or when the stack hands out a page that is (the entry stays empty).
 * B * max_pages is below 2^31.
 */
treewy_status_t treewy_pages_reserve(const treewy_page_pool_t *pool, int32_t B, int32_t T, const int32_t *context_len,
                                     const int32_t *row_offsets, int32_t *positions, int64_t *slots, int32_t *seq_status,
                                     void *cuda_stream);
/*
 * Release: the pages of sequence b whose tokens all lie in first[b] .. end[b] - 1 go back to the stack, in such an order that a
 * reserve of the same entries takes the same ones again; their entries become -1.  A page that is only partly in
 * the range stays; first >= end releases nothing; end is cut to max_pages pages, a negative first counts as 0.  An entry out of range
 * (>= n_pages) becomes -1 with TREEWY_SEQ_BAD_PAGE, as does one that the stack has no room for.
 * Who holds a page is not counted.  A page that stands in the tables of several sequences (a prompt that they share) goes back with the last of
 * them only: for the others `first` lies behind it.  One that is released twice is on the stack twice and is handed out twice, to
 * two sequences that then overwrite each other; that is not looked for, and shows only when the stack has no room.
 */
treewy_status_t treewy_pages_release(const treewy_page_pool_t *pool, int32_t B, const int32_t *first, const int32_t *end,
                                     int32_t *seq_status, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* TREEWY_PROMPT_H */
