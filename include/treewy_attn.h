/*
 * treewy_attn.h -- the attention layers of a Gated DeltaNet hybrid, beside the GDN calls of treewy.h:
 * draft trees verified through a softmax-attention layer over a paged key/value cache, and the
 * accepted path committed to that cache.  A speculative round of such a layer is
 *       treewy_rope         rotate the draft rows' queries and keys,
 *       treewy_attn_verify  attend from every node to its sequence's cache and to its ancestors,
 *       treewy_kv_commit    write the accepted path's keys and values to the cache;
 * a prompt, or a token that is not speculative, enters the cache through treewy_kv_append.
 *
 * The trees are the treewy_tree_t of treewy.h: the same node_offsets, parents and ancestor masks that
 * the round's GDN layers use, prepared once.  The draft rows stay packed ([T, heads, d]) until commit, as
 * q, k, v and U do in the GDN calls; rejected nodes never touch the cache.
 *
 * Conventions are those of treewy.h: device pointers, 16-byte aligned; no allocation, no host
 * synchronisation; host-checkable misuse returns an error and launches nothing; data-dependent errors
 * flag the sequence in seq_status (may be NULL; caller zeroes it) and skip it.  Element types are
 * TREEWY_BF16 and TREEWY_F32, one for all data of a call.  `ld_*` are the distances in elements between
 * the rows of consecutive tokens (a row is [heads, d], contiguous); they let q, k and v be column
 * ranges of one projection's output.  Row distances and the cache's strides are multiples of 16 bytes; a
 * row has fewer than 2^31 elements.
 */
#ifndef TREEWY_ATTN_H
#define TREEWY_ATTN_H

#include <stddef.h>

#include "treewy.h"

#ifdef __cplusplus
extern "C" {
#endif

/* further per-sequence status bits */
enum {
    TREEWY_SEQ_BAD_PAGE = 64,      /* a page index outside 0..n_pages-1 where a token of the sequence is */
    TREEWY_SEQ_BAD_LENGTH = 128,   /* context_len[b] negative, below shared_len, or rows past max_pages pages */
    TREEWY_SEQ_BAD_POSITION = 256  /* a position outside 0..max_positions-1 (or a pair's axis outside 0..n_axes-1) */
};

/*
 * A paged cache of keys and values.  Element c of head h of slot s (0 <= s < page_size) of page p is
 * k[p * stride_page + s * stride_slot + h * stride_head + c], and v likewise; token j of sequence b is slot
 * j % page_size of page page_table[b * max_pages + j / page_size].  Strides may put slots or heads first.
 */
typedef struct {
    void *k, *v;
    int64_t stride_page, stride_slot, stride_head; /* elements */
    const int32_t *page_table;                     /* [B, max_pages] device */
    const int32_t *context_len;                    /* [B] device: committed tokens of each sequence */
    int32_t n_pages, page_size, max_pages;
    int32_t H_kv, d_head;
} treewy_kv_cache_t;

/*
 * Rotary positions with several axes.  Pair p (0 <= p < rot_dim / 2) of every head of token t turns by the
 * angle whose cosine and sine are cos_sin[pos * rot_dim + p] and cos_sin[pos * rot_dim + rot_dim / 2 + p],
 * pos = positions[a * T + t], a = pair_axis[p] (time, height, width, ...; NULL: axis 0 for every pair):
 *       (x, y) -> (x cos - y sin, y cos + x sin) .
 * Members of pair p: elements p and p + rot_dim / 2 of the head, or (interleaved) 2p and 2p + 1.  Elements
 * rot_dim and up are copied.  Products are formed in fp32 and rounded once.
 */
typedef struct {
    const float *cos_sin;       /* [max_positions, rot_dim] device */
    const int32_t *positions;   /* [n_axes, T] device */
    const uint8_t *pair_axis;   /* [rot_dim / 2] device, or NULL */
    int32_t n_axes, max_positions, rot_dim, interleaved;
} treewy_rope_t;

/*
 * y[t, h, :] = rotated x[t, h, :], t < T, h < H, rows of d_head elements; y may be x.  inverse != 0 turns the
 * other way: the rotation's transpose, which is its backward pass.  One row_status word (may be NULL)
 * receives TREEWY_SEQ_BAD_POSITION when some token's position is out of range; such rows are not
 * written.  d_head and rot_dim are even, rot_dim <= d_head, n_axes <= 32.
 */
treewy_status_t treewy_rope(const treewy_rope_t *rope, const void *x, int64_t ld_x, void *y, int64_t ld_y, int32_t T,
                            int32_t H, int32_t d_head, int32_t inverse, treewy_dtype_t io_dtype, int32_t *row_status,
                            void *cuda_stream);
/* The same for the packed rows of sequences (row_offsets [B+1], as in treewy_kv_append): a position out of range flags
 * seq_status[b] (may be NULL) of the row's own sequence. */
treewy_status_t treewy_rope_rows(const treewy_rope_t *rope, int32_t B, int32_t T, const int32_t *row_offsets, const void *x,
                                 int64_t ld_x, void *y, int64_t ld_y, int32_t H, int32_t d_head, int32_t inverse,
                                 treewy_dtype_t io_dtype, int32_t *seq_status, void *cuda_stream);

/*
 * Append: row i of sequence b (packed rows row_offsets[b] .. row_offsets[b+1]-1 of T; none is legal) goes to slot
 * context_len[b] + i of the cache: v as it is, k rotated on the way (rope NULL: as it is).  With H_q > 0 the
 * rows' queries are rotated in the same pass, q [T, H_q, d] -> q_out [T, H_q, d] (q_out may be q).
 * context_len is not advanced: every layer of a step appends at the same place.  A sequence whose rows do
 * not fit its max_pages pages is flagged TREEWY_SEQ_BAD_LENGTH and skipped, one whose range leaves the packed rows
 * or runs backwards TREEWY_SEQ_BAD_OFFSETS; a row whose page is out of range or whose position is, is skipped with
 * its flag.  (A row that two sequences claim, beside one that runs backwards, goes to one of them.)
 */
treewy_status_t treewy_kv_append(const treewy_kv_cache_t *cache, const treewy_rope_t *rope, int32_t B, int32_t T,
                                 const int32_t *row_offsets, const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                                 int32_t H_q, const void *q, int64_t ld_q, void *q_out, int64_t ld_qo,
                                 treewy_dtype_t io_dtype, int32_t *seq_status, void *cuda_stream);

/*
 * Draft-tree attention.  Node i of sequence b, query head h, reads key/value head g = h / (H_q / H_kv):
 *       o = sum_j softmax_j(scale * q . k_j) v_j
 * over the sequence's context_len[b] cached tokens and the packed draft rows j whose bit is set in
 * tree->anc_mask[i] (ancestors and the node itself).  Trees of one node are ordinary decoding.  A node
 * that sees nothing (no context, an empty mask) gets o = 0; what no node may see is never multiplied, so
 * NaN or infinity there does not spread.  scale is positive and finite.
 *   q [T,H_q,d], k, v [T,H_kv,d]   the draft rows (rotated already);  O [T,H_q,d] contiguous, io_dtype
 *   shared_pages, shared_len       the first shared_len tokens (a multiple of page_size) of EVERY sequence
 *                                  are those of shared_pages [shared_len / page_size]: a prompt common to the
 *                                  batch, read once for all of it.  The page tables' entries for it are not
 *                                  read.  NULL and 0: nothing is shared.
 *   workspace                      treewy_attn_workspace bytes; no initial contents, nothing kept between
 *                                  calls; calls that may overlap in time need one each
 * Of the tree, B, T, max_nodes, node_offsets and anc_mask are read (as treewy_tree_prepare left it).
 * d_head is a multiple of 8, up to 256.  BF16 with d_head 64, 128 or 256 and page_size a power of two
 * from 8 takes the tensor-core kernel; everything else an fp32 SIMT kernel.  Scores, softmax statistics and
 * accumulators are fp32; the tensor-core kernel rounds the softmax weights to bf16 (at most 2^-8 of each) for
 * the product with v.
 * A bounded wait that gives up (treewy.h) flags TREEWY_SEQ_TIMEOUT on every sequence that has rows left unwritten.
 */
size_t treewy_attn_workspace(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, int32_t H_q,
                             int32_t shared_len, treewy_dtype_t io_dtype);
treewy_status_t treewy_attn_verify(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, const void *q,
                                   int64_t ld_q, const void *k, int64_t ld_k, const void *v, int64_t ld_v, int32_t H_q,
                                   float scale, const int32_t *shared_pages, int32_t shared_len,
                                   treewy_dtype_t io_dtype, void *O, void *workspace, size_t workspace_bytes,
                                   int32_t *seq_status, void *cuda_stream);
/* (treewy_debug_inject reaches the tensor-core kernel too: skip_item is then sequence * H_kv + key/value head.) */
/* The same contract, always through the SIMT kernel: a cross-check for the tensor-core kernel. */
treewy_status_t treewy_attn_verify_generic(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, const void *q,
                                           int64_t ld_q, const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                                           int32_t H_q, float scale, const int32_t *shared_pages, int32_t shared_len,
                                           treewy_dtype_t io_dtype, void *O, void *workspace, size_t workspace_bytes,
                                           int32_t *seq_status, void *cuda_stream);

/*
 * Commit of the accepted path to the cache: for a = accepted[b] >= 0 the r-th node of a's root path (r = 0 at
 * the root; bits of anc_mask[a] in ascending order) has its packed k and v rows copied to slot
 * context_len[b] + r.  new_context_len [B] (may be NULL; must not be context_len) receives context_len[b] + the
 * path's length, for accepted = -1 context_len[b].  A flagged sequence (bad range, no node or too many, accepted
 * index, length or page) is skipped whole, its new_context_len untouched.
 */
treewy_status_t treewy_kv_commit(const treewy_kv_cache_t *cache, const treewy_tree_t *tree, const void *k, int64_t ld_k,
                                 const void *v, int64_t ld_v, const int32_t *accepted, treewy_dtype_t io_dtype,
                                 int32_t *new_context_len, int32_t *seq_status, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* TREEWY_ATTN_H */
