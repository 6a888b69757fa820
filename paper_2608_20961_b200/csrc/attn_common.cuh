// What the kernels of the attention layers share: their argument blocks, the address of a cached
// token, and the checks of one sequence.
#pragma once

#include "../../include/treewy_attn.h"
#include "../../include/treewy_prompt.h"
#include "treewy_common.cuh"

namespace treewy {

// the cache as kernels read it (strides in elements)
struct CacheView {
    void *k, *v;
    long long stride_page, stride_slot, stride_head;
    const int32_t *page_table, *context_len;
    int n_pages, page_size, max_pages, H_kv, d;
};

struct RopeView {
    const float *cos_sin;  // NULL: no rotation
    const int32_t *positions;
    const uint8_t *pair_axis;
    int n_axes, max_positions, rot, interleaved, inverse;
};

// One pass over packed rows: rotate q -> q_out, rotate k into the cache, copy v into the cache.  treewy_rope is
// the part with H_kv = 0 (no cache).
struct RowsArgs {
    CacheView c;
    RopeView r;
    const int32_t *row_offsets;  // (for treewy_rope NULL)
    const void *q, *k, *v;
    void *q_out;
    long long ld_q, ld_k, ld_v, ld_qo;
    int B, T, H_q, d;
    int32_t *status;  // per sequence, or one word for treewy_rope
};

// A norm of each head ahead of its rotation (weight NULL: none)
struct NormView {
    const void *weight;
    int bf16, plus_one;
    float eps;
};
struct NormRowsArgs {
    RowsArgs rows;
    NormView q, k;
};
struct NormBackwardArgs {
    RowsArgs rows;  // q: x, q_out: dx, no cache
    NormView norm;
    const void *dy;
    long long ld_dy;
    float *dweight, *parts;
};

struct KvCommitArgs {
    CacheView c;
    const int32_t *node_offsets;
    const uint64_t *anc_mask;
    const void *k, *v;
    long long ld_k, ld_v;
    const int32_t *accepted;
    int32_t *new_len, *seq_status;
    int B, T, max_nodes;
};

struct AttnArgs {
    CacheView c;
    const int32_t *node_offsets;
    const uint64_t *anc_mask;
    const void *q, *k, *v;
    long long ld_q, ld_k, ld_v;
    void *O;
    const int32_t *shared_pages;
    int shared_len;
    float scale;
    int log_page;           // page_size = 1 << log_page (tensor-core kernel only)
    int B, T, max_nodes, H_q, G;  // G = H_q / H_kv query heads to a key/value head
    float *ws;
    int32_t *seq_status;
    long long wait_cycles;  // limit of the bounded waits (0: the default)
    int skip_item;          // test hook: the (b * H_kv + h) whose copies are never issued, or -1
};

cudaError_t launch_rows(const RowsArgs &a, treewy_dtype_t io, cudaStream_t stream);
// No packed rows: sequences whose range claims some are flagged, and (context_len not NULL) those whose length does not fit
cudaError_t launch_no_rows(const int32_t *row_offsets, const int32_t *context_len, int B, long long capacity, int32_t *status, cudaStream_t stream);
cudaError_t launch_kv_commit(const KvCommitArgs &a, treewy_dtype_t io, cudaStream_t stream);
cudaError_t launch_attn_generic(const AttnArgs &a, treewy_dtype_t io, cudaStream_t stream);
size_t attn_generic_workspace(const AttnArgs &a);
// bf16 on the tensor cores, where it applies
bool attn_tc_applies(const AttnArgs &a, treewy_dtype_t io);
cudaError_t launch_attn_tc(const AttnArgs &a, cudaStream_t stream);
size_t attn_tc_workspace(const AttnArgs &a);


// New rows over the cache (treewy_attn_chunk): row i of sequence b is its token context_len[b] + i
struct ChunkArgs {
    CacheView c;
    const int32_t *row_offsets;
    const void *q;
    long long ld_q;
    void *O;
    float scale;
    int window, sinks;      // window 0x7fffffff: all
    int log_page;           // page_size = 1 << log_page (tensor-core kernel only)
    int B, T, H_q, G;
    float *ws;
    int32_t *seq_status;
    long long wait_cycles;  // as in AttnArgs
    int skip_item;
};

struct PagesArgs {
    int32_t *page_table, *free_pages, *free_count;
    int n_pages, page_size, max_pages;
    int B, T;
    const int32_t *context_len, *row_offsets;  // reserve
    const int32_t *first, *end;                // release
    int32_t *positions;
    int64_t *slots;
    int32_t *seq_status;
};

cudaError_t launch_norm_rows(const NormRowsArgs &a, treewy_dtype_t io, cudaStream_t stream);
size_t norm_backward_workspace(int d);
cudaError_t launch_norm_backward(const NormBackwardArgs &a, treewy_dtype_t io, cudaStream_t stream);
cudaError_t launch_chunk_generic(const ChunkArgs &a, treewy_dtype_t io, cudaStream_t stream);
size_t chunk_generic_workspace(const ChunkArgs &a);
size_t chunk_generic_workspace_most(const ChunkArgs &a);
bool chunk_tc_applies(const ChunkArgs &a, treewy_dtype_t io);
cudaError_t launch_chunk_tc(const ChunkArgs &a, cudaStream_t stream);
size_t chunk_tc_workspace(const ChunkArgs &a);  // (grows with a.T; 0 for widths of heads without a tensor-core kernel)
cudaError_t launch_pages_reserve(const PagesArgs &a, cudaStream_t stream);
cudaError_t launch_pages_release(const PagesArgs &a, cudaStream_t stream);

// Status bits of sequence b of new rows, and its rows and length.
__device__ __forceinline__ int check_rows(const int32_t *row_offsets, const int32_t *context_len, int b, int T, long long capacity,
                                          int *lo, int *n, int *len)
{
    *lo = row_offsets[b];
    *n = row_offsets[b + 1] - *lo;
    *len = context_len[b];
    if (bad_offsets(*lo, *n, T)) return TREEWY_SEQ_BAD_OFFSETS;
    if (*len < 0 || (long long)*len + *n > capacity) return TREEWY_SEQ_BAD_LENGTH;
    return 0;
}

// Status bits of sequence b, and its rows and length: every kernel of the attention calls decides
// what to skip by this one function.  The cached part is read up to context_len, so it has to fit the table.
__device__ __forceinline__ int check_sequence(const int32_t *node_offsets, const int32_t *context_len, int b, int T,
                                              int max_nodes, long long capacity, int shared_len, int *lo, int *n,
                                              int *len)
{
    *lo = node_offsets[b];
    *n = node_offsets[b + 1] - *lo;
    *len = context_len[b];
    if (bad_offsets(*lo, *n, T)) return TREEWY_SEQ_BAD_OFFSETS;
    if (*n < 1 || *n > max_nodes) return TREEWY_SEQ_TOO_MANY_NODES;
    if (*len < shared_len || *len > capacity) return TREEWY_SEQ_BAD_LENGTH;  // (shared_len >= 0)
    return 0;
}

__device__ __forceinline__ uint64_t low_bits(int n) { return n >= 64 ? ~0ull : (1ull << n) - 1; }

}  // namespace treewy
