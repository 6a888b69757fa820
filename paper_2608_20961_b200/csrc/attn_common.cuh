// What the kernels of the attention layers share: their argument blocks, the address of a cached
// token, and the checks of one sequence.
#pragma once

#include "../../include/treewy_attn.h"
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
cudaError_t launch_kv_commit(const KvCommitArgs &a, treewy_dtype_t io, cudaStream_t stream);
cudaError_t launch_attn_generic(const AttnArgs &a, treewy_dtype_t io, cudaStream_t stream);
size_t attn_generic_workspace(const AttnArgs &a);
// bf16 on the tensor cores, where it applies
bool attn_tc_applies(const AttnArgs &a, treewy_dtype_t io);
cudaError_t launch_attn_tc(const AttnArgs &a, cudaStream_t stream);
size_t attn_tc_workspace(const AttnArgs &a);

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
