// Rotary positions with several axes, the append of packed rows to a paged cache, and the commit of an
// accepted path to it.  All three move every byte once and compute next to nothing: they are bound by HBM
// (a prompt) or by the latency of one launch (a decoding step).
//
// Rotation: pair p of a head turns by the angle of its own axis' position,
//     (x, y) -> (x cos - y sin, y cos + x sin),  its transpose (the backward pass) with -sin.
// A thread takes one unit: the two 16-byte vectors that hold 8 (bf16) or 4 (fp32) pairs of one head.  A
// warp takes a slice of one token's heads with the same pairs in every lane throughout, so a lane reads its
// cosines and sines once and keeps them in registers over the heads.
#include "rows_common.cuh"

namespace treewy {
namespace {

constexpr int ROWS_WARPS = 4;
constexpr int HEAD_UNROLL = 2;  // heads a lane has in flight

// VE: pairs of a unit.  Grid: one warp per (token, slice of heads).  A warp's first loads of x go out before anything
// that has to be looked up for the token (positions, then the table's rows; the sequence, then its length, then its
// page): the chains of dependent loads wait at the same time instead of one after the other (rotation of 8199 tokens x 24
// heads of 128: 32 -> 18 us together with a token's heads in one warp).  Two heads in flight and six CTAs to an SM: with the
// next step's loads held as well registers spill (26 us), one token over several warps repeats the lookups (27).  It
// measures 18.2 us there = 5.5 TB/s, 0.85 of a plain copy's rate; prompts of 5 x up to 4097 tokens into the cache 62 us = 5.1
// TB/s; 64 single tokens 4.0 us, one launch and its lookups.
template <typename T, int VE>
__global__ void __launch_bounds__(ROWS_WARPS * 32, 6) rows_kernel(const __grid_constant__ RowsArgs a, int heads_per_slice)
{
    const int lane = threadIdx.x & 31, t = blockIdx.x * ROWS_WARPS + (threadIdx.x >> 5);
    grid_dependency_wait();
    grid_dependency_trigger();
    if (t >= a.T) return;
    const int h_begin = blockIdx.y * heads_per_slice, h_end = min(a.H_q + 2 * a.c.H_kv, h_begin + heads_per_slice);
    const int units = a.d / (2 * VE);                 // of one head
    const int turned = a.r.cos_sin ? a.r.rot / (2 * VE) : 0, half = a.r.rot / 2;
    const int lph = min(units, 32), hpi = 32 / lph;   // lanes of a head, heads of a warp's step
    const int hl = lane / lph, ul = lane - hl * lph;
    const bool on = hl < hpi;

    Vec<T, VE> x[HEAD_UNROLL], y[HEAD_UNROLL];
    // a run of heads of q, k or v: the first and last of them in this slice, and where head 0 is
    struct Run {
        const T *src;
        int h0, h1;
        bool turn;
    };
    auto run_of = [&](int kind) {
        const int first = kind == 0 ? 0 : a.H_q + (kind - 1) * a.c.H_kv, count = kind == 0 ? a.H_q : a.c.H_kv;
        Run r;
        r.src = kind == 0   ? static_cast<const T *>(a.q) + t * a.ld_q
                : kind == 1 ? static_cast<const T *>(a.k) + t * a.ld_k
                            : static_cast<const T *>(a.v) + t * a.ld_v;
        r.h0 = max(h_begin - first, 0), r.h1 = min(h_end - first, count), r.turn = kind < 2;
        return r;
    };
    // the two vectors of unit u in a head: the members of a pair that is split are rot / 2 apart
    auto off0 = [&](int u, bool turn) { return turn && u < turned && !a.r.interleaved ? u * VE : 2 * u * VE; };
    auto off1 = [&](int u, bool turn) { return turn && u < turned && !a.r.interleaved ? half + u * VE : 2 * u * VE + VE; };
    auto load = [&](const Run &r, int h0, int u) {
        const T *p0 = r.src + off0(u, r.turn), *p1 = r.src + off1(u, r.turn);
#pragma unroll
        for (int i = 0; i < HEAD_UNROLL; ++i) {
            const int h = h0 + i * hpi + hl;
            if (on && u < units && h < r.h1) x[i].load(p0 + h * a.d), y[i].load(p1 + h * a.d);
        }
    };
    int kind = 0;
    Run run = run_of(0);
    while (run.h0 >= run.h1 && kind < 2) run = run_of(++kind);
    load(run, run.h0, ul);

    int pos;
    const bool bad_pos = token_position(a, t, turned, &pos);
    // where the row goes
    long long at = 0;
    if (!place_row(a, t, bad_pos, &at)) return;
    T *const kd = static_cast<T *>(a.c.k) + at, *const vd = static_cast<T *>(a.c.v) + at;

    bool first = true;
    for (int u0 = 0; u0 < units; u0 += 32) {
        const int u = u0 + ul;
        const bool turns = on && u < turned;
        float cs[VE], sn[VE];
        if (u0 < turned) unit_angles<VE>(a.r, u, turns, pos, cs, sn);
        for (int kd_ = kind; kd_ < 3; ++kd_) {
            run = run_of(kd_);
            const bool turn = turns && run.turn, split = turn && !a.r.interleaved;
            T *dst = kd_ == 0 ? static_cast<T *>(a.q_out) + t * a.ld_qo : kd_ == 1 ? kd : vd;
            const long long step = kd_ == 0 ? a.d : a.c.stride_head;
            T *d0 = dst + off0(u, run.turn), *d1 = dst + off1(u, run.turn);
            for (int h0 = run.h0; h0 < run.h1; h0 += hpi * HEAD_UNROLL) {
                if (!first) load(run, h0, u);         // (the very first ones are in)
                first = false;
#pragma unroll
                for (int i = 0; i < HEAD_UNROLL; ++i) {
                    const int h = h0 + i * hpi + hl;
                    if (!on || u >= units || h >= run.h1) continue;
                    if (turn) {
                        float f[VE], g[VE], rf[VE], rg[VE];
                        x[i].get(f), y[i].get(g);
                        turn_unit<VE>(f, g, cs, sn, split, rf, rg);
                        x[i].set(rf), y[i].set(rg);
                    }
                    x[i].store(d0 + h * step), y[i].store(d1 + h * step);
                }
            }
        }
    }
}

template <typename T, int VE> cudaError_t launch_rows_ve(const RowsArgs &a, cudaStream_t stream)
{
    const int heads = a.H_q + 2 * a.c.H_kv, units = a.d / (2 * VE);
    const int lph = units < 32 ? units : 32, hpi = 32 / lph;
    // Heads of a warp: all of a token's where there are warps enough without (a warp's lookups are as much work as some
    // twenty heads), else as many as it loads at once.
    int dev = 0, sms = 0;
    cudaError_t e = current_device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    const int step = hpi * HEAD_UNROLL, most = (heads + step - 1) / step;
    long long slices = (long long)sms * 24 / a.T;
    slices = slices < 1 ? 1 : slices > most ? most : slices;
    const int per = (int)((most + slices - 1) / slices) * step;
    const dim3 grid((a.T + ROWS_WARPS - 1) / ROWS_WARPS, (heads + per - 1) / per);
    if (grid.y > 65535) return cudaErrorInvalidValue;
    return launch_dependent(rows_kernel<T, VE>, grid, dim3(ROWS_WARPS * 32), 0, stream, a, per);
}

// Commit: one CTA per (sequence, slice of a row's bytes), one warp per path node.  Rows are copied as they are.  What bounds it
// is the launch and the way accepted node -> mask -> path -> page: 3.0 us for 64 paths of trees of 32 (heads 2 x 256), 5.8 for
// 509 chains of up to 8 (8 x 128, 17 MB).
constexpr int COMMIT_WARPS = 8;
constexpr int COMMIT_VECS = 128;  // 16-byte vectors of k (and of v) in a slice

__global__ void __launch_bounds__(COMMIT_WARPS * 32) kv_commit_kernel(KvCommitArgs a, int elem)
{
    const int b = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_wait();
    grid_dependency_trigger();
    int lo, n, len;
    const long long capacity = (long long)a.c.max_pages * a.c.page_size;
    int bad = check_sequence(a.node_offsets, a.c.context_len, b, a.T, a.max_nodes, capacity, 0, &lo, &n, &len);
    uint64_t path = 0;
    if (!bad) {
        const int acc = a.accepted[b];
        if (acc < -1 || acc >= n) bad = TREEWY_SEQ_BAD_ACCEPTED;
        else if (acc >= 0) path = a.anc_mask[lo + acc] & low_bits(n);
    }
    const int P = __popcll(path);
    if (!bad && (long long)len + P > capacity) bad = TREEWY_SEQ_BAD_LENGTH;
    bool bad_page = false;
    if (!bad && threadIdx.x < P) {
        const int page = a.c.page_table[(size_t)b * a.c.max_pages + (len + (int)threadIdx.x) / a.c.page_size];
        bad_page = page < 0 || page >= a.c.n_pages;
    }
    if (__syncthreads_or(bad_page)) bad = TREEWY_SEQ_BAD_PAGE;  // (bad is the same in every thread before this)
    if (bad) {
        if (threadIdx.x == 0 && blockIdx.y == 0 && a.seq_status) atomicOr(&a.seq_status[b], bad);
        return;
    }
    if (threadIdx.x == 0 && blockIdx.y == 0 && a.new_len) a.new_len[b] = len + P;
    const int vec_elems = 16 / elem, head_vecs = a.c.d / vec_elems, row_vecs = a.c.H_kv * head_vecs;
    const int v0 = blockIdx.y * COMMIT_VECS, v1 = min(row_vecs, v0 + COMMIT_VECS);
    for (int r = warp; r < P; r += COMMIT_WARPS) {
        const int node = nth_set_bit(path, r), slot = len + r, pi = slot / a.c.page_size;
        const long long page = a.c.page_table[(size_t)b * a.c.max_pages + pi];
        const long long at = page * a.c.stride_page + (slot - pi * a.c.page_size) * a.c.stride_slot;
        const char *ks = static_cast<const char *>(a.k) + (lo + node) * a.ld_k * elem;
        const char *vs = static_cast<const char *>(a.v) + (lo + node) * a.ld_v * elem;
        for (int i = v0 + lane; i < v1; i += 32) {
            const int h = i / head_vecs;
            const long long dst = (at + h * a.c.stride_head) * elem + (long long)(i - h * head_vecs) * 16;
            const uint4 x = *reinterpret_cast<const uint4 *>(ks + (long long)i * 16);
            const uint4 y = *reinterpret_cast<const uint4 *>(vs + (long long)i * 16);
            *reinterpret_cast<uint4 *>(static_cast<char *>(a.c.k) + dst) = x;
            *reinterpret_cast<uint4 *>(static_cast<char *>(a.c.v) + dst) = y;
        }
    }
}

__global__ void __launch_bounds__(256) no_rows_kernel(const int32_t *row_offsets, const int32_t *context_len, int B, long long capacity, int32_t *status)
{
    const int b = blockIdx.x * 256 + threadIdx.x;
    grid_dependency_wait();
    grid_dependency_trigger();
    if (b >= B) return;
    const int lo = row_offsets[b], n = row_offsets[b + 1] - lo;
    int bad = bad_offsets(lo, n, 0) ? TREEWY_SEQ_BAD_OFFSETS : 0;
    if (!bad && context_len && (context_len[b] < 0 || context_len[b] > capacity)) bad = TREEWY_SEQ_BAD_LENGTH;
    if (bad) atomicOr(&status[b], bad);
}

}  // namespace

cudaError_t launch_no_rows(const int32_t *row_offsets, const int32_t *context_len, int B, long long capacity, int32_t *status, cudaStream_t stream)
{
    return launch_dependent(no_rows_kernel, dim3((B + 255) / 256), dim3(256), 0, stream, row_offsets, context_len, B, capacity, status);
}

cudaError_t launch_rows(const RowsArgs &a, treewy_dtype_t io, cudaStream_t stream)
{
    // 16-byte units need whole vectors on both sides of every boundary (heads of d elements stay aligned then);
    // odd sizes go pair by pair
    const int ve = io == TREEWY_BF16 ? 8 : 4;
    const bool whole = a.d % (2 * ve) == 0 && (!a.r.cos_sin || a.r.rot % (2 * ve) == 0);
    if (io == TREEWY_BF16)
        return whole ? launch_rows_ve<__nv_bfloat16, 8>(a, stream) : launch_rows_ve<__nv_bfloat16, 1>(a, stream);
    return whole ? launch_rows_ve<float, 4>(a, stream) : launch_rows_ve<float, 1>(a, stream);
}

cudaError_t launch_kv_commit(const KvCommitArgs &a, treewy_dtype_t io, cudaStream_t stream)
{
    const int elem = io == TREEWY_BF16 ? 2 : 4;
    const int row_vecs = (int)((long long)a.c.H_kv * a.c.d * elem / 16);
    const dim3 grid(a.B, (row_vecs + COMMIT_VECS - 1) / COMMIT_VECS);
    return launch_dependent(kv_commit_kernel, grid, dim3(COMMIT_WARPS * 32), 0, stream, a, elem);
}

}  // namespace treewy
