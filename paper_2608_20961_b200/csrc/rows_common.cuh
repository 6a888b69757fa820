// What the kernels over packed rows share: vectors of the storage type, the sequence of a row, rows of the rotary table.
#pragma once

#include "attn_common.cuh"

namespace treewy {
namespace {

template <typename T, int VE> struct Vec;
template <> struct Vec<__nv_bfloat16, 8> {
    uint4 x;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { x = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = x; }
    __device__ __forceinline__ void get(float (&f)[8]) const { widen8(x, f); }
    __device__ __forceinline__ void set(const float (&f)[8])
    {
        x = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
};
template <> struct Vec<float, 4> {
    float4 x;
    __device__ __forceinline__ void load(const float *p) { x = __ldcs(reinterpret_cast<const float4 *>(p)); }
    __device__ __forceinline__ void store(float *p) const { *reinterpret_cast<float4 *>(p) = x; }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = x.x, f[1] = x.y, f[2] = x.z, f[3] = x.w; }
    __device__ __forceinline__ void set(const float (&f)[4]) { x = make_float4(f[0], f[1], f[2], f[3]); }
};
template <typename T> struct Vec<T, 1> {
    T x;
    __device__ __forceinline__ void load(const T *p) { x = *p; }
    __device__ __forceinline__ void store(T *p) const { *p = x; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f32(x); }
    __device__ __forceinline__ void set(const float (&f)[1]) { x = from_f32<T>(f[0]); }
};

// The sequence that owns packed row t (largest b with row_offsets[b] <= t among non-decreasing offsets), found
// by a whole warp: each round narrows the range 32-fold.  Any result is checked by the caller.
__device__ __forceinline__ int find_sequence(const int32_t *offsets, int B, int t)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, n = B;
    while (n > 1) {
        const int step = (n + 31) / 32;
        const int at = lo + lane * step;
        const bool le = lane * step < n && offsets[at] <= t;
        const unsigned m = __ballot_sync(0xffffffffu, le);
        const int last = m ? 31 - __clz(m) : 0;
        n = min(step, n - last * step);
        lo += last * step;
    }
    return lo;
}

// Four (or VE) consecutive entries of a table row
template <int VE> __device__ __forceinline__ void load_row(const float *p, float (&f)[VE])
{
    if constexpr (VE == 1) {
        f[0] = *p;
    } else {
#pragma unroll
        for (int i = 0; i < VE; i += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(p + i);
            f[i] = x.x, f[i + 1] = x.y, f[i + 2] = x.z, f[i + 3] = x.w;
        }
    }
}

// Positions of token t: lane i keeps the one of axis i.  Returns (to the whole warp) whether one is out of range.
__device__ __forceinline__ bool token_position(const RowsArgs &a, int t, int turned, int *pos)
{
    const int lane = threadIdx.x & 31;
    *pos = 0;
    if (turned == 0) return false;
    bool bad = false;
    if (lane < a.r.n_axes) {
        *pos = a.r.positions[(size_t)lane * a.T + t];
        bad = *pos < 0 || *pos >= a.r.max_positions;
    }
    if (a.r.pair_axis)
        for (int p = lane; p < a.r.rot / 2; p += 32) bad |= a.r.pair_axis[p] >= a.r.n_axes;
    return __any_sync(0xffffffffu, bad);
}

// Where packed row t goes in the cache, for the whole warp: `at` elements from its start.  False: nowhere, and the row's
// sequence is flagged if it is of one.
__device__ __forceinline__ bool place_row(const RowsArgs &a, int t, bool bad_pos, long long *at)
{
    const int lane = threadIdx.x & 31;
    int bad = bad_pos ? TREEWY_SEQ_BAD_POSITION : 0, b = 0;
    if (a.c.H_kv > 0) {
        b = find_sequence(a.row_offsets, a.B, t);
        const int lo = a.row_offsets[b], hi = a.row_offsets[b + 1];
        // Ranges outside the packed rows: no row need fall into one, so the last row's warp looks at all of them.
        if (t == a.T - 1 && a.status) {
#pragma unroll 4
            for (int i = lane; i < a.B; i += 32)
                if (bad_offsets(a.row_offsets[i], a.row_offsets[i + 1] - a.row_offsets[i], a.T)) atomicOr(&a.status[i], TREEWY_SEQ_BAD_OFFSETS);
        }
        if (t < lo || t >= hi || bad_offsets(lo, hi - lo, a.T)) return false;  // a row of no sequence
        const int len = a.c.context_len[b];
        if (len < 0 || (long long)len + (hi - lo) > (long long)a.c.max_pages * a.c.page_size) {
            bad = TREEWY_SEQ_BAD_LENGTH;
        } else {
            const int slot = len + (t - lo), pi = slot / a.c.page_size;
            const int page = a.c.page_table[(size_t)b * a.c.max_pages + pi];
            if (page < 0 || page >= a.c.n_pages)
                bad |= TREEWY_SEQ_BAD_PAGE;
            else
                *at = page * a.c.stride_page + (slot - pi * a.c.page_size) * a.c.stride_slot;
        }
    }
    if (bad) {
        if (a.c.H_kv == 0 && a.row_offsets) {         // no cache: the sequence is wanted for its flag only
            b = find_sequence(a.row_offsets, a.B, t);
            if (t < a.row_offsets[b] || t >= a.row_offsets[b + 1]) return false;
        }
        if (lane == 0 && a.status) atomicOr(&a.status[b], bad);
        return false;
    }
    return true;
}

// Cosines and sines of unit u's pairs, for the whole warp (lanes whose unit does not turn get none).
template <int VE>
__device__ __forceinline__ void unit_angles(const RopeView &r, int u, bool turns, int pos, float (&cs)[VE], float (&sn)[VE])
{
    int axis[VE], p0[VE];
    bool one = true;                              // all pairs of the unit at one position: whole vectors of the table
#pragma unroll
    for (int i = 0; i < VE; ++i) axis[i] = 0;
    if (turns && r.pair_axis) {
        if constexpr (VE == 8) {                  // (rot is a multiple of 2 VE here: the axes of a unit are aligned)
            const uint2 w = *reinterpret_cast<const uint2 *>(r.pair_axis + u * VE);
#pragma unroll
            for (int i = 0; i < 8; ++i) axis[i] = ((i < 4 ? w.x : w.y) >> (8 * (i & 3))) & 255;
        } else {
#pragma unroll
            for (int i = 0; i < VE; ++i) axis[i] = r.pair_axis[u * VE + i];
        }
    }
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        p0[i] = __shfl_sync(0xffffffffu, pos, axis[i]);
        one &= axis[i] == axis[0];
    }
    if (!turns) return;
    const int half = r.rot / 2;
    if (one) {
        const float *row = r.cos_sin + (size_t)p0[0] * r.rot + u * VE;
        load_row<VE>(row, cs);
        load_row<VE>(row + half, sn);
    } else {
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const float *row = r.cos_sin + (size_t)p0[i] * r.rot + u * VE + i;
            cs[i] = row[0], sn[i] = row[half];
        }
    }
    if (r.inverse)
#pragma unroll
        for (int i = 0; i < VE; ++i) sn[i] = -sn[i];
}

// A unit's pairs turned.  split: f and g hold the pairs' first and second members; else pairs are side by side, and the 2 VE
// elements of f, then g hold pairs 0 .. VE-1 in order.
template <int VE>
__device__ __forceinline__ void turn_unit(const float (&f)[VE], const float (&g)[VE], const float (&cs)[VE], const float (&sn)[VE],
                                          bool split, float (&rf)[VE], float (&rg)[VE])
{
    if (split) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            rf[e] = f[e] * cs[e] - g[e] * sn[e];
            rg[e] = g[e] * cs[e] + f[e] * sn[e];
        }
    } else if constexpr (VE == 1) {
        rf[0] = f[0] * cs[0] - g[0] * sn[0];
        rg[0] = g[0] * cs[0] + f[0] * sn[0];
    } else {
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
            rf[e] = f[e] * cs[e / 2] - f[e + 1] * sn[e / 2];
            rf[e + 1] = f[e + 1] * cs[e / 2] + f[e] * sn[e / 2];
            rg[e] = g[e] * cs[(VE + e) / 2] - g[e + 1] * sn[(VE + e) / 2];
            rg[e + 1] = g[e + 1] * cs[(VE + e) / 2] + g[e] * sn[(VE + e) / 2];
        }
    }
}

}  // namespace
}  // namespace treewy
