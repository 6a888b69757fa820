// treewy_attn_chunk on the CUDA cores, fp32 throughout: the path of F32 inputs and of sizes the tensor-core kernel does
// not take, and its cross-check.
//
// A CTA takes 64 query rows (in small calls and decoding 32 or 16) of one (sequence, key/value head) -- a row is a token and one of the G query heads that
// read this head -- and one part of the keys that some of them see: the sinks, then the window of the first row up to
// the last row, as one line.  It walks them in tiles of 64 with the running maximum, sum and output of a softmax; parts
// are joined by a second kernel with the same rule.  Only tiles that some row does not see whole are masked: a masked weight is
// a negative number that the product skips, so what a row may not see is never multiplied.
// It is bound by shared memory (4 x 4 scores to a thread, four keys of a row's weights at a time), small calls by the chain of one step and
// the join: fp32, a prompt of 2048 with 32 / 8 heads of 128 2.06 ms, 17 TFLOP/s (bf16 with heads of 80 1.34 ms, 16); one token over 8192 keys 68-83 us (157 in
// blocks of 64 rows); four pieces of up to 77 rows with heads of 80 16.6-22.
#include <type_traits>

#include "attn_common.cuh"

namespace treewy {
namespace {

constexpr int THREADS = 256, RB_MOST = 64, RB_LEAST = 16, KB_MOST = 64;
constexpr int TARGET_CTAS = 296;   // two to an SM (heads of 256: one, 220 KB)
constexpr int MAX_PARTS = 32;
constexpr float MASKED = -1.f, PAGE_BAD = -1.f;

struct Parts {
    int rb, kb;              // rows of a block, keys of a step (and of a part at least)
    int parts;
    long long blocks, rows;  // row blocks under one head (at most, of ranges that do not overlap); T * H_q
};
Parts parts_of(const ChunkArgs &a, int rb, int kb)
{
    Parts p;
    p.rb = rb, p.kb = kb;
    p.blocks = (long long)a.T * a.G / rb + (a.B < a.T ? a.B : a.T);
    p.rows = (long long)a.T * a.H_q;
    long long most = (long long)a.c.max_pages * a.c.page_size;
    const long long seen = (long long)a.window + a.sinks + rb;
    if (most > seen) most = seen;
    const long long ctas = p.blocks * a.c.H_kv;
    long long n = ctas > 0 ? (TARGET_CTAS + ctas - 1) / ctas : 1;
    if (n > most / kb) n = most / kb;
    if (a.B > 65535) n = 1;            // (the join's grid has a sequence a row)
    p.parts = (int)(n < 1 ? 1 : n > MAX_PARTS ? MAX_PARTS : n);
    return p;
}
// Blocks of 64 rows, of 32 or 16 where that many are a sequence's on average (decoding); and steps of 64 keys.  Where those would leave SMs without work blocks
// of half as many rows, and steps of 32 as well if they still do: a step is shorter then (four pieces of up to 77 rows behind a window of 100, heads
// of 80: 28 us, 19.6, 16.6).
Parts parts_of(const ChunkArgs &a)
{
    const long long sequences = a.B < a.T ? a.B : a.T, rows = (long long)a.T * a.G;
    int rb = RB_MOST;
    while (rb > RB_LEAST && rows <= rb / 2 * sequences) rb /= 2;
    Parts p = parts_of(a, rb, KB_MOST);
    auto few = [&]() { return p.blocks * a.c.H_kv * p.parts < TARGET_CTAS / 2; };
    if (few() && rb > RB_LEAST) p = parts_of(a, rb / 2, KB_MOST);
    if (few()) p = parts_of(a, p.rb, KB_MOST / 2);
    return p;
}

template <typename T> struct Ld4;
template <> struct Ld4<float> {
    static __device__ __forceinline__ float4 at(const float *p) { return *reinterpret_cast<const float4 *>(p); }
    static __device__ __forceinline__ void put(float *p, float4 x) { *reinterpret_cast<float4 *>(p) = x; }
};
template <> struct Ld4<__nv_bfloat16> {
    static __device__ __forceinline__ float4 at(const __nv_bfloat16 *p)
    {
        const uint2 x = *reinterpret_cast<const uint2 *>(p);
        return make_float4(bf16lo(x.x), bf16hi(x.x), bf16lo(x.y), bf16hi(x.y));
    }
    static __device__ __forceinline__ void put(__nv_bfloat16 *p, float4 x)
    {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
    }
};

struct Where {
    int b, lo, n, len, r0;  // b = -1: no such row block
};
struct ScanShared {
    long long warp_sum[THREADS / 32];
    Where found;
};
// Row block `x` of the batch (all sequences' blocks in one line), for the whole CTA.  Sequences that are flagged have none.
// total: row blocks of all.
template <int RB> __device__ Where find_block(const ChunkArgs &a, long long x, ScanShared &sh, long long *total, bool set_flags)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long before = 0;
    __syncthreads();
    if (tid == 0) sh.found.b = -1;
    for (int c0 = 0; c0 < a.B; c0 += THREADS) {
        const int b = c0 + tid;
        int lo = 0, n = 0, len = 0;
        if (b < a.B) {
            const int st = check_rows(a.row_offsets, a.c.context_len, b, a.T, (long long)a.c.max_pages * a.c.page_size, &lo, &n, &len);
            if (st) n = 0;
            if (st && set_flags && a.seq_status) atomicOr(&a.seq_status[b], st);
        }
        const long long mine = ((long long)n * a.G + RB - 1) / RB;
        long long incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        __syncthreads();
        if (lane == 31) sh.warp_sum[warp] = incl;
        __syncthreads();
        long long at = before + incl - mine;
        for (int i = 0; i < THREADS / 32; ++i) {
            if (i < warp) at += sh.warp_sum[i];
            before += sh.warp_sum[i];
        }
        if (x >= at && x < at + mine) sh.found = {b, lo, n, len, (int)(x - at)};  // (r0: the block, not yet its first row)
    }
    __syncthreads();
    *total = before;
    return sh.found;
}

// RB: rows of a block, KB: keys of a step, RPT: rows of a thread in the product with v, (RB / RPT) * (d / 4) <= THREADS.
template <typename T, int RB, int KB, int RPT>
__global__ void __launch_bounds__(THREADS) chunk_generic_kernel(const __grid_constant__ ChunkArgs a, int parts, float *part_ml, float *part_o)
{
    constexpr int PS = KB + 4, NE = KB / 32;       // a row of weights; keys of a lane
    extern __shared__ float4 smem4[];
    __shared__ ScanShared scan;
    __shared__ float s_alpha[RB], s_m[RB], s_l[RB];
    __shared__ long long s_at[2][KB];              // where a tile's keys are: elements into the cache
    __shared__ int s_pos[2][KB];
    const int D4 = a.c.d / 4, LD4 = D4 + 1;        // one float4 of padding a row
    float4 *sQ = smem4, *sK = sQ + RB * LD4, *sV = sK + KB * LD4;
    float *sP = reinterpret_cast<float *>(sV + KB * LD4);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int part = blockIdx.y, h = blockIdx.z;
    grid_dependency_wait();
    grid_dependency_trigger();

    long long total = 0x7fffffffffffffffll;        // (known after the first look)
    for (long long x = blockIdx.x; x < total; x += gridDim.x) {
        const Where w = find_block<RB>(a, x, scan, &total, x == blockIdx.x && blockIdx.x == 0 && part == 0 && h == 0);
        if (w.b < 0) break;                        // (the same in every thread)
        const long long rows = (long long)w.n * a.G, r0 = (long long)w.r0 * RB;
        const int b = w.b, lo = w.lo, len = w.len;
        const int t_first = (int)(r0 / a.G), t_last = (int)((min(rows, r0 + RB) - 1) / a.G);
        // the line of keys: sinks, then the first row's window up to the last row
        const int p_first = len + t_first, p_last = len + t_last;
        const int from = a.window > p_first ? 0 : p_first - a.window + 1, sinks = min(a.sinks, from);
        const int keys = sinks + p_last + 1 - from;
        const int per = ((keys + parts - 1) / parts + KB - 1) / KB * KB;
        const int k0 = (int)min((long long)keys, (long long)part * per), k1 = (int)min((long long)keys, (long long)k0 + per);
        auto token_of = [&](int j) { return j < sinks ? j : from + (j - sinks); };
        const int32_t *table = a.c.page_table + (size_t)b * a.c.max_pages;
        auto locate = [&](int t0, int buf) {
            for (int i = lane; i < KB; i += 32) {
                const int j = t0 + i;
                long long at = 0;
                int pos = 0x7fffffff;              // (no row sees it)
                if (j < k1) {
                    pos = token_of(j);
                    const int pi = pos / a.c.page_size;
                    at = table[pi] * a.c.stride_page + (pos - pi * a.c.page_size) * a.c.stride_slot + h * a.c.stride_head;
                }
                s_at[buf][i] = at, s_pos[buf][i] = pos;
            }
        };
        // every page that these rows see, whatever the part
        bool bad_page = false;
        auto look = [&](int t0, int t1) {          // tokens t0 .. t1 - 1
            for (long long p = (long long)(t0 / a.c.page_size) + tid; p * a.c.page_size < t1; p += THREADS)
                bad_page |= table[p] < 0 || table[p] >= a.c.n_pages;
        };
        look(0, sinks), look(from, p_last + 1);
        if (__syncthreads_or(bad_page)) {
            if (tid == 0 && a.seq_status) atomicOr(&a.seq_status[b], TREEWY_SEQ_BAD_PAGE);
            // the join skips rows whose first part says so
            if (parts > 1 && part == 0 && tid < RB && r0 + tid < rows) {
                const long long node = (r0 + tid) / a.G, g = (r0 + tid) - node * a.G;
                part_ml[2 * ((lo + node) * a.H_q + h * a.G + g) + 1] = PAGE_BAD;
            }
            continue;
        }
        for (int i = tid; i < RB * D4; i += THREADS) {
            const int r = i / D4, c = i - r * D4;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r0 + r < rows) {
                const long long node = (r0 + r) / a.G, g = (r0 + r) - node * a.G;
                y = Ld4<T>::at(static_cast<const T *>(a.q) + (lo + node) * a.ld_q + (h * a.G + g) * a.c.d + 4 * c);
            }
            sQ[r * LD4 + c] = y;
        }
        if (tid < RB) s_m[tid] = -INFINITY, s_l[tid] = 0.f;
        if (warp == THREADS / 32 - 1 && k0 < k1) locate(k0, 0);
        float4 acc[RPT];
#pragma unroll
        for (int i = 0; i < RPT; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        const int vc = tid % D4, vg = tid / D4;     // this thread's columns and group of rows
        const bool v_on = vg < RB / RPT;

        for (int t0 = k0; t0 < k1; t0 += KB) {
            __syncthreads();  // the tiles of the step before are read; first round: q, statistics are written
            const int buf = ((t0 - k0) / KB) & 1;
            for (int i = tid; i < KB * D4; i += THREADS) {
                const int r = i / D4, c = i - r * D4;
                float4 kx = make_float4(0.f, 0.f, 0.f, 0.f), vx = kx;
                if (t0 + r < k1) {
                    const long long at = s_at[buf][r];
                    kx = Ld4<T>::at(static_cast<const T *>(a.c.k) + at + 4 * c), vx = Ld4<T>::at(static_cast<const T *>(a.c.v) + at + 4 * c);
                }
                sK[r * LD4 + c] = kx, sV[r * LD4 + c] = vx;
            }
            if (warp == THREADS / 32 - 1 && t0 + KB < k1) locate(t0 + KB, buf ^ 1);
            __syncthreads();
            {   // scores: rows ty + 16 i, keys tx + 16 j of a thread
                constexpr int RI = RB / 16;
                const int tx = tid & 15, ty = tid >> 4;
                float s[RI][KB / 16] = {};
#pragma unroll 2
                for (int c = 0; c < D4; ++c) {
                    float4 u[RI], y[KB / 16];
#pragma unroll
                    for (int i = 0; i < KB / 16; ++i) y[i] = sK[(tx + 16 * i) * LD4 + c];
#pragma unroll
                    for (int i = 0; i < RI; ++i) u[i] = sQ[(ty + 16 * i) * LD4 + c];
#pragma unroll
                    for (int i = 0; i < RI; ++i)
#pragma unroll
                        for (int j = 0; j < KB / 16; ++j) s[i][j] += u[i].x * y[j].x + u[i].y * y[j].y + u[i].z * y[j].z + u[i].w * y[j].w;
                }
#pragma unroll
                for (int i = 0; i < RI; ++i)
#pragma unroll
                    for (int j = 0; j < KB / 16; ++j) sP[(ty + 16 * i) * PS + tx + 16 * j] = s[i][j];
            }
            __syncthreads();
            // whole tiles: seen by the first row up to their end, and by the last row's window from their start
            const int x0 = token_of(t0), x1 = t0 + KB <= k1 ? token_of(t0 + KB - 1) : 0x7fffffff;
            const bool masked = x1 > p_first || !(x1 < a.sinks || (x0 >= from && p_last - x0 < a.window));
            for (int r = warp; r < RB; r += THREADS / 32) {  // softmax step of one row, lane = one key or two
                float s[NE], p[NE];
                bool seen[NE];
                const int pr = len + (int)((r0 + r) / a.G);
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    const int pos = s_pos[buf][lane + 32 * e];
                    seen[e] = !masked || (pos <= pr && (pos < a.sinks || pr - pos < a.window));
                    s[e] = sP[r * PS + lane + 32 * e] * a.scale;
                }
                float top = -INFINITY;
#pragma unroll
                for (int e = 0; e < NE; ++e) top = fmaxf(top, seen[e] ? s[e] : -INFINITY);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float m0 = s_m[r], m1 = fmaxf(m0, top);
                const float ref = m1 == -INFINITY ? 0.f : m1;  // nothing seen so far: no difference of infinities
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    p[e] = seen[e] ? expf(s[e] - ref) : 0.f;
                    sP[r * PS + lane + 32 * e] = seen[e] ? p[e] : MASKED;
                }
                const float sum = warp_sum(NE == 2 ? p[0] + p[NE - 1] : p[0]);
                if (lane == 0) {
                    const float alpha = expf(m0 - ref);
                    s_alpha[r] = alpha, s_m[r] = m1, s_l[r] = s_l[r] * alpha + sum;
                }
            }
            __syncthreads();
            if (v_on) {
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    const float al = s_alpha[vg * RPT + i];
                    acc[i].x *= al, acc[i].y *= al, acc[i].z *= al, acc[i].w *= al;
                }
                auto product = [&](auto masked_) {
#pragma unroll 1
                    for (int j = 0; j < KB; j += 4) {
                        float4 y[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = sV[(j + e) * LD4 + vc];
#pragma unroll
                        for (int i = 0; i < RPT; ++i) {
                            const float4 p4 = *reinterpret_cast<const float4 *>(sP + (vg * RPT + i) * PS + j);
                            const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                // (a NaN weight, from a NaN a row does see, has to come through: only MASKED is skipped)
                                if (!decltype(masked_)::value || !(p[e] < 0.f))
                                    acc[i].x += p[e] * y[e].x, acc[i].y += p[e] * y[e].y, acc[i].z += p[e] * y[e].z, acc[i].w += p[e] * y[e].w;
                        }
                    }
                };
                if (masked) product(std::true_type{});
                else product(std::false_type{});
            }
        }
        __syncthreads();
        if (v_on) {
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const long long r = r0 + vg * RPT + i;
                if (r >= rows) continue;
                const long long node = r / a.G, g = r - node * a.G;
                const long long row = (lo + node) * a.H_q + h * a.G + g;
                const float l = s_l[vg * RPT + i];
                float4 y = acc[i];
                if (parts == 1) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    y.x *= inv, y.y *= inv, y.z *= inv, y.w *= inv;
                    Ld4<T>::put(static_cast<T *>(a.O) + row * a.c.d + 4 * vc, y);
                } else {
                    const long long at = (long long)part * a.T * a.H_q + row;
                    reinterpret_cast<float4 *>(part_o)[at * D4 + vc] = y;
                    if (vc == 0) part_ml[2 * at] = s_m[vg * RPT + i], part_ml[2 * at + 1] = l;
                }
            }
        }
    }
}

// Joins the parts: one warp to a row, a lane to each part's m and l.  Grid (warps' shares of the longest sequence's rows, B).
template <typename T>
__global__ void __launch_bounds__(256) chunk_join_kernel(const __grid_constant__ ChunkArgs a, int parts, const float *part_ml, const float *part_o)
{
    const int b = blockIdx.y, lane = threadIdx.x & 31;
    grid_dependency_wait();
    grid_dependency_trigger();
    int lo, n, len;
    if (check_rows(a.row_offsets, a.c.context_len, b, a.T, (long long)a.c.max_pages * a.c.page_size, &lo, &n, &len)) return;
    const long long stride = (long long)a.T * a.H_q;
    for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < (long long)n * a.H_q; r += (long long)gridDim.x * 8) {
        const long long row = (long long)lo * a.H_q + r;
        const float2 ml = lane < parts ? *reinterpret_cast<const float2 *>(part_ml + 2 * (lane * stride + row)) : make_float2(-INFINITY, 0.f);
        if (__any_sync(0xffffffffu, ml.y < 0.f)) continue;  // a bad page
        float m = ml.y != 0.f ? ml.x : -INFINITY;           // (0: this part saw nothing)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float ref = m == -INFINITY ? 0.f : m;
        const float w = ml.y == 0.f ? 0.f : expf(ml.x - ref);
        const float l = warp_sum(w * ml.y), inv = l == 0.f ? 0.f : 1.f / l;
        const int D4 = a.c.d / 4;
        for (int c0 = 0; c0 < D4; c0 += 32) {
            const int c = c0 + lane;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
            for (int p = 0; p < parts; ++p) {
                const float f = __shfl_sync(0xffffffffu, w, p);
                if (c >= D4 || f == 0.f) continue;          // (a part that saw nothing has left nothing either)
                const float4 y = reinterpret_cast<const float4 *>(part_o)[(p * stride + row) * D4 + c];
                x.x += f * y.x, x.y += f * y.y, x.z += f * y.z, x.w += f * y.w;
            }
            if (c < D4) Ld4<T>::put(static_cast<T *>(a.O) + row * a.c.d + 4 * c, make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
        }
    }
}

int smem_of(int rb, int kb, int d) { return ((rb + 2 * kb) * (d + 4) + rb * (kb + 4)) * (int)sizeof(float); }

template <typename T, int RB, int KB, int RPT> cudaError_t launch_rpt(const ChunkArgs &a, const Parts &p, cudaStream_t stream)
{
    float *part_o = a.ws, *part_ml = a.ws + (p.parts > 1 ? p.parts * p.rows * a.c.d : 0);
    int dev = 0, sms = 0;
    cudaError_t e = current_device_sms(&dev, &sms);
    if (e == cudaSuccess) e = ensure_dynamic_smem(reinterpret_cast<const void *>(chunk_generic_kernel<T, RB, KB, RPT>), smem_of(RB, KB, 256), dev);
    if (e != cudaSuccess) return e;
    const long long x = p.blocks < 1 ? 1 : p.blocks > 0x7fffffffll ? 0x7fffffffll : p.blocks;
    if (a.c.H_kv > 65535) return cudaErrorInvalidValue;
    e = launch_dependent(chunk_generic_kernel<T, RB, KB, RPT>, dim3((unsigned)x, p.parts, a.c.H_kv), dim3(THREADS), smem_of(RB, KB, a.c.d), stream, a, p.parts, part_ml,
                         part_o);
    if (e != cudaSuccess || p.parts == 1) return e;
    long long join = (p.rows + 7) / 8;
    const long long share = (8 * 148 + a.B - 1) / a.B;
    if (join > share) join = share;
    return launch_dependent(chunk_join_kernel<T>, dim3((unsigned)join, a.B), dim3(256), 0, stream, a, p.parts, part_ml, part_o);
}

template <typename T> cudaError_t launch_typed(const ChunkArgs &a, cudaStream_t stream)
{
    const Parts p = parts_of(a);
    auto launch = [&](auto rb, auto kb) {
        constexpr int RB = decltype(rb)::value, KB = decltype(kb)::value;
        return a.c.d > 128 ? launch_rpt<T, RB, KB, RB / 4>(a, p, stream) : a.c.d > 64 ? launch_rpt<T, RB, KB, RB / 8>(a, p, stream) : launch_rpt<T, RB, KB, RB / 16>(a, p, stream);
    };
    auto rows = [&](auto kb) {
        return p.rb == 16 ? launch(std::integral_constant<int, 16>{}, kb) : p.rb == 32 ? launch(std::integral_constant<int, 32>{}, kb) : launch(std::integral_constant<int, 64>{}, kb);
    };
    return p.kb == KB_MOST ? rows(std::integral_constant<int, 64>{}) : rows(std::integral_constant<int, 32>{});
}

}  // namespace

size_t chunk_generic_workspace(const ChunkArgs &a)
{
    const Parts p = parts_of(a);
    return p.parts > 1 ? (size_t)p.parts * p.rows * (a.c.d + 2) * sizeof(float) : 0;
}

// What calls of up to a.T rows need.  With more than one part there are fewer than TARGET_CTAS row blocks, T H_q / RB_MOST at least, and
// parts <= TARGET_CTAS / blocks + 1: parts * rows is at most TARGET_CTAS * RB_MOST + rows (and MAX_PARTS * rows).
size_t chunk_generic_workspace_most(const ChunkArgs &a)
{
    const long long all = TARGET_CTAS * RB_MOST, rows = (long long)a.T * a.H_q < all ? (long long)a.T * a.H_q : all;
    const long long n = MAX_PARTS * rows < all + rows ? MAX_PARTS * rows : all + rows;
    return (size_t)n * (a.c.d + 2) * sizeof(float);
}

cudaError_t launch_chunk_generic(const ChunkArgs &a, treewy_dtype_t io, cudaStream_t stream)
{
    return io == TREEWY_BF16 ? launch_typed<__nv_bfloat16>(a, stream) : launch_typed<float>(a, stream);
}

}  // namespace treewy
