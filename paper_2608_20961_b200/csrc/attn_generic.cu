// treewy_attn_verify on the CUDA cores, fp32 throughout: the path of F32 inputs and of sizes the tensor-core
// kernel does not take, and its cross-check.
//
// One CTA takes 32 query rows of one (sequence, key/value head) -- a row is a node and one of the G query heads
// that read this head, so all of them share every key they load -- and one part of the keys.  It walks the
// keys in tiles of 32 with the running maximum m, sum l and output o of a softmax,
//     m' = max(m, max_j s_j),  o' = o e^{m - m'} + sum_j e^{s_j - m'} v_j,  l' likewise,
// and parts are joined by a second kernel with the same rule.  Keys are split until the grid fills the GPU:
// the calls that come here are small, and what bounds them is the length of one CTA's walk (5 trees of 3 nodes, 777 keys, 6 / 2
// heads of 64 in fp32: 19.8 us with one 32-key step to a part, 22.6 with longer parts).
// A masked weight is a negative number that the product skips, so what a row may not see is never multiplied.
#include "attn_common.cuh"

namespace treewy {
namespace {

constexpr int THREADS = 256, RB = 32, KB = 32;
constexpr int TARGET_CTAS = 592;   // four to an SM, which their shared memory allows up to heads of 128 (256: two, 100 KB each)
constexpr int MIN_KEYS = 32;       // of a part: one step
constexpr int MAX_PARTS = 64;
constexpr float MASKED = -1.f;

struct Parts {
    int parts, row_blocks;
    long long rows;  // T * H_q
};
Parts parts_of(const AttnArgs &a)
{
    Parts p;
    p.row_blocks = (int)(((long long)a.max_nodes * a.G + RB - 1) / RB);
    p.rows = (long long)a.T * a.H_q;
    const long long most = (long long)a.c.max_pages * a.c.page_size + a.max_nodes;
    const long long ctas = (long long)a.B * a.c.H_kv * p.row_blocks;
    long long n = (TARGET_CTAS + ctas - 1) / (ctas > 0 ? ctas : 1);
    if (n > most / MIN_KEYS) n = most / MIN_KEYS;
    p.parts = (int)(n < 1 ? 1 : n > MAX_PARTS ? MAX_PARTS : n);
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

// RPT: rows of a thread in the product with v, (RB / RPT) * (d / 4) <= THREADS.
template <typename T, int RPT>
__global__ void __launch_bounds__(THREADS) attn_generic_kernel(AttnArgs a, int parts, float *part_ml, float *part_o)
{
    extern __shared__ float4 smem4[];
    __shared__ float s_alpha[RB], s_m[RB], s_l[RB], s_p[RB][KB + 1];
    __shared__ uint64_t s_mask[RB];
    __shared__ long long s_at[2][KB];              // where a tile's keys are: elements into the cache, or -1 - the draft row's
    const int D4 = a.c.d / 4, LD4 = D4 + 1;  // one float4 of padding a row
    float4 *sQ = smem4, *sK = sQ + RB * LD4, *sV = sK + KB * LD4;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int part = blockIdx.x % parts, bh = blockIdx.x / parts;
    const int b = bh / a.c.H_kv, h = bh - b * a.c.H_kv;
    grid_dependency_wait();
    grid_dependency_trigger();

    int lo, n, len;
    const int bad = check_sequence(a.node_offsets, a.c.context_len, b, a.T, a.max_nodes,
                                   (long long)a.c.max_pages * a.c.page_size, a.shared_len, &lo, &n, &len);
    if (bad) {
        if (tid == 0 && part == 0 && h == 0 && blockIdx.y == 0 && a.seq_status) atomicOr(&a.seq_status[b], bad);
        return;
    }
    const int rows = n * a.G, r0 = blockIdx.y * RB;
    if (r0 >= rows) return;
    const int keys = len + n;
    const int per = ((keys + parts - 1) / parts + KB - 1) / KB * KB;
    const int k0 = (int)min((long long)keys, (long long)part * per), k1 = (int)min((long long)keys, (long long)k0 + per);
    auto page_of = [&](int j) {
        return j < a.shared_len ? a.shared_pages[j / a.c.page_size]
                                : a.c.page_table[(size_t)b * a.c.max_pages + j / a.c.page_size];
    };
    // the addresses of a tile's keys, looked up one tile ahead by one warp
    auto locate = [&](int t0, int buf) {
        const int j = t0 + lane;
        long long at = 0;
        if (j < len) {
            const int pi = j / a.c.page_size;
            at = page_of(j) * a.c.stride_page + (j - pi * a.c.page_size) * a.c.stride_slot + h * a.c.stride_head;
        } else if (j < keys) {
            at = -1 - (long long)(lo + j - len);
        }
        s_at[buf][lane] = at;
    };
    // every page of the sequence, whatever the part: a sequence with a bad page is skipped by all of them
    bool bad_page = false;
    for (long long p = tid; p * a.c.page_size < len; p += THREADS) {
        const int page = page_of((int)(p * a.c.page_size));
        bad_page |= page < 0 || page >= a.c.n_pages;
    }
    if (__syncthreads_or(bad_page)) {
        if (tid == 0 && part == 0 && h == 0 && blockIdx.y == 0 && a.seq_status)
            atomicOr(&a.seq_status[b], TREEWY_SEQ_BAD_PAGE);
        // the join skips rows whose first part says so
        if (parts > 1 && part == 0 && tid < RB && r0 + tid < rows) {
            const int node = (r0 + tid) / a.G, g = (r0 + tid) - node * a.G;
            part_ml[2 * ((long long)(lo + node) * a.H_q + h * a.G + g) + 1] = -1.f;
        }
        return;
    }

    for (int i = tid; i < RB * D4; i += THREADS) {
        const int r = i / D4, c = i - r * D4;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r0 + r < rows) {
            const int node = (r0 + r) / a.G, g = (r0 + r) - node * a.G;
            x = Ld4<T>::at(static_cast<const T *>(a.q) + (lo + node) * a.ld_q + (long long)(h * a.G + g) * a.c.d + 4 * c);
        }
        sQ[r * LD4 + c] = x;
    }
    if (tid < RB) {
        s_m[tid] = -INFINITY, s_l[tid] = 0.f;
        s_mask[tid] = r0 + tid < rows ? a.anc_mask[lo + (r0 + tid) / a.G] & low_bits(n) : 0;
    }
    if (warp == THREADS / 32 - 1 && k0 < k1) locate(k0, 0);
    float4 acc[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    const int vc = tid % D4, vg = tid / D4;         // this thread's columns and group of rows
    const bool v_on = vg < RB / RPT;

    for (int t0 = k0; t0 < k1; t0 += KB) {
        __syncthreads();  // the tiles of the step before are read; first round: q, masks, statistics are written
        const int buf = ((t0 - k0) / KB) & 1;
        for (int i = tid; i < KB * D4; i += THREADS) {
            const int r = i / D4, c = i - r * D4;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
            if (t0 + r < k1) {
                const long long at = s_at[buf][r];
                const bool cached = at >= 0;
                const T *kp = cached ? static_cast<const T *>(a.c.k) + at : static_cast<const T *>(a.k) + (-1 - at) * a.ld_k + (long long)h * a.c.d;
                const T *vp = cached ? static_cast<const T *>(a.c.v) + at : static_cast<const T *>(a.v) + (-1 - at) * a.ld_v + (long long)h * a.c.d;
                x = Ld4<T>::at(kp + 4 * c), y = Ld4<T>::at(vp + 4 * c);
            }
            sK[r * LD4 + c] = x, sV[r * LD4 + c] = y;
        }
        if (warp == THREADS / 32 - 1 && t0 + KB < k1) locate(t0 + KB, buf ^ 1);
        __syncthreads();
        {   // scores: 2 rows x 2 keys of a thread
            const int tx = tid & 15, ty = tid >> 4;
            float s00 = 0.f, s01 = 0.f, s10 = 0.f, s11 = 0.f;
            const float4 *q0 = sQ + 2 * ty * LD4, *q1 = q0 + LD4, *x0 = sK + tx * LD4, *x1 = sK + (tx + 16) * LD4;
#pragma unroll 4
            for (int c = 0; c < D4; ++c) {
                const float4 u = q0[c], w = q1[c], x = x0[c], y = x1[c];
                s00 += u.x * x.x + u.y * x.y + u.z * x.z + u.w * x.w;
                s01 += u.x * y.x + u.y * y.y + u.z * y.z + u.w * y.w;
                s10 += w.x * x.x + w.y * x.y + w.z * x.z + w.w * x.w;
                s11 += w.x * y.x + w.y * y.y + w.z * y.z + w.w * y.w;
            }
            s_p[2 * ty][tx] = s00, s_p[2 * ty][tx + 16] = s01;
            s_p[2 * ty + 1][tx] = s10, s_p[2 * ty + 1][tx + 16] = s11;
        }
        __syncthreads();
        for (int r = warp; r < RB; r += THREADS / 32) {  // softmax step of one row, lane = key
            const int j = t0 + lane;
            const bool seen = j < k1 && (j < len || ((s_mask[r] >> (j - len)) & 1));
            const float s = s_p[r][lane] * a.scale;
            float top = seen ? s : -INFINITY;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float m0 = s_m[r], m1 = fmaxf(m0, top);
            const float ref = m1 == -INFINITY ? 0.f : m1;  // nothing seen so far: no difference of infinities
            const float p = seen ? expf(s - ref) : 0.f;
            const float sum = warp_sum(p);
            s_p[r][lane] = seen ? p : MASKED;
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
            for (int j = 0; j < KB; ++j) {
                const float4 y = sV[j * LD4 + vc];
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    const float p = s_p[vg * RPT + i][j];
                    // (a NaN weight, from a NaN a row does see, has to come through: only MASKED is skipped)
                    if (!(p < 0.f)) acc[i].x += p * y.x, acc[i].y += p * y.y, acc[i].z += p * y.z, acc[i].w += p * y.w;
                }
            }
        }
    }
    __syncthreads();
    if (v_on) {
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = r0 + vg * RPT + i;
            if (r >= rows) continue;
            const int node = r / a.G, g = r - node * a.G;
            const long long row = (long long)(lo + node) * a.H_q + h * a.G + g;
            const float l = s_l[vg * RPT + i];
            float4 x = acc[i];
            if (parts == 1) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                x.x *= inv, x.y *= inv, x.z *= inv, x.w *= inv;
                Ld4<T>::put(static_cast<T *>(a.O) + row * a.c.d + 4 * vc, x);
            } else {
                const long long at = (long long)part * a.T * a.H_q + row;
                reinterpret_cast<float4 *>(part_o)[at * D4 + vc] = x;
                if (vc == 0) part_ml[2 * at] = s_m[vg * RPT + i], part_ml[2 * at + 1] = l;
            }
        }
    }
}

// Joins the parts: one warp to a row, a lane to each part's m and l.  Grid (row warps of the longest tree, B).  Latency of two
// rounds of L2 reads.
template <typename T>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs a, int parts, const float *part_ml, const float *part_o)
{
    const int b = blockIdx.y, lane = threadIdx.x & 31;
    const long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    grid_dependency_wait();
    grid_dependency_trigger();
    int lo, n, len;
    if (check_sequence(a.node_offsets, a.c.context_len, b, a.T, a.max_nodes,
                       (long long)a.c.max_pages * a.c.page_size, a.shared_len, &lo, &n, &len))
        return;
    if (r >= (long long)n * a.H_q) return;
    const long long row = (long long)lo * a.H_q + r, stride = (long long)a.T * a.H_q;
    // lane p has the weights of parts p and p + 32
    float2 ml[2];
    float m = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = lane + 32 * i;
        ml[i] = p < parts ? *reinterpret_cast<const float2 *>(part_ml + 2 * (p * stride + row)) : make_float2(-INFINITY, 0.f);
        bad |= ml[i].y < 0.f;
        if (ml[i].y != 0.f) m = fmaxf(m, ml[i].x);  // (0: this part saw nothing)
    }
    if (__any_sync(0xffffffffu, bad)) return;       // a bad page
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ref = m == -INFINITY ? 0.f : m;
    float w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = ml[i].y == 0.f ? 0.f : expf(ml[i].x - ref);
    const float l = warp_sum(w[0] * ml[0].y + w[1] * ml[1].y);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int D4 = a.c.d / 4;
    for (int c0 = 0; c0 < D4; c0 += 32) {
        const int c = c0 + lane;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int p = 0; p < parts; ++p) {
            const float f = __shfl_sync(0xffffffffu, p < 32 ? w[0] : w[1], p & 31);
            if (c >= D4 || f == 0.f) continue;      // (a part that saw nothing has left nothing either)
            const float4 y = reinterpret_cast<const float4 *>(part_o)[(p * stride + row) * D4 + c];
            x.x += f * y.x, x.y += f * y.y, x.z += f * y.z, x.w += f * y.w;
        }
        if (c < D4) Ld4<T>::put(static_cast<T *>(a.O) + row * a.c.d + 4 * c, make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
    }
}

template <typename T, int RPT> cudaError_t launch_rpt(const AttnArgs &a, const Parts &p, cudaStream_t stream)
{
    float *part_o = a.ws, *part_ml = a.ws + (p.parts > 1 ? p.parts * p.rows * a.c.d : 0);
    const int smem = (RB + 2 * KB) * (a.c.d + 4) * (int)sizeof(float);
    int dev = 0, sms = 0;
    cudaError_t e = current_device_sms(&dev, &sms);
    if (e == cudaSuccess)
        e = ensure_dynamic_smem(reinterpret_cast<const void *>(attn_generic_kernel<T, RPT>),
                                (RB + 2 * KB) * (256 + 4) * (int)sizeof(float), dev);
    if (e != cudaSuccess) return e;
    const long long x = (long long)a.B * a.c.H_kv * p.parts;
    if (x > 0x7fffffffll || p.row_blocks > 65535 || (p.parts > 1 && a.B > 65535)) return cudaErrorInvalidValue;
    e = launch_dependent(attn_generic_kernel<T, RPT>, dim3((unsigned)x, p.row_blocks), dim3(THREADS), smem, stream, a,
                         p.parts, part_ml, part_o);
    if (e != cudaSuccess || p.parts == 1) return e;
    return launch_dependent(attn_join_kernel<T>, dim3((unsigned)(((long long)a.max_nodes * a.H_q + 7) / 8), a.B), dim3(256),
                            0, stream, a, p.parts, part_ml, part_o);
}

template <typename T> cudaError_t launch_typed(const AttnArgs &a, cudaStream_t stream)
{
    const Parts p = parts_of(a);
    if (a.c.d > 128) return launch_rpt<T, 8>(a, p, stream);
    if (a.c.d > 64) return launch_rpt<T, 4>(a, p, stream);
    return launch_rpt<T, 2>(a, p, stream);
}

}  // namespace

size_t attn_generic_workspace(const AttnArgs &a)
{
    const Parts p = parts_of(a);
    return p.parts > 1 ? (size_t)p.parts * p.rows * (a.c.d + 2) * sizeof(float) : 0;
}

cudaError_t launch_attn_generic(const AttnArgs &a, treewy_dtype_t io, cudaStream_t stream)
{
    return io == TREEWY_BF16 ? launch_typed<__nv_bfloat16>(a, stream) : launch_typed<float>(a, stream);
}

}  // namespace treewy
