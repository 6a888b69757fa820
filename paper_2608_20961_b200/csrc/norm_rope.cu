// Norms of heads with the rotation in the same pass, forward (packed rows, or into a paged cache) and backward.
//
// With r = 1 / sqrt(mean_c x_c^2 + eps) and R the rotation of the token's positions,
//     y = R (w x r) ;   backward, g = R^T dy:   dx = r (w g - x r mean_c(w g x r)),   dw = sum over rows and heads of g x r.
// A head is held in registers by a group of lanes (a power of two of them, so that its sums are a few exchanges), each
// with UPL units: the vectors that hold VE pairs.  As in the rotation alone a warp takes heads of one token with the same pairs
// in every lane, so cosines, sines, weights and dw's partial sums stay in registers over the heads.  Every row is read once and
// written once.  15800 rows of 16 query and 2 + 2 key and value heads of 256 into a cache take 76 us, 4.25 TB/s or 0.66 of the copy rate, with 0.55
// instructions issued a cycle: warps wait for loads, of which registers hold no more.  8199 rows of 32 heads of 128: forward alone 32 us, 4.3 TB/s, backward 45 us,
// 4.5 TB/s.  A decoding step of 64 tokens 4.4 us (3.4 without a cache): one launch and its lookups.  Loads a step ahead in the forward pass cost registers (76 -> 81-92 us), over the ends of tokens in the backward pass too (45 -> 50).
#include "ptx_sm100.cuh"
#include "rows_common.cuh"

namespace treewy {
namespace {

constexpr int NORM_WARPS = 4;
constexpr int BACKWARD_CTAS = 592;  // four to an SM; each leaves one partial sum of dw
// Few rows: one cluster, whose CTAs join their sums among themselves, instead of a second launch.  61 rows of 5 heads of 80: one call after
// another 7.5 us for 9.6, in a graph 5.2 for 4.5; at four items a warp (64 rows of 32 heads of 128) 9.1 for 4.7 in a graph, so two at most.
constexpr int CLUSTER = 8, CLUSTER_WARPS = 16, CLUSTER_ITEMS = CLUSTER * CLUSTER_WARPS * 2;
constexpr int JOIN_COLS = 32, JOIN_ROWS = 16;

// lanes of a head: units rounded up to a power of two, at most a warp
__device__ __forceinline__ int lanes_of(int units) { return units >= 32 ? 32 : units <= 1 ? 1 : 1 << (32 - __clz(units - 1)); }
__device__ __forceinline__ float group_sum(float x, int lanes)
{
    for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// Elementwise operations on VE numbers, two to an instruction: these kernels issue about as long as they wait for memory.
template <int VE> __device__ __forceinline__ void mul_each(const float (&a)[VE], const float (&b)[VE], float (&r)[VE])
{
    if constexpr (VE == 1) {
        r[0] = a[0] * b[0];
    } else {
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
            const float2 y = ptx::mul2(make_float2(a[e], a[e + 1]), make_float2(b[e], b[e + 1]));
            r[e] = y.x, r[e + 1] = y.y;
        }
    }
}
template <int VE> __device__ __forceinline__ void mul_all(const float (&a)[VE], float b, float (&r)[VE])
{
    if constexpr (VE == 1) {
        r[0] = a[0] * b;
    } else {
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
            const float2 y = ptx::mul2(make_float2(a[e], a[e + 1]), make_float2(b, b));
            r[e] = y.x, r[e + 1] = y.y;
        }
    }
}
// r = a b + c
template <int VE> __device__ __forceinline__ void fma_each(const float (&a)[VE], const float (&b)[VE], const float (&c)[VE], float (&r)[VE])
{
    if constexpr (VE == 1) {
        r[0] = fmaf(a[0], b[0], c[0]);
    } else {
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
            const float2 y = ptx::fma2(make_float2(a[e], a[e + 1]), make_float2(b[e], b[e + 1]), make_float2(c[e], c[e + 1]));
            r[e] = y.x, r[e + 1] = y.y;
        }
    }
}
template <int VE> __device__ __forceinline__ void fma_all(const float (&a)[VE], float b, const float (&c)[VE], float (&r)[VE])
{
    if constexpr (VE == 1) {
        r[0] = fmaf(a[0], b, c[0]);
    } else {
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
            const float2 y = ptx::fma2(make_float2(a[e], a[e + 1]), make_float2(b, b), make_float2(c[e], c[e + 1]));
            r[e] = y.x, r[e + 1] = y.y;
        }
    }
}
// sum of a b over the VE numbers, onto two running sums
template <int VE> __device__ __forceinline__ void dot_onto(const float (&a)[VE], const float (&b)[VE], float2 &sum)
{
    if constexpr (VE == 1) {
        sum.x = fmaf(a[0], b[0], sum.x);
    } else {
#pragma unroll
        for (int e = 0; e < VE; e += 2) sum = ptx::fma2(make_float2(a[e], a[e + 1]), make_float2(b[e], b[e + 1]), sum);
    }
}
// A unit's pairs turned in place (split pairs: two numbers to an instruction)
template <int VE> __device__ __forceinline__ void turn_pairs(float (&f)[VE], float (&g)[VE], const float (&cs)[VE], const float (&sn)[VE], bool split)
{
    float rf[VE], rg[VE];
    if (VE > 1 && split) {
        mul_each<VE>(g, cs, rg), mul_each<VE>(g, sn, rf);
        fma_each<VE>(f, sn, rg, rg), mul_each<VE>(f, cs, f);
        fma_all<VE>(rf, -1.f, f, f);
#pragma unroll
        for (int e = 0; e < VE; ++e) g[e] = rg[e];
    } else {
        turn_unit<VE>(f, g, cs, sn, split, rf, rg);
#pragma unroll
        for (int e = 0; e < VE; ++e) f[e] = rf[e], g[e] = rg[e];
    }
}
// `VE` weights from element e on
template <int VE> __device__ __forceinline__ void load_weight(const NormView &n, int e, float (&w)[VE])
{
    if (VE == 1) {
        w[0] = n.bf16 ? to_f32(static_cast<const __nv_bfloat16 *>(n.weight)[e]) : static_cast<const float *>(n.weight)[e];
    } else if (n.bf16) {  // (e is a multiple of VE)
#pragma unroll
        for (int i = 0; i < VE; i += 4) {
            const uint2 x = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(n.weight) + e + i);
            w[i] = bf16lo(x.x), w[i + 1] = bf16hi(x.x), w[i + 2] = bf16lo(x.y), w[i + 3] = bf16hi(x.y);
        }
    } else {
        load_row<VE>(static_cast<const float *>(n.weight) + e, w);
    }
    if (n.plus_one)
#pragma unroll
        for (int i = 0; i < VE; ++i) w[i] += 1.f;
}

// Grid: one warp per (token, slice of heads): heads 0 .. H_q-1 of q, then those of k, then those of v.
template <typename T, int VE, int UPL, int HU>
__global__ void __launch_bounds__(NORM_WARPS * 32, UPL == 1 ? 5 : 4) norm_rows_kernel(const __grid_constant__ NormRowsArgs na, int heads_per_slice)
{
    const RowsArgs &a = na.rows;
    const int lane = threadIdx.x & 31, t = blockIdx.x * NORM_WARPS + (threadIdx.x >> 5);
    grid_dependency_wait();
    grid_dependency_trigger();
    if (t >= a.T) return;
    const int h_begin = blockIdx.y * heads_per_slice, h_end = min(a.H_q + 2 * a.c.H_kv, h_begin + heads_per_slice);
    const int units = a.d / (2 * VE), turned = a.r.cos_sin ? a.r.rot / (2 * VE) : 0, half = a.r.rot / 2;
    const int lph = lanes_of(units), hpi = 32 / lph, hl = lane / lph, ul = lane - hl * lph;

    auto off0 = [&](int u, bool turn) { return turn && u < turned && !a.r.interleaved ? u * VE : 2 * u * VE; };
    auto off1 = [&](int u, bool turn) { return turn && u < turned && !a.r.interleaved ? half + u * VE : 2 * u * VE + VE; };
    struct Run {
        const T *src;
        int h0, h1;
    };
    auto run_of = [&](int kind) {
        const int first = kind == 0 ? 0 : a.H_q + (kind - 1) * a.c.H_kv, count = kind == 0 ? a.H_q : a.c.H_kv;
        Run r;
        r.src = kind == 0   ? static_cast<const T *>(a.q) + t * a.ld_q
                : kind == 1 ? static_cast<const T *>(a.k) + t * a.ld_k
                            : static_cast<const T *>(a.v) + t * a.ld_v;
        r.h0 = max(h_begin - first, 0), r.h1 = min(h_end - first, count);
        return r;
    };
    Vec<T, VE> x[HU][UPL], y[HU][UPL];
    auto load = [&](const Run &r, int h0, bool turn) {
#pragma unroll
        for (int i = 0; i < HU; ++i) {
            const int h = h0 + i * hpi + hl;
#pragma unroll
            for (int j = 0; j < UPL; ++j) {
                const int u = ul + j * 32;
                if (u < units && h < r.h1) x[i][j].load(r.src + h * a.d + off0(u, turn)), y[i][j].load(r.src + h * a.d + off1(u, turn));
            }
        }
    };
    // the first loads of x go out before anything that has to be looked up for the token
    int kind = 0;
    Run run = run_of(0);
    while (run.h0 >= run.h1 && kind < 2) run = run_of(++kind);
    load(run, run.h0, kind < 2);
    // and a word to L2 about the rest, more than registers have room for (15800 rows of 16 and 2 heads of 256: 81 -> 76 us)
    if (VE > 1 && lane < 3 && h_end - h_begin > hpi * HU) {
        const Run rest = run_of(lane);
        const int h0 = lane == kind ? min(rest.h0 + hpi * HU, rest.h1) : rest.h0;
        if (h0 < rest.h1) ptx::prefetch_l2(rest.src + h0 * a.d, (uint32_t)min((long long)(rest.h1 - h0) * a.d * (int)sizeof(T), 65536ll));
    }

    int pos;
    const bool bad_pos = token_position(a, t, turned, &pos);
    long long at = 0;
    if (!place_row(a, t, bad_pos, &at)) return;
    const bool split = !a.r.interleaved;
    float cs[UPL][VE], sn[UPL][VE];
    if (turned > 0)
#pragma unroll
        for (int j = 0; j < UPL; ++j) unit_angles<VE>(a.r, ul + j * 32, ul + j * 32 < turned, pos, cs[j], sn[j]);

    const float inv_d = 1.f / a.d;
    bool first = true;
#pragma unroll 1
    for (; kind < 3; ++kind) {
        run = run_of(kind);
        if (run.h0 >= run.h1) continue;
        const bool turn = kind < 2;
        const NormView &n = kind == 0 ? na.q : na.k;
        const bool normed = turn && n.weight;
        float w0[UPL][VE], w1[UPL][VE];
        if (normed)
#pragma unroll
            for (int j = 0; j < UPL; ++j) {
                const int u = ul + j * 32;
                if (u < units) load_weight<VE>(n, off0(u, true), w0[j]), load_weight<VE>(n, off1(u, true), w1[j]);
            }
        T *dst = kind == 0   ? static_cast<T *>(a.q_out) + t * a.ld_qo
                 : kind == 1 ? static_cast<T *>(a.c.k) + at
                             : static_cast<T *>(a.c.v) + at;
        const long long step = kind == 0 ? a.d : a.c.stride_head;
#pragma unroll 1
        for (int h0 = run.h0; h0 < run.h1; h0 += hpi * HU) {
            if (!first) load(run, h0, turn);
            first = false;
            float r[HU];
            if (normed) {
#pragma unroll
                for (int i = 0; i < HU; ++i) {
                    float ss = 0.f;
#pragma unroll
                    for (int j = 0; j < UPL; ++j) {
                        float f[VE], g[VE];
                        x[i][j].get(f), y[i][j].get(g);
                        float2 s = make_float2(0.f, 0.f);
                        dot_onto<VE>(f, f, s), dot_onto<VE>(g, g, s);
                        if (ul + j * 32 < units && h0 + i * hpi + hl < run.h1) ss += s.x + s.y;
                    }
                    r[i] = ss;
                }
#pragma unroll
                for (int i = 0; i < HU; ++i) r[i] = rsqrtf(group_sum(r[i], lph) * inv_d + n.eps);
            }
#pragma unroll
            for (int i = 0; i < HU; ++i) {
                const int h = h0 + i * hpi + hl;
                if (h >= run.h1) continue;
#pragma unroll
                for (int j = 0; j < UPL; ++j) {
                    const int u = ul + j * 32;
                    if (u >= units) continue;
                    if (turn) {
                        float f[VE], g[VE];
                        x[i][j].get(f), y[i][j].get(g);
                        if (normed) {
                            float wr[VE];
                            mul_all<VE>(w0[j], r[i], wr), mul_each<VE>(f, wr, f);
                            mul_all<VE>(w1[j], r[i], wr), mul_each<VE>(g, wr, g);
                        }
                        if (u < turned) turn_pairs<VE>(f, g, cs[j], sn[j], split);
                        x[i][j].set(f), y[i][j].set(g);
                    }
                    x[i][j].store(dst + h * step + off0(u, turn)), y[i][j].store(dst + h * step + off1(u, turn));
                }
            }
        }
    }
}

// Warps walk (token, slice of heads) in strides of the grid, so that the grid's size alone decides the order of dw's sums.
template <typename T, int VE, int UPL, int HU, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 16 / WARPS) norm_backward_kernel(const __grid_constant__ NormBackwardArgs na, int slices, int heads_per_slice)
{
    __shared__ float s_dw[WARPS][256];
    const RowsArgs &a = na.rows;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_dependency_trigger();
    const int units = a.d / (2 * VE), turned = a.r.cos_sin ? a.r.rot / (2 * VE) : 0, half = a.r.rot / 2;
    const int lph = lanes_of(units), hpi = 32 / lph, hl = lane / lph, ul = lane - hl * lph;
    auto off0 = [&](int u) { return u < turned && !a.r.interleaved ? u * VE : 2 * u * VE; };
    auto off1 = [&](int u) { return u < turned && !a.r.interleaved ? half + u * VE : 2 * u * VE + VE; };
    float w0[UPL][VE], w1[UPL][VE], dw0[UPL][VE], dw1[UPL][VE];
#pragma unroll
    for (int j = 0; j < UPL; ++j) {
        const int u = ul + j * 32;
        if (u < units) load_weight<VE>(na.norm, off0(u), w0[j]), load_weight<VE>(na.norm, off1(u), w1[j]);
#pragma unroll
        for (int e = 0; e < VE; ++e) dw0[j][e] = dw1[j][e] = 0.f;
    }
    const float inv_d = 1.f / a.d;
    const long long work = (long long)a.T * slices;
#pragma unroll 1
    for (long long wi = (long long)blockIdx.x * WARPS + warp; wi < work; wi += (long long)gridDim.x * WARPS) {
        const int t = (int)(wi / slices), h_begin = (int)(wi - (long long)t * slices) * heads_per_slice, h_end = min(a.H_q, h_begin + heads_per_slice);
        const T *xs = static_cast<const T *>(a.q) + t * a.ld_q, *ys = static_cast<const T *>(na.dy) + t * na.ld_dy;
        T *dst = static_cast<T *>(a.q_out) + t * a.ld_qo;
        Vec<T, VE> x0[HU][UPL], x1[HU][UPL], y0[HU][UPL], y1[HU][UPL];
        auto load = [&](int h0) {
#pragma unroll
            for (int i = 0; i < HU; ++i) {
                const int h = h0 + i * hpi + hl;
#pragma unroll
                for (int j = 0; j < UPL; ++j) {
                    const int u = ul + j * 32;
                    if (u >= units || h >= h_end) continue;
                    x0[i][j].load(xs + h * a.d + off0(u)), x1[i][j].load(xs + h * a.d + off1(u));
                    y0[i][j].load(ys + h * a.d + off0(u)), y1[i][j].load(ys + h * a.d + off1(u));
                }
            }
        };
        load(h_begin);
        int pos;
        if (token_position(a, t, turned, &pos)) {
            if (lane == 0 && a.status) atomicOr(a.status, TREEWY_SEQ_BAD_POSITION);
            continue;
        }
        const bool split = !a.r.interleaved;
        float cs[UPL][VE], sn[UPL][VE];
        if (turned > 0)
#pragma unroll
            for (int j = 0; j < UPL; ++j) unit_angles<VE>(a.r, ul + j * 32, ul + j * 32 < turned, pos, cs[j], sn[j]);
#pragma unroll 1
        for (int h0 = h_begin; h0 < h_end; h0 += hpi * HU) {
            Vec<T, VE> p0[HU][UPL], p1[HU][UPL], q0[HU][UPL], q1[HU][UPL];
#pragma unroll
            for (int i = 0; i < HU; ++i)
#pragma unroll
                for (int j = 0; j < UPL; ++j) p0[i][j] = x0[i][j], p1[i][j] = x1[i][j], q0[i][j] = y0[i][j], q1[i][j] = y1[i][j];
            if (h0 + hpi * HU < h_end) load(h0 + hpi * HU);  // (on their way while these are worked on: 8199 rows of 32 heads of 128 54 -> 45 us)
#pragma unroll
            for (int i = 0; i < HU; ++i) {
                const int h = h0 + i * hpi + hl;
                float f[UPL][VE], g[UPL][VE], gf[UPL][VE], gg[UPL][VE];
                float2 ss = make_float2(0.f, 0.f), sg = ss;
#pragma unroll
                for (int j = 0; j < UPL; ++j) {
                    const int u = ul + j * 32;
                    if (u >= units || h >= h_end) continue;
                    p0[i][j].get(f[j]), p1[i][j].get(g[j]), q0[i][j].get(gf[j]), q1[i][j].get(gg[j]);
                    if (u < turned) turn_pairs<VE>(gf[j], gg[j], cs[j], sn[j], split);
                    dot_onto<VE>(f[j], f[j], ss), dot_onto<VE>(g[j], g[j], ss);
                    float p[VE];
                    mul_each<VE>(w0[j], gf[j], p), dot_onto<VE>(p, f[j], sg);
                    mul_each<VE>(w1[j], gg[j], p), dot_onto<VE>(p, g[j], sg);
                }
                const float r = rsqrtf(group_sum(ss.x + ss.y, lph) * inv_d + na.norm.eps);
                // dx = r w g - x r^3 mean(w g x)
                const float c = -(group_sum(sg.x + sg.y, lph) * inv_d * r * r * r);
                if (h >= h_end) continue;
#pragma unroll
                for (int j = 0; j < UPL; ++j) {
                    const int u = ul + j * 32;
                    if (u >= units) continue;
                    float p[VE], q[VE];
                    // (g r, and of it dw += (g r) x and dx = w (g r) + c x)
                    mul_all<VE>(gf[j], r, gf[j]), mul_all<VE>(gg[j], r, gg[j]);
                    fma_each<VE>(gf[j], f[j], dw0[j], dw0[j]), fma_each<VE>(gg[j], g[j], dw1[j], dw1[j]);
                    mul_all<VE>(f[j], c, p), mul_all<VE>(g[j], c, q);
                    fma_each<VE>(w0[j], gf[j], p, p), fma_each<VE>(w1[j], gg[j], q, q);
                    p0[i][j].set(p), p1[i][j].set(q);
                    p0[i][j].store(dst + h * a.d + off0(u)), p1[i][j].store(dst + h * a.d + off1(u));
                }
            }
        }
    }
    // dw: the groups of a warp, the warps of a CTA, then (the join) the CTAs
#pragma unroll
    for (int j = 0; j < UPL; ++j) {
        const int u = ul + j * 32;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            for (int o = lph; o < 32; o <<= 1) {
                dw0[j][e] += __shfl_xor_sync(0xffffffffu, dw0[j][e], o);
                dw1[j][e] += __shfl_xor_sync(0xffffffffu, dw1[j][e], o);
            }
            if (hl == 0 && u < units) s_dw[warp][off0(u) + e] = dw0[j][e], s_dw[warp][off1(u) + e] = dw1[j][e];
        }
    }
    __syncthreads();
    constexpr bool IN_CLUSTER = WARPS == CLUSTER_WARPS;
    __shared__ float s_sum[IN_CLUSTER ? 256 : 1];
    for (int c = threadIdx.x; c < a.d; c += WARPS * 32) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) s += s_dw[i][c];
        if constexpr (IN_CLUSTER) s_sum[c] = s;
        else na.parts[(long long)blockIdx.x * a.d + c] = s;
    }
    if constexpr (IN_CLUSTER) {
        ptx::cluster_sync();
        const int c = blockIdx.x * (256 / CLUSTER) + threadIdx.x;  // (the grid is the cluster)
        if (threadIdx.x < 256 / CLUSTER && c < a.d) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < CLUSTER; ++i) s += ptx::load_shared_of(&s_sum[c], i);
            na.dweight[c] = s;
        }
        ptx::cluster_sync();           // (none leaves before its sums are read)
    }
}

// dw from the CTAs' partial sums: JOIN_COLS columns a CTA, JOIN_ROWS running sums of each, then a tree.
__global__ void __launch_bounds__(JOIN_COLS * JOIN_ROWS) norm_join_kernel(const float *parts, int n, int d, float *dweight)
{
    __shared__ float s[JOIN_ROWS][JOIN_COLS];
    const int tx = threadIdx.x % JOIN_COLS, ty = threadIdx.x / JOIN_COLS, c = blockIdx.x * JOIN_COLS + tx;
    grid_dependency_wait();
    grid_dependency_trigger();
    float x = 0.f;
    if (c < d)
#pragma unroll 8
        for (int i = ty; i < n; i += JOIN_ROWS) x += parts[(long long)i * d + c];
    s[ty][tx] = x;
    __syncthreads();
    for (int o = JOIN_ROWS / 2; o > 0; o >>= 1) {
        if (ty < o) s[ty][tx] += s[ty + o][tx];
        __syncthreads();
    }
    if (ty == 0 && c < d) dweight[c] = s[0][tx];
}

// Units are whole 16-byte vectors where the sizes let them (as in the rotation alone); odd sizes go pair by pair.
bool whole_units(const RowsArgs &a, int ve) { return a.d % (2 * ve) == 0 && (!a.r.cos_sin || a.r.rot % (2 * ve) == 0); }

// Heads of a warp: all of a token's where there are warps enough without, else as many as it loads at once.
struct Slices {
    int n, heads;
};
cudaError_t slices_of(int T, int heads, int step, Slices *s)
{
    int dev = 0, sms = 0;
    const cudaError_t e = current_device_sms(&dev, &sms);
    const int most = (heads + step - 1) / step;
    long long n = (long long)sms * 20 / (T > 0 ? T : 1);
    n = n < 1 ? 1 : n > most ? most : n;
    s->heads = (int)((most + n - 1) / n) * step;
    s->n = (heads + s->heads - 1) / s->heads;
    return e;
}
int heads_of_a_step(int d, int ve)
{
    int lanes = 1;
    while (lanes < 32 && lanes < d / (2 * ve)) lanes *= 2;
    return 32 / lanes;
}

template <typename T, int VE, int UPL, int HU> cudaError_t launch_rows_of(const NormRowsArgs &a, cudaStream_t stream)
{
    Slices s;
    const cudaError_t e = slices_of(a.rows.T, a.rows.H_q + 2 * a.rows.c.H_kv, heads_of_a_step(a.rows.d, VE) * HU, &s);
    if (e != cudaSuccess) return e;
    if (s.n > 65535) return cudaErrorInvalidValue;
    return launch_dependent(norm_rows_kernel<T, VE, UPL, HU>, dim3((a.rows.T + NORM_WARPS - 1) / NORM_WARPS, s.n), dim3(NORM_WARPS * 32), 0, stream, a,
                            s.heads);
}

template <typename T, int VE, int UPL, int HU> cudaError_t launch_backward_of(const NormBackwardArgs &a, cudaStream_t stream)
{
    Slices s;
    cudaError_t e = slices_of(a.rows.T, a.rows.H_q, heads_of_a_step(a.rows.d, VE) * HU, &s);
    if (e != cudaSuccess) return e;
    if ((long long)a.rows.T * s.n <= CLUSTER_ITEMS) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(CLUSTER), cfg.blockDim = dim3(CLUSTER_WARPS * 32), cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = CLUSTER, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr, cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&cfg, norm_backward_kernel<T, VE, UPL, HU, CLUSTER_WARPS>, a, s.n, s.heads);
    }
    const long long ctas = ((long long)a.rows.T * s.n + NORM_WARPS - 1) / NORM_WARPS;
    const int grid = (int)(ctas < 1 ? 1 : ctas > BACKWARD_CTAS ? BACKWARD_CTAS : ctas);
    e = launch_dependent(norm_backward_kernel<T, VE, UPL, HU, NORM_WARPS>, dim3(grid), dim3(NORM_WARPS * 32), 0, stream, a, s.n, s.heads);
    if (e != cudaSuccess) return e;
    return launch_dependent(norm_join_kernel, dim3((a.rows.d + JOIN_COLS - 1) / JOIN_COLS), dim3(JOIN_COLS * JOIN_ROWS), 0, stream, a.parts, grid,
                            a.rows.d, a.dweight);
}

}  // namespace

cudaError_t launch_norm_rows(const NormRowsArgs &a, treewy_dtype_t io, cudaStream_t stream)
{
    if (io == TREEWY_BF16)
        return whole_units(a.rows, 8) ? launch_rows_of<__nv_bfloat16, 8, 1, 2>(a, stream) : launch_rows_of<__nv_bfloat16, 1, 4, 1>(a, stream);
    return whole_units(a.rows, 4) ? launch_rows_of<float, 4, 1, 2>(a, stream) : launch_rows_of<float, 1, 4, 1>(a, stream);
}

size_t norm_backward_workspace(int d) { return (size_t)BACKWARD_CTAS * d * sizeof(float); }

cudaError_t launch_norm_backward(const NormBackwardArgs &a, treewy_dtype_t io, cudaStream_t stream)
{
    if (io == TREEWY_BF16)
        return whole_units(a.rows, 8) ? launch_backward_of<__nv_bfloat16, 8, 1, 1>(a, stream) : launch_backward_of<__nv_bfloat16, 1, 4, 1>(a, stream);
    return whole_units(a.rows, 4) ? launch_backward_of<float, 4, 1, 1>(a, stream) : launch_backward_of<float, 1, 4, 1>(a, stream);
}

}  // namespace treewy
