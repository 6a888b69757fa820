// The page table's upkeep: pages for new rows from a stack of free ones, and back to it.
//
// Ranks decide everything: entry e of sequence b that wants a page takes the one at free_count - 1 - rank, rank = wanting
// entries before it in the order (b, e); released pages are pushed by their rank from the end, so that the same entries would
// take them again.  Sequences a thread each, then their entries in one line, which is cut evenly over the warps of one CTA, or of a
// cluster of eight where there can be many; a warp takes 32 neighbours at a time and finds their ranks by ballots, the line's
// by a scan of the CTA and of the CTAs' sums.  A few kB to a few hundred are moved, so what bounds it is the launch and a
// chain of dependent reads (offsets, entries, stack), and with one CTA for many entries what one SM can have in flight.
// A release and a reserve of the same entries, in us, one CTA and eight: 64 entries 8.4, 11.6; 4096 11.3, 13.2; 8192 13.6, 13.2;
// 16384 21, 13.7; 65536 68, 18.9.  How many a release has the host does not know, only how many there may be: that
// call, most often for a few rejected drafts, takes eight CTAs from four times as many on.
#include "attn_common.cuh"
#include "ptx_sm100.cuh"

namespace treewy {
namespace {

constexpr int PT = 1024, PW = PT / 32;
constexpr int MOST = 8;              // entries of a lane at a time
constexpr int CLUSTER = 8;
constexpr int MANY = 8192;           // entries that one CTA is left with
constexpr int ROWS_IN_PLACE = 8192;  // rows up to which the same kernel writes positions and slots too

struct PagesShared {
    int first[PT], row0[PT];        // of each sequence of a chunk: its first entry; its first packed row
    int off[PT + 1], row_off[PT + 1];  // entries and rows of the sequences before it
    int end_rank[PT];               // wanting entries up to its last one
    int len[PT];
    int warp_sum[2][PW];
    int cta_sum[2][CLUSTER];        // of the cluster's CTAs
    int control[2][4];              // what decides how often all go round: the first CTA's word for it
    int taken;
};

using ptx::address_in;
using ptx::cluster_rank;
template <int CL> __device__ __forceinline__ void sync_all()
{
    if constexpr (CL == 1) __syncthreads();
    else ptx::cluster_sync();
}
__device__ __forceinline__ void store_in(const int *x, int rank, int v) { asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(address_in(x, rank)), "r"(v) : "memory"); }
__device__ __forceinline__ void max_in(const int *x, int rank, int v)
{
    asm volatile("red.relaxed.cluster.shared::cluster.max.s32 [%0], %1;" ::"r"(address_in(x, rank)), "r"(v) : "memory");
}

// Exclusive sum of x over the CTA's threads; *total: over all.  Two barriers; buf alternates between calls that follow each other.
__device__ __forceinline__ int block_scan(int x, int (&sums)[PW], int *total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    int s = sums[lane];             // (as many warps as lanes)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
    }
    *total = __shfl_sync(0xffffffffu, s, 31);
    const int before = __shfl_sync(0xffffffffu, s, warp == 0 ? 0 : warp - 1);
    __syncthreads();
    return incl - x + (warp == 0 ? 0 : before);
}
static_assert(PW == 32, "a lane to each warp's sum");

// Exclusive sum over the cluster's warps, in the order of the line, of x (the same in all lanes of a warp).  turn: alternates.
template <int CL> __device__ __forceinline__ int line_scan(PagesShared &sh, int x, int turn, int *total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = CL == 1 ? 0 : cluster_rank();
    if (lane == 0) sh.warp_sum[turn][warp] = x;
    __syncthreads();
    int s = sh.warp_sum[turn][lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
    }
    *total = __shfl_sync(0xffffffffu, s, 31);
    int before = __shfl_sync(0xffffffffu, s, warp == 0 ? 0 : warp - 1);
    if (warp == 0) before = 0;
    if constexpr (CL > 1) {
        if (warp == 0 && lane < CL) store_in(&sh.cta_sum[turn][rank], lane, *total);
        sync_all<CL>();
        int all = 0;
#pragma unroll
        for (int r = 0; r < CL; ++r) {
            const int y = sh.cta_sum[turn][r];
            if (r < rank) before += y;
            all += y;
        }
        *total = all;
    }
    return before;
}

// the sequence (of a chunk of `n`) that element x of the line is of: the last i >= lo with off[i] <= x
__device__ __forceinline__ int owner(const int *off, int n, int x, int lo = 0)
{
    int hi = n;                     // off[lo] <= x < off[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Entries of a line that a warp takes at a time: 32 neighbours, and as many times that as the line needs
template <int CL> __device__ __forceinline__ int times(int entries)
{
    const int most = CL * PT;
    return entries <= most ? 1 : entries >= most * MOST ? MOST : (entries + most - 1) / most;
}

__device__ __forceinline__ void flag(int32_t *status, int b, int bits)
{
    if (status && bits) atomicOr(&status[b], bits);
}

template <int CL> __global__ void __launch_bounds__(PT, 1) pages_reserve_kernel(const __grid_constant__ PagesArgs a)
{
    __shared__ PagesShared sh;
    const int tid = threadIdx.x, lane = tid & 31, rank = CL == 1 ? 0 : cluster_rank(), warp = rank * PW + (tid >> 5);  // (on the line)
    grid_dependency_wait();
    grid_dependency_trigger();
    const long long capacity = (long long)a.max_pages * a.page_size;
    if (CL > 1) sync_all<CL>();     // (all are there, before any writes to another)
    const int stored = *a.free_count;
    int used = 0;                   // pages wanted by the chunks before
    if (tid == 0) sh.taken = 0;
    const bool rows_here = (a.positions || a.slots) && a.T <= ROWS_IN_PLACE;
    int turn = 0, chunk = 0;
    for (int c0 = 0; c0 < a.B; c0 += PT, chunk ^= 1) {
        const int b = c0 + tid, nb = min(PT, a.B - c0);
        int cnt = 0, rows = 0, bad = 0;
        if (b < a.B) {
            int lo, n, len;
            bad = check_rows(a.row_offsets, a.context_len, b, a.T, capacity, &lo, &n, &len);
            if (!bad) {
                rows = n, sh.len[tid] = len, sh.row0[tid] = lo;
                const int e0 = len / a.page_size;
                sh.first[tid] = e0;
                if (n > 0) cnt = (len + n - 1) / a.page_size + 1 - e0;
                if (n > 0 && len % a.page_size != 0) {  // the page in use has to be there
                    const int p = a.page_table[(size_t)b * a.max_pages + e0];
                    if (p < 0 || p >= a.n_pages) bad = TREEWY_SEQ_BAD_PAGE, cnt = 0;
                }
            }
            if (rank == 0) flag(a.seq_status, b, bad);
        }
        int E, R;
        const int at = block_scan(cnt, sh.warp_sum[0], &E);
        const int row_at = block_scan(rows, sh.warp_sum[1], &R);
        sh.off[tid] = at, sh.row_off[tid] = row_at, sh.end_rank[tid] = 0;
        if (tid == 0) sh.off[nb] = E, sh.row_off[nb] = R;
        // All CTAs have found the same, unless someone writes to the lengths meanwhile.  So that they meet at the same barriers whatever
        // happens, they go by the first one's numbers, and within their own.
        if (rank == 0 && tid < CL) store_in(&sh.control[chunk][0], tid, E), store_in(&sh.control[chunk][1], tid, stored);
        sync_all<CL>();
        const int line = sh.control[chunk][0], had = sh.control[chunk][1];
        E = min(E, line);
        const int count = had < 0 || had > a.n_pages ? 0 : had;  // (no stack to take from)
        // pass 0 assigns where there is enough for every entry; else it only counts and pass 1 assigns
        const bool enough = used + (long long)line <= count;
        int wants = 0, most = 0;
        const int each = times<CL>(line);
        for (int pass = 0; pass < (enough ? 1 : 2); ++pass) {
            int carry = used;
            for (unsigned x0 = 0; x0 < (unsigned)line; x0 += CL * PT * each, turn ^= 1) {
                int entry[MOST], page[MOST], i = 0, wanted = 0;
                unsigned ballot[MOST];
#pragma unroll
                for (int q = 0; q < MOST; ++q) {
                    entry[q] = -1, page[q] = 0;
                    const unsigned x = x0 + (warp * each + q) * 32 + lane;
                    if (q >= each || x >= (unsigned)E) continue;
                    if (q == 0 || ((int)x >= sh.off[i + 1] && (int)x >= sh.off[++i + 1])) i = owner(sh.off, nb, x, i);  // (often the next one)
                    entry[q] = (c0 + i) * a.max_pages + sh.first[i] + (int)x - sh.off[i];
                    page[q] = a.page_table[entry[q]];
                }
#pragma unroll
                for (int q = 0; q < MOST; ++q) ballot[q] = __ballot_sync(0xffffffffu, page[q] < 0), wanted += __popc(ballot[q]);
                int total;
                int first = carry + line_scan<CL>(sh, wanted, turn, &total);
#pragma unroll
                for (int q = 0; q < MOST; ++q) {
                    const int at = first + __popc(ballot[q] & ((1u << lane) - 1));
                    first += __popc(ballot[q]);
                    if (entry[q] >= 0 && page[q] >= a.n_pages && pass == 0) flag(a.seq_status, entry[q] / a.max_pages, TREEWY_SEQ_BAD_PAGE);
                    if (page[q] >= 0) continue;
                    if (enough) {
                        const int p = a.free_pages[count - 1 - at];
                        if (p >= 0 && p < a.n_pages) a.page_table[entry[q]] = p;
                        else flag(a.seq_status, entry[q] / a.max_pages, TREEWY_SEQ_BAD_PAGE);
                        most = max(most, at + 1);
                        continue;
                    }
                    const int b = entry[q] / a.max_pages;
                    if (pass == 0) {
#pragma unroll 1
                        for (int r = 0; r < CL; ++r) max_in(&sh.end_rank[b - c0], r, at + 1);
                        continue;
                    }
                    const int end = sh.end_rank[b - c0];
                    if (end <= count && at < end) {
                        const int p = a.free_pages[count - 1 - at];
                        if (p >= 0 && p < a.n_pages) a.page_table[entry[q]] = p;
                        else flag(a.seq_status, b, TREEWY_SEQ_BAD_PAGE);
                        most = max(most, end);
                    } else {
                        flag(a.seq_status, b, TREEWY_SEQ_NO_PAGES);
                    }
                }
                carry += total;
            }
            wants = carry - used;
            sync_all<CL>();
        }
        most = __reduce_max_sync(0xffffffffu, most);
        if (most > 0 && lane == 0) max_in(&sh.taken, 0, most);
        used += wants;
        if (rows_here) {
            for (int x = rank * PT + tid; x < R; x += CL * PT) {
                const int i = owner(sh.row_off, nb, x), j = x - sh.row_off[i], token = sh.len[i] + j;
                if (a.positions) a.positions[sh.row0[i] + j] = token;
                if (a.slots) {
                    const int e = token / a.page_size, p = __ldcg(&a.page_table[(size_t)(c0 + i) * a.max_pages + e]);  // (others' writes)
                    a.slots[sh.row0[i] + j] = p >= 0 && p < a.n_pages ? (int64_t)p * a.page_size + (token - e * a.page_size) : -1;
                }
            }
        }
        __syncthreads();
    }
    sync_all<CL>();
    if (rank == 0 && tid == 0 && sh.taken > 0) *a.free_count = stored - sh.taken;
}

// Positions and slots of many rows, once the table is complete: grid (sequences, CTAs that share one's rows).
__global__ void __launch_bounds__(256) pages_rows_kernel(const __grid_constant__ PagesArgs a)
{
    grid_dependency_wait();
    grid_dependency_trigger();
    const int b = blockIdx.x;
    int lo, n, len;
    if (check_rows(a.row_offsets, a.context_len, b, a.T, (long long)a.max_pages * a.page_size, &lo, &n, &len)) return;
    for (long long j = (long long)blockIdx.y * 256 + threadIdx.x; j < n; j += (long long)gridDim.y * 256) {
        const int token = len + (int)j;
        if (a.positions) a.positions[lo + j] = token;
        if (a.slots) {
            const int e = token / a.page_size, p = a.page_table[(size_t)b * a.max_pages + e];
            a.slots[lo + j] = p >= 0 && p < a.n_pages ? (int64_t)p * a.page_size + (token - e * a.page_size) : -1;
        }
    }
}

template <int CL> __global__ void __launch_bounds__(PT, 1) pages_release_kernel(const __grid_constant__ PagesArgs a)
{
    __shared__ PagesShared sh;
    const int tid = threadIdx.x, lane = tid & 31, rank = CL == 1 ? 0 : cluster_rank(), warp = rank * PW + (tid >> 5);  // (on the line)
    grid_dependency_wait();
    grid_dependency_trigger();
    if (CL > 1) sync_all<CL>();     // (all are there, before any writes to another)
    const int stored = *a.free_count;
    long long count = stored, begin = stored;
    // from the last sequence and entry to the first
    int turn = 0, chunk = 0;
    for (int c0 = 0; c0 < a.B; c0 += PT, chunk ^= 1) {
        const int nb = min(PT, a.B - c0), b = a.B - 1 - c0 - tid;
        int cnt = 0;
        if (tid < nb) {
            const int lo = max(a.first[b], 0);
            const int e0 = (int)(((long long)lo + a.page_size - 1) / a.page_size);
            const int e1 = min(a.end[b] / a.page_size, a.max_pages);  // (a negative end rounds to 0 or below)
            sh.first[tid] = e1 - 1;
            cnt = max(e1 - e0, 0);
        }
        int E;
        const int at = block_scan(cnt, sh.warp_sum[0], &E);
        sh.off[tid] = at;
        if (tid == 0) sh.off[nb] = E;
        // (as above: barriers by the first CTA's numbers)
        if (rank == 0 && tid < CL) store_in(&sh.control[chunk][0], tid, E), store_in(&sh.control[chunk][1], tid, stored);
        sync_all<CL>();
        const int line = sh.control[chunk][0], each = times<CL>(line);
        E = min(E, line);
        if (c0 == 0) {
            const int had = sh.control[0][1];
            begin = count = had < 0 || had > a.n_pages ? a.n_pages : had;  // (no stack to push on)
        }
        for (unsigned x0 = 0; x0 < (unsigned)line; x0 += CL * PT * each, turn ^= 1) {
            int entry[MOST], page[MOST], i = 0, back = 0;
            unsigned ballot[MOST];
#pragma unroll
            for (int q = 0; q < MOST; ++q) {
                entry[q] = -1, page[q] = -1;
                const unsigned x = x0 + (warp * each + q) * 32 + lane;
                if (q >= each || x >= (unsigned)E) continue;
                if (q == 0 || ((int)x >= sh.off[i + 1] && (int)x >= sh.off[++i + 1])) i = owner(sh.off, nb, x, i);  // (often the next one)
                entry[q] = (a.B - 1 - c0 - i) * a.max_pages + sh.first[i] - ((int)x - sh.off[i]);
                page[q] = a.page_table[entry[q]];
            }
#pragma unroll
            for (int q = 0; q < MOST; ++q)
                ballot[q] = __ballot_sync(0xffffffffu, page[q] >= 0 && page[q] < a.n_pages), back += __popc(ballot[q]);
            int total;
            long long first = count + line_scan<CL>(sh, back, turn, &total);
#pragma unroll
            for (int q = 0; q < MOST; ++q) {
                const long long to = first + __popc(ballot[q] & ((1u << lane) - 1));
                first += __popc(ballot[q]);
                if (page[q] < 0) continue;
                a.page_table[entry[q]] = -1;
                if (page[q] < a.n_pages && to < a.n_pages) a.free_pages[to] = page[q];
                else flag(a.seq_status, entry[q] / a.max_pages, TREEWY_SEQ_BAD_PAGE);
            }
            count = min((long long)a.n_pages, count + total);
        }
        __syncthreads();
    }
    if (CL > 1) sync_all<CL>();
    if (rank == 0 && tid == 0 && count > begin) *a.free_count = (int)count;
}

// more: entries enough for eight SMs
template <typename K> cudaError_t launch_pages(K one, K eight, bool more, cudaStream_t stream, const PagesArgs &a)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(more ? CLUSTER : 1), cfg.blockDim = dim3(PT), cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CLUSTER, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr, cfg.numAttrs = more ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, more ? eight : one, a);
}

}  // namespace

cudaError_t launch_pages_reserve(const PagesArgs &a, cudaStream_t stream)
{
    const bool more = a.T / a.page_size + 2ll * a.B > MANY;
    cudaError_t e = launch_pages(pages_reserve_kernel<1>, pages_reserve_kernel<CLUSTER>, more, stream, a);
    if (e != cudaSuccess || a.T <= ROWS_IN_PLACE || !(a.positions || a.slots)) return e;
    long long share = (4 * 148 + a.B - 1) / a.B;
    const long long most = ((long long)a.T + 255) / 256;
    share = share < 1 ? 1 : share > most ? most : share;
    return launch_dependent(pages_rows_kernel, dim3(a.B, (unsigned)share), dim3(256), 0, stream, a);
}

cudaError_t launch_pages_release(const PagesArgs &a, cudaStream_t stream)
{
    return launch_pages(pages_release_kernel<1>, pages_release_kernel<CLUSTER>, (long long)a.B * a.max_pages > 4 * MANY, stream, a);
}

}  // namespace treewy
