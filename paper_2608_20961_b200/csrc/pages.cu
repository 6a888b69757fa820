// The page table's upkeep: pages for new rows from a stack of free ones, and back to it.
//
// Ranks decide everything: entry e of sequence b that wants a page takes the one at free_count - 1 - rank, rank = wanting
// entries before it in the order (b, e); released pages are pushed by their rank from the end, so that the same entries would
// take them again.  One CTA: sequences a thread each, then their entries in one line, cut evenly over the threads, with a
// scan of the CTA for the ranks.  A few kB are moved; what bounds it is the launch and three or four dependent reads.
#include "attn_common.cuh"

namespace treewy {
namespace {

constexpr int PT = 1024, PW = PT / 32;
constexpr int MOST = 8;              // entries of a thread at a time
constexpr int ROWS_IN_PLACE = 8192;  // rows up to which the one CTA writes positions and slots too

struct PagesShared {
    int first[PT], row0[PT];        // of each sequence of a chunk: its first entry; its first packed row
    int off[PT + 1], row_off[PT + 1];  // entries and rows of the sequences before it
    int end_rank[PT];               // wanting entries up to its last one
    int len[PT];
    int warp_sum[2][PW];
    int taken;
};

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

// the sequence (of a chunk of `n`) that element x of the line is of: the last i with off[i] <= x
__device__ __forceinline__ int owner(const int *off, int n, int x)
{
    int lo = 0, hi = n;             // off[lo] <= x < off[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void flag(int32_t *status, int b, int bits)
{
    if (status && bits) atomicOr(&status[b], bits);
}

__global__ void __launch_bounds__(PT, 1) pages_reserve_kernel(const __grid_constant__ PagesArgs a)
{
    __shared__ PagesShared sh;
    const int tid = threadIdx.x;
    grid_dependency_wait();
    grid_dependency_trigger();
    const long long capacity = (long long)a.max_pages * a.page_size;
    int count = *a.free_count;
    const int stored = count;
    if (count < 0 || count > a.n_pages) count = 0;  // (no stack to take from)
    int used = 0;                   // pages wanted by the chunks before
    if (tid == 0) sh.taken = 0;
    const bool rows_here = (a.positions || a.slots) && a.T <= ROWS_IN_PLACE;
    for (int c0 = 0; c0 < a.B; c0 += PT) {
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
            flag(a.seq_status, b, bad);
        }
        int E, R;
        const int at = block_scan(cnt, sh.warp_sum[0], &E);
        const int row_at = block_scan(rows, sh.warp_sum[1], &R);
        sh.off[tid] = at, sh.row_off[tid] = row_at, sh.end_rank[tid] = 0;
        if (tid == 0) sh.off[nb] = E, sh.row_off[nb] = R;
        __syncthreads();
        // pass 0 assigns where there is enough for every entry; else it only counts and pass 1 assigns
        const bool enough = used + (long long)E <= count;
        int wants = 0, most = 0;
        const int each = E <= PT ? 1 : E >= PT * MOST ? MOST : (E + PT - 1) / PT;
        for (int pass = 0; pass < (enough ? 1 : 2); ++pass) {
            int carry = used;
            for (int x0 = 0; x0 < E; x0 += PT * each) {
                const int x1 = x0 + tid * each, here = min(each, E - x1);  // (none: negative)
                const int i0 = here > 0 ? owner(sh.off, nb, x1) : 0;
                int page[MOST], wanted = 0;
                int i = i0;
#pragma unroll
                for (int q = 0; q < MOST; ++q) {
                    page[q] = 0;
                    if (q >= here) continue;
                    while (x1 + q >= sh.off[i + 1]) ++i;
                    page[q] = a.page_table[(size_t)(c0 + i) * a.max_pages + sh.first[i] + x1 + q - sh.off[i]];
                }
#pragma unroll
                for (int q = 0; q < MOST; ++q) wanted += page[q] < 0;
                int total;
                int rank = carry + block_scan(wanted, sh.warp_sum[0], &total);
                i = i0;
#pragma unroll
                for (int q = 0; q < MOST; ++q) {
                    if (q >= here) continue;
                    while (x1 + q >= sh.off[i + 1]) ++i;
                    const int b = c0 + i;
                    if (page[q] >= a.n_pages && pass == 0) flag(a.seq_status, b, TREEWY_SEQ_BAD_PAGE);
                    if (page[q] >= 0) continue;
                    if (pass == 0 && !enough) {
                        atomicMax(&sh.end_rank[i], rank + 1);
                    } else {
                        const int end = enough ? rank + 1 : sh.end_rank[i];
                        if (end <= count) {
                            const int p = a.free_pages[count - 1 - rank];
                            if (p >= 0 && p < a.n_pages) a.page_table[(size_t)b * a.max_pages + sh.first[i] + x1 + q - sh.off[i]] = p;
                            else flag(a.seq_status, b, TREEWY_SEQ_BAD_PAGE);
                            most = max(most, end);
                        } else {
                            flag(a.seq_status, b, TREEWY_SEQ_NO_PAGES);
                        }
                    }
                    ++rank;
                }
                carry += total;
            }
            wants = carry - used;
            __syncthreads();
        }
        if (most > 0) atomicMax(&sh.taken, most);
        used += wants;
        if (rows_here) {
            for (int x = tid; x < R; x += PT) {
                const int i = owner(sh.row_off, nb, x), j = x - sh.row_off[i], token = sh.len[i] + j;
                if (a.positions) a.positions[sh.row0[i] + j] = token;
                if (a.slots) {
                    const int e = token / a.page_size, p = a.page_table[(size_t)(c0 + i) * a.max_pages + e];
                    a.slots[sh.row0[i] + j] = p >= 0 && p < a.n_pages ? (int64_t)p * a.page_size + (token - e * a.page_size) : -1;
                }
            }
        }
        __syncthreads();
    }
    if (tid == 0 && sh.taken > 0) *a.free_count = stored - sh.taken;
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

__global__ void __launch_bounds__(PT, 1) pages_release_kernel(const __grid_constant__ PagesArgs a)
{
    __shared__ PagesShared sh;
    const int tid = threadIdx.x;
    grid_dependency_wait();
    grid_dependency_trigger();
    int count = *a.free_count;
    if (count < 0 || count > a.n_pages) count = a.n_pages;  // (no stack to push on)
    const int begin = count;
    // from the last sequence and entry to the first
    for (int c0 = 0; c0 < a.B; c0 += PT) {
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
        __syncthreads();
        const int each = E <= PT ? 1 : E >= PT * MOST ? MOST : (E + PT - 1) / PT;
        for (int x0 = 0; x0 < E; x0 += PT * each) {
            const int x1 = x0 + tid * each, here = min(each, E - x1);  // (none: negative)
            const int i0 = here > 0 ? owner(sh.off, nb, x1) : 0;
            auto entry = [&](int i, int q) { return &a.page_table[(size_t)(a.B - 1 - c0 - i) * a.max_pages + sh.first[i] - (x1 + q - sh.off[i])]; };
            int page[MOST], back = 0;
            int i = i0;
#pragma unroll
            for (int q = 0; q < MOST; ++q) {
                page[q] = -1;
                if (q >= here) continue;
                while (x1 + q >= sh.off[i + 1]) ++i;
                page[q] = *entry(i, q);
            }
#pragma unroll
            for (int q = 0; q < MOST; ++q) back += page[q] >= 0 && page[q] < a.n_pages;
            int total;
            int to = count + block_scan(back, sh.warp_sum[0], &total);
            i = i0;
#pragma unroll
            for (int q = 0; q < MOST; ++q) {
                if (q >= here) continue;
                while (x1 + q >= sh.off[i + 1]) ++i;
                if (page[q] < 0) continue;
                *entry(i, q) = -1;
                const bool is_page = page[q] < a.n_pages;
                if (is_page && to < a.n_pages) a.free_pages[to] = page[q];
                else flag(a.seq_status, a.B - 1 - c0 - i, TREEWY_SEQ_BAD_PAGE);
                to += is_page;
            }
            count = (int)min((long long)a.n_pages, (long long)count + total);
        }
        __syncthreads();
    }
    if (tid == 0 && count > begin) *a.free_count = count;
}

}  // namespace

cudaError_t launch_pages_reserve(const PagesArgs &a, cudaStream_t stream)
{
    cudaError_t e = launch_dependent(pages_reserve_kernel, dim3(1), dim3(PT), 0, stream, a);
    if (e != cudaSuccess || a.T <= ROWS_IN_PLACE || !(a.positions || a.slots)) return e;
    long long share = (4 * 148 + a.B - 1) / a.B;
    const long long most = ((long long)a.T + 255) / 256;
    share = share < 1 ? 1 : share > most ? most : share;
    return launch_dependent(pages_rows_kernel, dim3(a.B, (unsigned)share), dim3(256), 0, stream, a);
}

cudaError_t launch_pages_release(const PagesArgs &a, cudaStream_t stream)
{
    return launch_dependent(pages_release_kernel, dim3(1), dim3(PT), 0, stream, a);
}

}  // namespace treewy
