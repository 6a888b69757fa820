// treewy_attn_verify, bf16: draft-tree attention over a paged cache on the tensor cores.
//
// Rows.  All N nodes of a tree and the G query heads of one key/value head read the same keys, so a row of the
// contraction is a (node, query head) pair and a tile is 128 of them (decoding: the G heads of one token).  A
// prompt shared by the batch is the same with the rows of all sequences in one list.  Every key and value is then
// read from HBM once for up to 128 rows, which is what bounds the kernel: 4 D bytes a key against 4 D * 128
// operations, half of the machine's balance.
// Keys.  A sequence's cached tokens in tiles of 64, then its draft rows as one last tile.  Only that tile and the
// last cached one are masked.
// One tile:  S = Q K^T (Q in tensor memory, K as the TMA left it), the softmax step in registers, P = weights as bf16
// over S's own columns of tensor memory, O += P V (V read with its rows as the K index; O in tensor memory).
// The running maximum m moves only when a row's new maximum exceeds it by more than 8 (in log2): until then
// weights are at most 2^8 and nothing overflows, and the pass over O that a new m costs is rare after a
// row's first tiles.
//
// Work.  (sequence, head, group of row tiles) x key tiles in one line, cut into equal parts, one for each CTA: no
// CTA waits for a longer neighbour, whatever the lengths, and a single long sequence fills the GPU.  A cut
// item leaves unnormalised outputs with their m and l in the workspace; a second kernel joins them in the
// order of the keys.  When trees have more rows than a tile, `group` CTAs walk the same part with a row tile each,
// so that the second one reads the keys out of L2.
//
// Roles: two softmax warpgroups that take turns at the key tiles (the maxima travel between them, row by row),
// one thread that walks the work and copies K tiles, one that copies V tiles, one each for the MMAs of
// S = Q K^T and O += P V (a single one for both was the slowest role: its waits alone took as long as a tile).
//
// What it measures and what bounds it (floor at a plain copy's 6.5 TB/s in brackets), 32 query over 8 key/value heads of 128
// unless said: decoding 64 x up to 8192 keys 173 us [146], two chains of 5 over 65537 keys 93 us [82]: HBM, in the main
// kernel at 0.92 of the copy's rate.  32 trees of up to 32 nodes over 8192 keys, 16 over 2 heads of 256, 88 to 94 us [43]: the
// copies out of L2, which bring each tile to two CTAs at 40 bytes a cycle.  64 trees of 8 under a prompt of 4096, 69 to 75 us
// [17]: with 128 rows the copies of a tile and the softmax step, two groups in turn, are equally long; leaving out all of the
// softmax's arithmetic saves 5 us.  One sequence of 1023 keys 14 us [0.6]: latency.
#include <type_traits>

#include "attn_common.cuh"
#include "attn_phases.cuh"
#include "ptx_sm100.cuh"
#include "tma_host.cuh"

namespace treewy {
namespace {

constexpr int KT = 64;                 // keys of a tile
constexpr int MT = 128;                // rows of a tile
constexpr int MAX_CTAS = 160;
constexpr int THREADS = 384, PRODUCER_K = 8, PRODUCER_V = 9, MMA_QK = 10, MMA_PV = 11;
constexpr int ITEMS = 8;               // ring of work items between the producer and the other roles
constexpr int MAX_START = 40, MAX_TILE = 5;
// Least units of a CTA's part.  A part within an item's tiles has to hold the beginning of one of them: the joins read a block
// from every part between an item's first and its last.  (Some parts of a small batch lie in an item's start and have no
// tile; more and smaller parts still end earlier.  One sequence of 1023 keys with 4, 8, 12, 20: 14.1, 13.8, 13.6, 14.0 us.)
constexpr int MIN_UNITS = 8;
static_assert(MIN_UNITS >= MAX_TILE, "a part within an item's tiles holds the beginning of one");
// What a tile and the start of an item cost, in quarters of a tile of few rows, by the rows of the row tile.  With up to
// 32 rows one softmax warp in four works and a tile takes 0.47 us (0.53 where HBM bounds it); with 128 all of them do, and it
// takes 0.6.  A start (queries into tensor memory, the pipeline's start, the output) takes 2 us, 3.1 beside a shared prompt
// (every output is a block in fp32) and 3 to 6 with 128 rows.  (A part's time against its tiles and items, least squares over
// the 148 parts; heads of 128, pages of 16.)  Heads of 64 and 256 have other tiles and the same figures: with starts of half /
// twice as much decoding takes 148 / 136 us instead of 135 (64) and 97 / 99 instead of 97 (256), 32 trees of 32 with heads
// of 256 95 / 91 instead of 89; with tiles of 4 / 7 units above 32 rows those trees take 88 / 91.
__device__ __forceinline__ int tile_cost(long long rows) { return rows > 32 ? 5 : 4; }
__device__ __forceinline__ int start_cost(long long rows, bool shared) { return rows > 32 ? MAX_START : shared ? 30 : 20; }
constexpr float LAZY = 8.f;

template <int D> struct Cfg {
    static constexpr int NC = D / 64;                              // 64-column chunks of a row
    static constexpr int STAGE = NC * KT * 128;                    // bytes of a tile
    // Heads of 256 leave tensor memory for two S buffers only.  With the weights in S's place the Q K^T after next would
    // wait for this tile's P V; so there P goes through shared memory and S is free as soon as it has been read.
    static constexpr bool P_SMEM = D == 256;
    // Softmax: half a row of S in registers at a time, read twice (for the maximum and for the weights), or all of it, read
    // once.  Halves are half the code, which the roles' shared instruction cache rewards with heads of 128 (256 sequences of
    // 512 keys 102 us instead of 111, a shared prompt of 4096 under 64 trees 71 instead of 74); with heads of 64 the second read
    // costs more (decoding 143 us instead of 132), with 256 S would stay taken for longer (shared prompt 161 instead of 141).
    static constexpr bool HALVES = D == 128;
    static constexpr int P_BYTES = P_SMEM ? MT * KT * 2 : 0;       // of one of the two P buffers
    // K tiles and V tiles have a ring of stages each, up to 192 KB together.  K runs further ahead: V is wanted a softmax
    // step later (8 and 4 stages of 128: 92 us where 6 and 6 take 98).
    static constexpr int NK = D == 256 ? 3 : 8, NV = D == 256 ? 2 : D == 128 ? 4 : 8;
    static constexpr int NSB = D == 256 ? 2 : 4;                   // S buffers: what 512 columns leave
    static_assert(!P_SMEM || NV == NSB, "P's two buffers go around with the V stages");
    static constexpr int NQ = q_buffers(D);                        // Q buffers, and barriers that say they are filled
    static constexpr int TM_Q = D, TM_S = D + NQ * (D / 2);
};

// Where the copies put a tile, and in how many pieces.  A box is rows of one page (all of it, or 64 of it) and holds the
// chunks of its rows one after the other.  V comes so: rows are its K index, and any 16 of one page make an MMA step.  K
// needs its 8-row groups equally far apart: whole boxes one chunk at a time, or all chunks of 8 rows, whichever makes
// fewer copies.  (One thread issues them; a copy of 16 rows of 128 bytes takes the TMA 70 cycles, one of 64 rows 200: a
// tile of 64 keys with heads of 128 and pages of 16, K and V, takes about 1000 where the softmax of 128 rows takes 1100.)
template <int D, int BOX> struct Boxes {
    static constexpr int NC = D / 64, P = KT / BOX;  // boxes of a tile
    static constexpr bool K_BY_CHUNK = P * NC <= KT / 8;
    static constexpr int K_CHUNK = K_BY_CHUNK ? KT * 128 : 1024, K_GROUP = K_BY_CHUNK ? 1024 : NC * 1024;
};
struct Layout {                  // the same for the roles that read the tiles
    int k_chunk, k_group;        // bytes between K's chunks, and between its 8-row groups
    int v_rows, log_v_rows;      // rows of a V box
};

struct Item {
    int b, h, lo, n, len;       // b = -1: the shared prompt
    int row0, rows;             // this CTA's row tile: first row, rows in it
    int kt0, tiles, kts;        // first key tile here, tiles here, tiles of the whole item
    // tiles by their keys: 0 .. full-1 are whole, the draft rows are tile `draft`, any other is the cached tokens' last
    // one, with `rest` keys
    int full, draft, rest;
    // where this part's unnormalised output goes; cap 0: the item is whole and goes to O as it is
    float *blk_o, *blk_ml;
    int cap;
};
__device__ __forceinline__ int keys_of(int j, int full, int draft, int rest, int n) { return j < full ? KT : j == draft ? n : rest; }

struct Seq {
    int lo, n, len, kts, row_tiles, groups;
    int ov, wt;                 // cost of an item's start and of a tile
    unsigned per;               // of an item: ov + wt * kts
    unsigned units;             // H_kv * groups * per, below 2^31 (the launcher has checked)
};

// A CTA's part of the line of work
struct Part {
    long long u0, u1, W;        // its units, and all of the line
    int parts, group, member, R;
};

struct Shared {
    // s_full of tile g (Q K^T done: S is there, the K stage is free) goes around with the K stages, pv_done (P V done: the V
    // stage and P's place are free) with the V stages: one commit of the MMAs says both
    uint64_t k_full[8], s_full[8], v_full[8], pv_done[8], p_full[4], s_free[4], q_full[2], o_free, item_full[ITEMS], item_empty[ITEMS],
        exch[4];
    Item items[ITEMS];
    // running maximum of each row beside the number + 1 of the tile that decided it: one 64-bit word, so that a row's next
    // tile needs no barrier to know that it reads the right one
    unsigned long long m[MT];
    float l[2][2][MT];
    unsigned bad_item[16];      // ordinal + 1 of an item that met a page out of range
    unsigned nonfinite[4][2];   // draft rows of an item with NaN or infinity among their values
    long long scan[THREADS / 32], first_off, last_off;
    Seq first_seq;              // of sequence first_b
    Part part;
    int first_b, last_b;
    unsigned unfinished;        // first of this CTA's items whose output is not all stored, once a wait has run out; else ~0
    unsigned copied[2];         // tiles whose copies of K and of V were issued
    uint32_t tmem;
};

// The workspace.  A block holds unnormalised outputs of up to `cap` rows of one row tile, column groups of 4 first:
// element (row, c) at ((c / 4) * cap + row) * 4 + c % 4, so that the rows of a warp are neighbours when its threads
// write a column group each of their own row; (m, l) of the rows beside it.
struct Ws {
    int *desc;                  // [MAX_CTAS][8]: the item that a CTA's part cuts at its end
    int4 *own_at, *shared_at;   // beside a shared prompt: where each item's parts are, [B][H_kv][own_tiles], [H_kv][tiles]
    float *slot_ml, *slot_o;    // cut items: [2 * CTAs] blocks
    float *own_ml, *own_o;      // whole items beside a shared prompt: [B][H_kv][own_tiles] blocks
    float *shared_ml, *shared_o;  // the shared prompt's whole items: [H_kv][tiles] blocks of MT rows
    int slot_cap, own_cap, own_tiles, shared_tiles;
};

__device__ __forceinline__ int tiles_of(int tokens) { return (tokens + KT - 1) / KT; }

// b = -1: the shared prompt, whose rows are those of all sequences
// (What the main kernel does not do once a tile is out of line: its roles run at the same time and share the
// instruction cache.)
static __device__ __noinline__ Seq load_seq(const AttnArgs &a, int b, int R, int *status)
{
    Seq s;
    *status = 0;
    if (b < 0) {
        s.lo = 0, s.n = 0, s.len = a.shared_len, s.kts = tiles_of(a.shared_len);
        s.row_tiles = (int)(((long long)a.T * a.G + MT - 1) / MT), s.ov = start_cost((long long)a.T * a.G, true), s.wt = tile_cost((long long)a.T * a.G);
    } else {
        *status = check_sequence(a.node_offsets, a.c.context_len, b, a.T, a.max_nodes,
                                 (long long)a.c.max_pages * a.c.page_size, a.shared_len, &s.lo, &s.n, &s.len);
        if (*status) {
            s.units = 0;
            return s;
        }
        s.kts = tiles_of(s.len - a.shared_len) + 1;
        s.row_tiles = (s.n * a.G + MT - 1) / MT, s.ov = start_cost((long long)s.n * a.G, a.shared_len > 0), s.wt = tile_cost((long long)s.n * a.G);
    }
    s.groups = (s.row_tiles + R - 1) / R;
    s.per = s.ov + s.wt * s.kts;
    s.units = (unsigned)a.c.H_kv * s.groups * s.per;
    return s;
}
// (a 64-bit division takes several times as long as a 32-bit one, and nearly every line of work is short)
static __device__ __noinline__ long long div64(long long x, long long y)
{
    return ((x | y) >> 32) == 0 ? (long long)((unsigned)x / (unsigned)y) : x / y;
}
// parts: CTA groups that get work.  Part g has units g W / parts .. (g + 1) W / parts - 1.  An item takes ov + wt kts
// units and tile t begins at ov + wt t of them: it belongs to the part that this unit is in.
__device__ __forceinline__ long long part_begin(long long g, long long W, int parts) { return div64(g * W, parts); }
__device__ __forceinline__ int part_of(long long unit, long long W, int parts) { return (int)div64((unit + 1) * parts - 1, W); }
// tiles of an item that begin before unit o of it
__device__ __forceinline__ int tiles_before(int o, int ov, int wt, int kts) { return o <= ov ? 0 : min(kts, (o - ov + wt - 1) / wt); }
// Slot of part g's piece of the item that begins at `begin`: a part cuts at most two items, the one its own start
// falls into and one more.
__device__ __forceinline__ int slot_of(int g, long long begin, long long u0) { return begin <= u0 ? 2 * g : 2 * g + 1; }

// A CTA's way along its part
struct Walk {
    int b;
    unsigned off;               // in the units of sequence b
    long long u;                // on the line
    Seq s;
};
// The next item that has tiles here and rows for this member of the group; 0 tiles: the end.  An item that begins here beside a
// shared prompt leaves word of where its parts are.
template <int D> __device__ __forceinline__ void next_item(const AttnArgs &a, const Ws &ws, const Part &p, Walk &w, Item &it)
{
    int st;
    it.tiles = 0;
    while (w.u < p.u1 && it.tiles == 0) {
        if (w.off >= w.s.units) {  // (a sequence without work has no units)
            w.off = 0, ++w.b;
            w.s = load_seq(a, w.b, p.R, &st);
            continue;
        }
        const Seq &s = w.s;
        const int b = w.b;
        const unsigned i_ = w.off / s.per, o = w.off - i_ * s.per, h = i_ / s.groups, rg = i_ - h * s.groups;
        const int span = (int)min((long long)(s.per - o), p.u1 - w.u);
        const int kt0 = tiles_before(o, s.ov, s.wt, s.kts), kt1 = tiles_before(o + span, s.ov, s.wt, s.kts);
        const long long begin = w.u - o;
        const long long row0 = (long long)(rg * p.R + p.member) * MT, rows = (long long)(b < 0 ? a.T : s.n) * a.G;
        w.off += span, w.u += span;
        if (row0 >= rows) continue;
        it.b = b, it.h = h, it.lo = s.lo, it.n = s.n, it.len = s.len;
        it.row0 = (int)row0, it.rows = (int)min((long long)MT, rows - row0);
        it.kt0 = kt0, it.tiles = kt1 - kt0, it.kts = s.kts;
        const int own = b < 0 ? s.len : s.len - a.shared_len;
        it.full = own / KT - kt0, it.rest = own % KT, it.draft = b < 0 ? 0x7fffffff : s.kts - 1 - kt0;
        long long blk = 0;
        it.blk_o = it.blk_ml = nullptr, it.cap = 0;
        const bool cut = kt0 > 0 || kt1 < s.kts;
        if (cut || a.shared_len > 0) {
            const int tile = it.row0 / MT;
            const long long i = b < 0 ? (long long)h * s.row_tiles + tile : ((long long)b * a.c.H_kv + h) * ws.own_tiles + tile;
            blk = cut ? (long long)slot_of(p.group, begin, p.u0) * p.R + p.member : i;
            it.blk_o = cut ? ws.slot_o : b < 0 ? ws.shared_o : ws.own_o, it.blk_ml = cut ? ws.slot_ml : b < 0 ? ws.shared_ml : ws.own_ml;
            it.cap = cut ? ws.slot_cap : b < 0 ? MT : ws.own_cap;
            if (kt0 == 0 && kt1 > 0 && a.shared_len > 0)
                (b < 0 ? ws.shared_at : ws.own_at)[i] =
                    make_int4((int)blk, cut ? part_of(begin + s.ov + s.wt * (s.kts - 1), p.W, p.parts) - p.group + 1 : 0, p.group, 0);
        }
        it.blk_o += blk * it.cap * D, it.blk_ml += blk * it.cap * 2;
    }
}
// l of a row whose part is not there
constexpr float PAGE_BAD = -1.f, NOT_DONE = -2.f;
// After a wait that ran out: from item `unfinished` on, this CTA's blocks say that they are not there and the sequences are
// flagged (for a shared prompt's items the join does that, by the rows that want them).
template <int D> __device__ __noinline__ void mark_unfinished(const AttnArgs &a, const Ws &ws, const Part &p, Walk w, unsigned unfinished)
{
    Item it;
    for (unsigned ord = 0;; ++ord) {
        next_item<D>(a, ws, p, w, it);
        if (it.tiles == 0) return;
        if (ord < unfinished) continue;
        if (it.cap > 0 && threadIdx.x < it.rows) reinterpret_cast<float2 *>(it.blk_ml)[threadIdx.x] = make_float2(0.f, NOT_DONE);
        if (it.b >= 0 && threadIdx.x == 0 && a.seq_status) atomicOr(&a.seq_status[it.b], TREEWY_SEQ_TIMEOUT);
    }
}

__device__ __forceinline__ bool nonfinite2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// a wait with one outcome for the whole warp: what follows needs all of its lanes
__device__ __forceinline__ bool wait_warp(uint64_t *bar, uint32_t parity)
{
    return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity));
}

// The maximum that tile g left for this thread's row, once it is there; for the whole warp.
static __device__ __noinline__ bool row_max_slow(const volatile unsigned long long *p, unsigned g)
{
    for (;;) {
        if (__all_sync(0xffffffffu, (unsigned)(*p >> 32) == g + 1)) return true;
        if (__any_sync(0xffffffffu, ptx::wait_deadline_passed())) return false;
        __nanosleep(40);
    }
}
__device__ __forceinline__ bool row_max(const volatile unsigned long long *p, unsigned g, float *m)
{
    unsigned long long w = *p;
    if (!__all_sync(0xffffffffu, (unsigned)(w >> 32) == g + 1)) {
        if (!row_max_slow(p, g)) return false;
        w = *p;
    }
    *m = __uint_as_float((unsigned)w);
    return true;
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
attn_tc_kernel(const __grid_constant__ AttnArgs a, int R, const __grid_constant__ Ws ws, Layout lay, const __grid_constant__ CUtensorMap map_kc, const __grid_constant__ CUtensorMap map_vc,
               const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using C = Cfg<D>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Shared sh;
    unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char *v_stages = stages + C::NK * C::STAGE, *p_bufs = v_stages + C::NV * C::STAGE;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int group = blockIdx.x / R, member = blockIdx.x - group * R, n_groups = gridDim.x / R;

    if (tid == 0) {
        ptx::wait_deadline_init(a.wait_cycles);
#pragma unroll 1
        for (int i = 0; i < 8; ++i)
            ptx::mbar_init(&sh.k_full[i], 1), ptx::mbar_init(&sh.s_full[i], 1), ptx::mbar_init(&sh.v_full[i], 1), ptx::mbar_init(&sh.pv_done[i], 1);
        for (int i = 0; i < C::NSB; ++i)
            ptx::mbar_init(&sh.s_free[i], 4), ptx::mbar_init(&sh.p_full[i], 4);
        for (int i = 0; i < C::NQ; ++i) ptx::mbar_init(&sh.q_full[i], 8);
        ptx::mbar_init(&sh.o_free, 8);
        for (int i = 0; i < ITEMS; ++i) ptx::mbar_init(&sh.item_full[i], 1), ptx::mbar_init(&sh.item_empty[i], 11);
        for (int i = 0; i < 4; ++i) ptx::mbar_init(&sh.exch[i], 2);
        ptx::fence_barrier_init();
        sh.unfinished = ~0u;
        sh.first_b = sh.last_b = -2;
        ptx::prefetch_tmap(&map_kc), ptx::prefetch_tmap(&map_vc), ptx::prefetch_tmap(&map_k), ptx::prefetch_tmap(&map_v);
    }
    if (tid < 16) sh.bad_item[tid] = 0;
    if (tid < MT) sh.m[tid] = 0;
    if (tid < 8) sh.nonfinite[tid >> 1][tid & 1] = 0;
    if (warp == MMA_QK) {
        ptx::tmem_alloc(&sh.tmem, 512);
        ptx::tmem_relinquish();
    }
    grid_dependency_wait();
    grid_dependency_trigger();

    // ---- the line of work and this CTA's part of it
    int st;
    const long long shared_units = a.shared_len > 0 ? (long long)load_seq(a, -1, R, &st).units : 0;
    const int chunk = (a.B + THREADS - 1) / THREADS, b_begin = min(a.B, tid * chunk), b_end = min(a.B, b_begin + chunk);
    long long sum = 0;
    Seq only;                    // a thread's one sequence is not read again
#pragma unroll 1
    for (int b = b_begin; b < b_end; ++b) {
        only = load_seq(a, b, R, &st);
        sum += only.units;
        if (st && blockIdx.x == 0 && a.seq_status) atomicOr(&a.seq_status[b], st);
    }
    long long incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) sh.scan[warp] = incl;
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    long long before = shared_units, W = shared_units;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        if (i < warp) before += sh.scan[i];
        W += sh.scan[i];
    }
    before += incl - sum;
    const int parts = (int)max(1ll, min((long long)n_groups, W / MIN_UNITS));
    const long long u0 = group < parts && W > 0 ? part_begin(group, W, parts) : 0;
    const long long u1 = group < parts && W > 0 ? part_begin(group + 1, W, parts) : 0;
#pragma unroll 1
    for (int b = b_begin; b < b_end; ++b) {
        if (chunk > 1) only = load_seq(a, b, R, &st);
        const long long units = only.units;
        if (u1 > u0) {
            if (u0 >= before && u0 < before + units) sh.first_b = b, sh.first_off = u0 - before, sh.first_seq = only;
            if (u1 - 1 >= before && u1 - 1 < before + units) sh.last_b = b, sh.last_off = u1 - 1 - before;
        }
        before += units;
    }
    if (tid == 0) {
        if (u1 > u0 && u0 < shared_units) sh.first_b = -1, sh.first_off = u0, sh.first_seq = load_seq(a, -1, R, &st);
        if (u1 > u0 && u1 - 1 < shared_units) sh.last_b = -1, sh.last_off = u1 - 1;
        sh.part = {u0, u1, W, parts, group, member, R};
    }
    __syncthreads();
    const uint32_t tmem = sh.tmem;
    const float sl2 = a.scale * 1.4426950408889634f;

    if (warp == PRODUCER_K || warp == PRODUCER_V) {
        // ---------------------------------------------------------------- work items and TMA copies: one thread each
        if (ptx::elect_one()) {
            const int ps = 1 << a.log_page;
            unsigned filled = 0;    // tiles whose copies were issued
            auto mark_bad = [&](int b, unsigned ord) {
                sh.bad_item[ord % 16] = ord + 1;
                if (b >= 0 && a.seq_status) atomicOr(&a.seq_status[b], TREEWY_SEQ_BAD_PAGE);
            };
            // (returns early when a wait runs out)
            auto run = [&](auto box_, auto is_v_) {
                constexpr int BOX = decltype(box_)::value;
                constexpr bool IS_V = decltype(is_v_)::value;
                using B = Boxes<D, BOX>;
                const CUtensorMap *cache = IS_V ? &map_vc : &map_kc, *rows_map = IS_V ? &map_v : &map_k;
                constexpr int NS = IS_V ? C::NV : C::NK;
                uint64_t *fulls = IS_V ? sh.v_full : sh.k_full, *empties = IS_V ? sh.pv_done : sh.s_full;
                unsigned char *ring = IS_V ? v_stages : stages;
                Walk walk{sh.first_b, (unsigned)sh.first_off, u0, sh.first_seq};
                const Part part{u0, u1, W, parts, group, member, R};
                for (unsigned ord = 0;; ++ord) {
                    const unsigned r = ord % ITEMS;
                    Item it;
                    if constexpr (!IS_V) {
                        next_item<D>(a, ws, part, walk, it);
                        if (ord >= ITEMS && !ptx::mbar_wait(&sh.item_empty[r], (ord / ITEMS - 1) & 1)) return;
                        sh.items[r] = it;
                        ptx::mbar_arrive(&sh.item_full[r]);
                    } else {
                        if (!ptx::mbar_wait(&sh.item_full[r], (ord / ITEMS) & 1)) return;
                        it = sh.items[r];
                        if (it.tiles > 0) ptx::mbar_arrive(&sh.item_empty[r]);
                    }
                    if (it.tiles == 0) return;
                    if (it.b >= 0 && it.b * a.c.H_kv + it.h == a.skip_item) return;  // (test hook)

                    const int n = it.tiles, key0 = it.b < 0 ? 0 : a.shared_len;
                    const int *table = it.b < 0 ? a.shared_pages : a.c.page_table + (size_t)it.b * a.c.max_pages;
                    // whole tiles of cached tokens; the last of an item may be short, and then there are the draft rows
                    const int whole = it.full;
                    int pages[B::P];
                    auto load_pages = [&](int j) {
                        const int *t = table + ((key0 + (it.kt0 + j) * KT) >> a.log_page);
                        if (j < n && j < whole)
#pragma unroll
                            for (int i = 0; i < B::P; ++i) pages[i] = t[i];
                    };
                    load_pages(0);
                    bool bad = false;
                    for (int j = 0; j < n; ++j) {
                        const unsigned sidx = filled % NS;
                        const int kt = it.kt0 + j, token = key0 + kt * KT, slot0 = token & (ps - 1);
                        if (filled >= NS && !ptx::mbar_wait(&empties[sidx], (filled / NS - 1) & 1)) return;
                        ++filled;
                        unsigned char *dst = ring + sidx * C::STAGE;
                        uint64_t *full = &fulls[sidx];
                        if (j < whole) {
                            bool out = false;
#pragma unroll
                            for (int i = 0; i < B::P; ++i) out |= (unsigned)pages[i] >= (unsigned)a.c.n_pages;
                            if (out) {  // (one past the pool reads as zeros)
                                bad = true;
#pragma unroll
                                for (int i = 0; i < B::P; ++i)
                                    if ((unsigned)pages[i] >= (unsigned)a.c.n_pages) pages[i] = a.c.n_pages;
                            }
                            if (bad && !IS_V) mark_bad(it.b, ord);
                            ptx::mbar_arrive_expect_tx(full, C::STAGE);
                            if constexpr (IS_V) {
#pragma unroll
                                for (int i = 0; i < B::P; ++i)
                                    ptx::tma_load_5d(dst + i * (BOX * C::NC * 128), cache, 0, slot0, 0, it.h, pages[i], full);
                            } else if constexpr (B::K_BY_CHUNK) {
#pragma unroll
                                for (int i = 0; i < B::P; ++i)
#pragma unroll
                                    for (int c = 0; c < C::NC; ++c)
                                        ptx::tma_load_5d(dst + i * (BOX * 128) + c * B::K_CHUNK, cache, 0, slot0, c, it.h, pages[i], full);
                            } else {
#pragma unroll
                                for (int i = 0; i < KT / 8; ++i)
                                    ptx::tma_load_5d(dst + i * B::K_GROUP, cache, 0, (8 * i) % BOX, 0, it.h, pages[8 * i / BOX], full);
                            }
                        } else if (j == it.draft) {  // draft rows, 8 and one chunk at a time
                            const int groups = (it.n + 7) / 8;
                            ptx::mbar_arrive_expect_tx(full, groups * C::NC * 1024u);
#pragma unroll 1
                            for (int i = 0; i < groups; ++i) {
                                unsigned char *to = dst + (IS_V ? (8 * i / BOX) * (BOX * C::NC * 128) + (8 * i % BOX) * 128 : i * B::K_GROUP);
#pragma unroll
                                for (int c = 0; c < C::NC; ++c)
                                    ptx::tma_load_2d(to + c * (IS_V ? BOX * 128 : B::K_CHUNK), rows_map, it.h * D + c * 64, it.lo + i * 8, full);
                            }
                        } else {  // the short tile
                            constexpr int ROWS = IS_V || B::K_BY_CHUNK ? BOX : 8, COPIES = !IS_V && B::K_BY_CHUNK ? C::NC : 1;
                            const int boxes = (it.len - token + ROWS - 1) / ROWS;
                            for (int i = 0; i < boxes; ++i) bad |= (unsigned)table[(token + i * ROWS) >> a.log_page] >= (unsigned)a.c.n_pages;
                            if (bad && !IS_V) mark_bad(it.b, ord);
                            ptx::mbar_arrive_expect_tx(full, boxes * ROWS * C::NC * 128u);
#pragma unroll 1
                            for (int i = 0; i < boxes; ++i) {
                                int page = table[(token + i * ROWS) >> a.log_page];
                                if ((unsigned)page >= (unsigned)a.c.n_pages) page = a.c.n_pages;
#pragma unroll
                                for (int c = 0; c < COPIES; ++c)
                                    ptx::tma_load_5d(dst + i * (COPIES > 1 ? BOX * 128 : ROWS * C::NC * 128) + c * B::K_CHUNK, cache, 0,
                                                     (token + i * ROWS) & (ps - 1), c, it.h, page, full);
                            }
                        }
                        load_pages(j + 1);
                    }
                }
            };
            auto run_box = [&](auto box_) { return warp == PRODUCER_V ? run(box_, std::true_type{}) : run(box_, std::false_type{}); };
            if (lay.v_rows == 64) run_box(std::integral_constant<int, 64>{});
            else if (lay.v_rows == 32) run_box(std::integral_constant<int, 32>{});
            else if (lay.v_rows == 8) run_box(std::integral_constant<int, 8>{});
            else run_box(std::integral_constant<int, 16>{});
            sh.copied[warp == PRODUCER_V] = filled;
        }
        __syncwarp();
    } else if (warp == MMA_QK || warp == MMA_PV) {
        // ---------------------------------------------------------------- MMAs: one thread for Q K^T, one for P V
        if (ptx::elect_one()) {
            constexpr uint32_t idesc_qk = ptx::umma_idesc_bf16_f32(MT, KT), idesc_pv = ptx::umma_idesc_bf16_f32_bmn(MT, D);
            // Descriptors: the stage and the step only add to the address, 16 bytes a unit in the low bits.  A step of V is 16
            // rows.
            const uint64_t kd = ptx::umma_desc_k_sw128(ptx::smem_u32(stages), lay.k_group);
            const uint64_t k_hi = kd & ~0xffffffffull;
            const uint32_t k_lo = (uint32_t)kd, k_chunk = lay.k_chunk / 16;
            uint64_t v_hi = 0;
            uint32_t v_lo[KT / 16];
#pragma unroll
            for (int s = 0; s < KT / 16; ++s) {
                const uint32_t off = ((16 * s) >> lay.log_v_rows) * (lay.v_rows * C::NC * 128) + ((16 * s) & (lay.v_rows - 1)) * 128;
                const uint64_t vd = ptx::umma_desc_mn_sw128(ptx::smem_u32(v_stages) + off, lay.v_rows * 128, lay.v_rows == 8 ? C::NC * 1024 : 1024);
                v_hi = vd & ~0xffffffffull, v_lo[s] = (uint32_t)vd;
            }
            if (warp == MMA_PV && a.shared_len == 0) {  // what the join needs of the item that this part cuts at its end
                int st;
                int *d = ws.desc + 8 * blockIdx.x;
                int pieces = 0;
                if (u1 > u0) {
                    const Seq s = load_seq(a, sh.last_b, R, &st);
                    const unsigned last = (unsigned)sh.last_off, per = s.per, it = last / per;
                    const long long begin = u1 - 1 - (last - it * per);
                    const int kt0 = tiles_before((int)max(0ll, u0 - begin), s.ov, s.wt, s.kts), kt1 = tiles_before((int)(u1 - begin), s.ov, s.wt, s.kts);
                    const int row0 = ((int)(it % s.groups) * R + member) * MT;
                    if (kt0 == 0 && kt1 > 0 && kt1 < s.kts && row0 < s.n * a.G) {
                        pieces = part_of(begin + s.ov + s.wt * (s.kts - 1), W, parts) - group + 1;
                        d[1] = slot_of(group, begin, u0);
                        d[2] = s.lo, d[3] = (int)(it / s.groups), d[4] = row0, d[5] = min(MT, s.n * a.G - row0), d[6] = group;
                    }
                }
                d[0] = pieces;
            }
            uint64_t *newest = nullptr;  // barrier of the last commit, and its phase
            unsigned newest_phase = 0;
            auto wait_pv = [&](unsigned g) { return ptx::mbar_wait(&sh.pv_done[g % C::NV], (g / C::NV) & 1); };
            auto run = [&]() -> bool {
                unsigned tile = 0;  // tiles of the items before
                for (unsigned ord = 0;; ++ord) {
                    const unsigned r = ord % ITEMS;
                    if (!ptx::mbar_wait(&sh.item_full[r], (ord / ITEMS) & 1)) return false;
                    const Item it = sh.items[r];
                    if (it.tiles == 0) return true;
                    ptx::mbar_arrive(&sh.item_empty[r]);
                    const int n = it.tiles;
                    if (warp == MMA_QK) {
                        const Phase q = q_phase(ord, C::NQ);
                        if (!ptx::mbar_wait(&sh.q_full[q.barrier], q.parity)) return false;
                        for (int j = 0; j < n; ++j) {
                            const unsigned g = tile + j, sidx = g % C::NK, buf = g % C::NSB;
                            if (g >= C::NSB && !(C::P_SMEM ? ptx::mbar_wait(&sh.s_free[buf], (g / C::NSB - 1) & 1) : wait_pv(g - C::NSB))) return false;
                            if (!ptx::mbar_wait(&sh.k_full[sidx], (g / C::NK) & 1)) return false;
                            ptx::tc_fence_after_sync();
                            const uint32_t lo = k_lo + sidx * (C::STAGE / 16);
#pragma unroll
                            for (int s = 0; s < D / 16; ++s)
                                ptx::umma_bf16_ts(tmem + C::TM_S + buf * KT, tmem + C::TM_Q + (ord % C::NQ) * (D / 2) + s * 8,
                                                  k_hi | (lo + (s / 4) * k_chunk + (s % 4) * 2), idesc_qk, s > 0);
                            ptx::umma_commit(&sh.s_full[sidx]);
                            newest = &sh.s_full[sidx], newest_phase = (g / C::NK) & 1;
                        }
                    } else {
                        for (int j = 0; j < n; ++j) {
                            const unsigned g = tile + j, sidx = g % C::NV, buf = g % C::NSB;
                            if (!ptx::mbar_wait(&sh.v_full[sidx], (g / C::NV) & 1)) return false;
                            if (j == 0 && ord > 0 && !ptx::mbar_wait(&sh.o_free, (ord - 1) & 1)) return false;
                            if (!ptx::mbar_wait(&sh.p_full[buf], (g / C::NSB) & 1)) return false;
                            ptx::tc_fence_after_sync();
                            const int steps = (keys_of(j, it.full, it.draft, it.rest, it.n) + 15) / 16;
#pragma unroll
                            for (int s = 0; s < KT / 16; ++s)
                                if (s < steps) {
                                    const uint64_t vd = v_hi | (v_lo[s] + sidx * (C::STAGE / 16));
                                    if (C::P_SMEM)
                                        ptx::umma_bf16(tmem, ptx::umma_desc_k_sw128(ptx::smem_u32(p_bufs + (g & 1) * C::P_BYTES) + s * 32), vd,
                                                       idesc_pv, j > 0 || s > 0);
                                    else
                                        ptx::umma_bf16_ts(tmem, tmem + C::TM_S + buf * KT + s * 8, vd, idesc_pv, j > 0 || s > 0);
                                }
                            ptx::umma_commit(&sh.pv_done[sidx]);
                            newest = &sh.pv_done[sidx], newest_phase = (g / C::NV) & 1;
                        }
                    }
                    tile += n;
                }
            };
            if (!run() && newest)  // MMAs in flight have to end before the CTA may leave
                for (int t = 0; t < 100000 && !ptx::mbar_try_wait(newest, newest_phase); ++t) __nanosleep(20);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- softmax, epilogue
        const int wg = warp >> 2, w4 = warp & 3, row = w4 * 32 + lane;
        const uint32_t lane_base = (uint32_t)(w4 * 32) << 16;
        unsigned ord = ~0u;    // the item in work
        // An item and this thread's row of it: its packed row, its query head, the draft rows it sees
        struct Mine {
            const Item *it;  // (stays in its slot of the ring until this warp says that it is done)
            int t, hq;
            uint64_t tree;
        };
        // Takes over item `nr`: finds this thread's row and brings its half of the row's query into tensor memory.
        auto take = [&](unsigned nr, Mine &x) -> bool {
            if (!wait_warp(&sh.item_full[nr % ITEMS], (nr / ITEMS) & 1)) return false;
            const Item &it = sh.items[nr % ITEMS];
            x.it = &it, x.tree = 0;
            if (it.tiles == 0) return true;
            if (w4 * 32 < it.rows) {
                const bool on = row < it.rows;
                const unsigned rr = it.row0 + (on ? row : 0), node = rr / (unsigned)a.G;
                x.t = it.lo + (int)node, x.hq = it.h * a.G + (int)(rr - node * a.G);
                const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.q) + x.t * a.ld_q +
                                                                   (long long)x.hq * D + wg * (D / 2));
                if (it.b >= 0 && on && it.kt0 + it.tiles == it.kts) x.tree = a.anc_mask[x.t] & low_bits(it.n);
                const uint32_t dst = tmem + lane_base + C::TM_Q + (nr % C::NQ) * (D / 2) + wg * (D / 4);
                constexpr int QC = D / 4 < 32 ? D / 4 : 32;  // columns at a time
#pragma unroll 1
                for (int c = 0; c < D / 4; c += QC) {
                    uint32_t q[QC];
#pragma unroll
                    for (int i = 0; i < QC / 4; ++i) {
                        const uint4 y = on ? src[c / 4 + i] : make_uint4(0, 0, 0, 0);
                        q[4 * i] = y.x, q[4 * i + 1] = y.y, q[4 * i + 2] = y.z, q[4 * i + 3] = y.w;
                    }
#pragma unroll
                    for (int i = 0; i < QC; i += 16) ptx::tmem_st16(dst + c + i, *reinterpret_cast<const uint32_t(*)[16]>(&q[i]));
                }
                ptx::tmem_wait_st();
            }
            ptx::tc_fence_before_sync();
            ptx::mbar_arrive_warp(&sh.q_full[q_phase(nr, C::NQ).barrier]);
            return true;
        };
        auto run = [&]() -> bool {
            unsigned tile = 0;
            Mine me{&sh.items[0], 0, 0, 0}, next;
            int n = 0;
            int full = 0, draft_at = 0, rest = 0;     // (registers: read at every tile)
            // (the round before the first item only takes that one)
            for (;; ++ord) {
                const Item &it = *me.it;
                const bool warp_on = n > 0 && w4 * 32 < it.rows, on = n > 0 && row < it.rows;
                const unsigned last = tile + n - 1;
                bool taken = false;                   // the next item
                float m = -INFINITY, l = 0.f, m_l = -INFINITY;
                for (int j = (int)(tile & 1) == wg ? 0 : 1;; j += 2) {
                    const unsigned g = tile + j, buf = g % C::NSB;
                    if (j >= n && n > 0 && (int)(last & 1) != wg) {  // the other warpgroup's last maximum
                        if (!row_max(&sh.m[row], last, &m)) return false;
                    }
                    // With two Q buffers the next item's queries come in before this warpgroup's last tile, while it
                    // would wait for S: the buffer's last reader was the item before this one.  With one, at the end: the
                    // last Q K^T is done, its S has been read.
                    if (!taken && (j >= n || (C::NQ == 2 && j + 2 >= n))) {
                        if (!take(ord + 1, next)) return false;
                        taken = true;
                    }
                    if (j >= n) break;
                    const int valid = keys_of(j, full, draft_at, rest, it.n);
                    const bool draft = j == draft_at;
                    float m0 = -INFINITY;
                    if (g > 0) {
                        if (!row_max(&sh.m[row], g - 1, &m0)) return false;
                        if (j == 0) m0 = -INFINITY;  // (another item's)
                    }
                    if (!wait_warp(&sh.s_full[g % C::NK], (g / C::NK) & 1)) return false;
                    ptx::tc_fence_after_sync();
                    const uint32_t ts = tmem + lane_base + C::TM_S + buf * KT;
                    if (warp_on && (draft || valid < KT)) {
                        // masked tiles (an item has two at most): minus infinity goes into S itself, so that the step
                        // below stays one piece of straight code
                        const uint64_t seen = draft ? me.tree : low_bits(valid);
#pragma unroll 1
                        for (int c = 0; c < KT; c += 16) {
                            const uint32_t bits = (uint32_t)(seen >> c) & 0xffffu;
                            uint32_t x[16];
                            ptx::tmem_ld16(ts + c, x);
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (!(bits & (1u << i))) x[i] = 0xff800000u;
                            ptx::tmem_st16(ts + c, x);
                        }
                        ptx::tmem_wait_st();
                    }
                    constexpr int HK = C::HALVES ? KT / 2 : KT;  // keys of a row in registers at a time
                    uint32_t raw[HK];
                    float top = -INFINITY;
                    if (warp_on) {
                        float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
                        for (int h = 0; h < KT; h += HK) {
#pragma unroll
                            for (int i = 0; i < HK; i += 32) ptx::tmem_ld32(ts + h + i, *reinterpret_cast<uint32_t(*)[32]>(&raw[i]));
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < HK; i += 2)
                                t[(i >> 1) & 3] = ptx::max3(t[(i >> 1) & 3], __uint_as_float(raw[i]), __uint_as_float(raw[i + 1]));
                        }
                        top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])) * sl2;
                        if (C::P_SMEM) ptx::tc_fence_before_sync();
                    }
                    if (C::P_SMEM) ptx::mbar_arrive_warp(&sh.s_free[buf]);
                    const bool grow = top > m0 + LAZY || (m0 == -INFINITY && top > m0);
                    m = grow ? top : m0;
                    *reinterpret_cast<volatile unsigned long long *>(&sh.m[row]) = (unsigned long long)(g + 1) << 32 | __float_as_uint(m);
                    if (warp_on) {
                        const float ref = m == -INFINITY ? 0.f : m;
                        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                        for (int h = 0; h < KT; h += HK) {
                            if (C::HALVES) {
                                ptx::tmem_ld32(ts + h, *reinterpret_cast<uint32_t(*)[32]>(&raw[0]));
                                ptx::tmem_wait_ld();
                            }
#pragma unroll
                            for (int i = 0; i < HK; i += 2) {
                                const float x = ptx::ex2(fmaf(__uint_as_float(raw[i]), sl2, -ref));
                                const float y = ptx::ex2(fmaf(__uint_as_float(raw[i + 1]), sl2, -ref));
                                acc[i & 2] += x, acc[(i & 2) + 1] += y;
                                // weights as bf16: at most 2^-8 of each, independent from key to key
                                raw[i / 2] = pack_bf16(x, y);
                            }
                            if (!C::P_SMEM)
#pragma unroll
                                for (int i = 0; i < HK / 2; i += 16) ptx::tmem_st16(ts + h / 2 + i, *reinterpret_cast<const uint32_t(*)[16]>(&raw[i]));
                        }
                        if (m != m_l) l *= ptx::ex2(m_l - ref);
                        m_l = m;
                        l += (acc[0] + acc[1]) + (acc[2] + acc[3]);
                    }
                    if constexpr (C::P_SMEM) {
                        if (g >= 2 && !wait_warp(&sh.pv_done[g % C::NV], (g / C::NV - 1) & 1)) return false;  // the buffer's last reader
                        if (warp_on) {  // row of 128 bytes, swizzled as the MMA reads it
                            unsigned char *p = p_bufs + (g & 1) * C::P_BYTES + row * 128;
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                *reinterpret_cast<uint4 *>(p + ((i ^ (row & 7)) * 16)) =
                                    make_uint4(raw[4 * i], raw[4 * i + 1], raw[4 * i + 2], raw[4 * i + 3]);
                            ptx::fence_proxy_async();
                        }
                    }
                    if (draft || valid < KT) {
                        // Rows of V that no weight may meet: past the end (left over from the stage's last use, or the
                        // page's unused slots), and draft rows with NaN or infinity, which the epilogue adds where they
                        // are seen.  A zero weight would make NaN of them.
                        const unsigned sidx = g % C::NV;
                        if (!wait_warp(&sh.v_full[sidx], (g / C::NV) & 1)) return false;
                        unsigned char *v = v_stages + sidx * C::STAGE;
                        const int upto = (valid + 15) / 16 * 16;
                        constexpr int VR = C::NC * 8;  // 16-byte vectors of a row
                        for (int i = (draft ? 0 : valid * VR) + w4 * 32 + lane; i < upto * VR; i += 128) {
                            const int key = i / VR, c = i - key * VR;
                            uint4 *p = reinterpret_cast<uint4 *>(v + (key >> lay.log_v_rows) * (lay.v_rows * C::NC * 128) +
                                                                 ((c >> 3) * lay.v_rows + (key & (lay.v_rows - 1))) * 128 + (c & 7) * 16);
                            if (key >= valid) {
                                *p = make_uint4(0, 0, 0, 0);
                                continue;
                            }
                            uint4 x = *p;
                            if (nonfinite2(x.x) || nonfinite2(x.y) || nonfinite2(x.z) || nonfinite2(x.w)) {
                                atomicOr(&sh.nonfinite[ord & 3][key >> 5], 1u << (key & 31));
                                uint32_t *xw = reinterpret_cast<uint32_t *>(&x);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if ((xw[e] & 0x7f80u) == 0x7f80u) xw[e] &= 0xffff0000u;
                                    if ((xw[e] & 0x7f800000u) == 0x7f800000u) xw[e] &= 0x0000ffffu;
                                }
                                *p = x;
                            }
                        }
                        ptx::fence_proxy_async();
                        __syncwarp();
                    }
                    if (j > 0 && __any_sync(0xffffffffu, grow)) {
                        const unsigned pg = g - 1;
                        if (!wait_warp(&sh.pv_done[pg % C::NV], (pg / C::NV) & 1)) return false;
                        ptx::tc_fence_after_sync();
                        const float f = grow ? ptx::ex2(m0 - m) : 1.f;  // (grow: m is finite or +infinity)
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t o[32];
                            ptx::tmem_ld32(tmem + lane_base + c, o);
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            ptx::tmem_st16(tmem + lane_base + c, *reinterpret_cast<const uint32_t(*)[16]>(&o[0]));
                            ptx::tmem_st16(tmem + lane_base + c + 16, *reinterpret_cast<const uint32_t(*)[16]>(&o[16]));
                        }
                    }
                    ptx::tmem_wait_st();
                    ptx::tc_fence_before_sync();
                    ptx::mbar_arrive_warp(&sh.p_full[buf]);
                }
                if (n > 0) {
                // ---- end of the item: the sum of both, the output
                const float ref = m == -INFINITY ? 0.f : m;
                if (m != m_l) l *= ptx::ex2(m_l - ref);
                sh.l[ord & 1][wg][row] = l;
                ptx::mbar_arrive_warp(&sh.exch[w4]);
                if (!wait_warp(&sh.exch[w4], ord & 1)) return false;
                l += sh.l[ord & 1][wg ^ 1][row];
                // (a parity names a phase only to who has seen the one before it: where Q K^T does not wait for P V, the
                // product before the last comes first)
                if (C::P_SMEM && last > 0 && !wait_warp(&sh.pv_done[(last - 1) % C::NV], ((last - 1) / C::NV) & 1)) return false;
                if (!wait_warp(&sh.pv_done[last % C::NV], (last / C::NV) & 1)) return false;
                ptx::tc_fence_after_sync();
                const bool bad = sh.bad_item[ord % 16] == ord + 1;
                if (tid == 0) sh.nonfinite[(ord + 2) & 3][0] = sh.nonfinite[(ord + 2) & 3][1] = 0;
                uint64_t nf = me.tree & ((uint64_t)sh.nonfinite[ord & 3][0] | (uint64_t)sh.nonfinite[ord & 3][1] << 32);
                const int cap = it.cap;
                const long long orow = (long long)me.t * a.H_q + me.hq;
                __nv_bfloat16 *const out_row = static_cast<__nv_bfloat16 *>(a.O) + orow * D;
                const float inv = l == 0.f ? 0.f : 1.f / l;  // (a row that saw nothing has 0 everywhere)
                constexpr int HALF = D / 2, EC = 32;  // this warpgroup's columns, and how many at a time
#pragma unroll 1
                for (int c = wg * HALF; c < (wg + 1) * HALF; c += EC) {
                    uint32_t o[EC];
                    if (warp_on) {
#pragma unroll
                        for (int i = 0; i < EC; i += 32) ptx::tmem_ld32(tmem + lane_base + c + i, *reinterpret_cast<uint32_t(*)[32]>(&o[i]));
                        ptx::tmem_wait_ld();
                    }
                    if (c + EC == (wg + 1) * HALF) {  // all read: the next item's products may overwrite it
                        ptx::tc_fence_before_sync();
                        ptx::mbar_arrive_warp(&sh.o_free);
                    }
                    if (on) {
                        if (cap == 0) {
                            __nv_bfloat16 *out = out_row + c;
                            if (!bad) {
#pragma unroll
                                for (int i = 0; i < EC; i += 8) {
                                    uint4 y;
                                    uint32_t *yw = reinterpret_cast<uint32_t *>(&y);
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        yw[e] = pack_bf16(__uint_as_float(o[i + 2 * e]) * inv, __uint_as_float(o[i + 2 * e + 1]) * inv);
                                    *reinterpret_cast<uint4 *>(out + i) = y;
                                }
                            }
                        } else {
                            if (wg == 0 && c == 0) *reinterpret_cast<float2 *>(it.blk_ml + 2 * row) = make_float2(m, bad ? PAGE_BAD : l);
                            float *po = it.blk_o + (c / 4 * cap + row) * 4;
#pragma unroll
                            for (int i = 0; i < EC; i += 4)
                                *reinterpret_cast<uint4 *>(po + i * cap) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                        }
                    }
                    __syncwarp();
                }
                if (on)
                    for (; nf; nf &= nf - 1) {  // seen draft rows with NaN or infinity: those elements, onto what was stored
                        const int jn = __ffsll((long long)nf) - 1;
                        const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(a.v) + (it.lo + jn) * a.ld_v + (long long)it.h * D;
#pragma unroll 1
                        for (int c = wg * HALF; c < (wg + 1) * HALF; ++c) {
                            const float x = to_f32(v[c]);
                            if (isfinite(x)) continue;
                            if (cap == 0) {
                                __nv_bfloat16 *out = out_row + c;
                                if (!bad) *out = __float2bfloat16_rn(to_f32(*out) + x);
                            } else {
                                float *out = it.blk_o + (c / 4 * cap + row) * 4 + c % 4;
                                *out += x;
                            }
                        }
                    }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sh.item_empty[ord % ITEMS]);
                }
                if (next.it->tiles == 0) return true;
                tile += n;
                me = next, n = me.it->tiles;
                full = me.it->full, draft_at = me.it->draft, rest = me.it->rest;
            }
        };
        if (!run()) {
            ptx::tmem_wait_st();
            if (lane == 0) atomicMin(&sh.unfinished, ord == ~0u ? 0u : ord);
        }
        __syncwarp();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    if (sh.unfinished != ~0u) {
        if (tid < 2) {  // copies in flight have to land before the CTA may leave
            const unsigned filled = sh.copied[tid], ns = tid ? C::NV : C::NK;
            uint64_t *fulls = tid ? sh.v_full : sh.k_full;
            for (unsigned i = filled > ns ? filled - ns : 0; i < filled; ++i)
                for (int t = 0; t < 100000 && !ptx::mbar_try_wait(&fulls[i % ns], (i / ns) & 1); ++t) __nanosleep(20);
        }
        mark_unfinished<D>(a, ws, sh.part, Walk{sh.first_b, (unsigned)sh.first_off, sh.part.u0, sh.first_seq}, sh.unfinished);
    }
    if (warp == MMA_QK) ptx::tmem_dealloc(tmem, 512);
}

// The join: o = sum_p 2^{m_p - m} o_p / sum_p 2^{m_p - m} l_p over the parts p of an item in the order of its keys.  A warp
// takes 8 rows and 16 STEPS columns of them: lane = row + 8 * column group, 4 groups of 4 columns a step, so that both the
// blocks (8 rows of a group are 128 bytes) and the output (4 groups of a row are 32) move in whole sectors.  Warps share out
// columns, not parts: nothing has to meet.  (With the parts over warps that met in shared memory too few of a CTA's warps had
// work: 32 trees of 32 nodes, heads of 256, took 94 us instead of 87.)  The blocks come out of L2, where the main kernel left
// them; what bounds it is the chain launch, lookup, blocks, output: 3 us with few rows, 6 to 10 with 20 MB of blocks.
// A part with a bad page, or one that was not worked out, has a negative l: the row is left.
template <int STEPS> struct Join {
    float4 acc[STEPS];
    float m = -INFINITY, l = 0.f;
    int bad = 0;  // status bits
    __device__ __forceinline__ Join()
    {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ __forceinline__ void add(float2 x, const float4 (&y)[STEPS])
    {
        if (x.y < 0.f) bad |= x.y == PAGE_BAD ? TREEWY_SEQ_BAD_PAGE : TREEWY_SEQ_TIMEOUT;
        if (x.y == 0.f) return;  // saw nothing
        const float mn = fmaxf(m, x.x), ref = mn == -INFINITY ? 0.f : mn;
        const float f0 = ptx::ex2(m - ref), f1 = ptx::ex2(x.x - ref);
        m = mn, l = l * f0 + x.y * f1;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            acc[i].x = acc[i].x * f0 + y[i].x * f1, acc[i].y = acc[i].y * f0 + y[i].y * f1;
            acc[i].z = acc[i].z * f0 + y[i].z * f1, acc[i].w = acc[i].w * f0 + y[i].w * f1;
        }
    }
    // out: this lane's row, at the warp's first column
    __device__ __forceinline__ void store(__nv_bfloat16 *out, int cg)
    {
        if (bad) return;
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            *reinterpret_cast<uint2 *>(out + 16 * i + 4 * cg) =
                make_uint2(pack_bf16(acc[i].x * inv, acc[i].y * inv), pack_bf16(acc[i].z * inv, acc[i].w * inv));
    }
};
// column groups 4 i + cg from column c0 on, of one row of a block of cap rows
template <int STEPS> __device__ __forceinline__ void load_part(float4 (&y)[STEPS], const float *block, int cap, int row, int c0, int cg)
{
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
        y[i] = __ldcs(reinterpret_cast<const float4 *>(block + ((long long)(c0 / 4 + 4 * i + cg) * cap + row) * 4));
}

constexpr int JOIN_WARPS = 8;

// Items that a part cut: grid (CTAs of the main kernel, warps of a block / 8).  UN parts are loaded at a time: with few rows
// there are few warps and many parts (up to one for each CTA), with many rows the other way round.
template <int D, int STEPS, int UN>
__global__ void __launch_bounds__(JOIN_WARPS * 32) attn_join_cut_kernel(const __grid_constant__ AttnArgs a, int R, Ws ws)
{
    constexpr int CW = D / (16 * STEPS);         // warps that share a row
    const int w = blockIdx.y * JOIN_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31, cg = lane >> 3;
    const int row = w / CW * 8 + (lane & 7), c0 = w % CW * (16 * STEPS);
    grid_dependency_wait();
    grid_dependency_trigger();
    const int4 d0 = *reinterpret_cast<const int4 *>(ws.desc + 8 * blockIdx.x), d1 = *reinterpret_cast<const int4 *>(ws.desc + 8 * blockIdx.x + 4);
    const int pieces = d0.x;
    if (pieces == 0 || row >= d1.y) return;
    const int member = blockIdx.x % R, cap = ws.slot_cap;
    Join<STEPS> jn;
#pragma unroll 1
    for (int p0 = 0; p0 < pieces; p0 += UN) {
        float2 x[UN];
        float4 y[UN][STEPS];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int p = min(p0 + i, pieces - 1);
            const long long blk = ((long long)(p == 0 ? d0.y : 2 * (d1.z + p)) * R + member) * cap;
            x[i] = __ldcs(reinterpret_cast<const float2 *>(ws.slot_ml + (blk + row) * 2));
            load_part<STEPS>(y[i], ws.slot_o + blk * D, cap, row, c0, cg);
        }
#pragma unroll
        for (int i = 0; i < UN; ++i)
            if (p0 + i < pieces) jn.add(x[i], y[i]);
    }
    const int rr = d1.x + row, node = rr / a.G;
    jn.store(static_cast<__nv_bfloat16 *>(a.O) + ((long long)(d0.z + node) * a.H_q + d0.w * a.G + rr - node * a.G) * D + c0, cg);
}

// With a shared prompt every row has two items, its sequence's and the prompt's, each whole or cut.  Grid (warps of the
// longest tree under one key/value head / 8, key/value heads, sequences).
template <int D, int STEPS>
__global__ void __launch_bounds__(JOIN_WARPS * 32) attn_join_shared_kernel(const __grid_constant__ AttnArgs a, int R, Ws ws)
{
    constexpr int CW = D / (16 * STEPS);
    const int w = blockIdx.x * JOIN_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31, cg = lane >> 3, h = blockIdx.y, b = blockIdx.z;
    const int r = w / CW * 8 + (lane & 7), c0 = w % CW * (16 * STEPS);  // row among the sequence's under this head
    grid_dependency_wait();
    grid_dependency_trigger();
    int lo, n, len;
    if (check_sequence(a.node_offsets, a.c.context_len, b, a.T, a.max_nodes, (long long)a.c.max_pages * a.c.page_size, a.shared_len, &lo, &n, &len) ||
        r >= n * a.G)
        return;
    // the two items: their parts, and what is loaded first of each
    struct Where {
        const float *ml, *o;
        int cap, row, slot, more;  // slot: the block of the part after the first, if there is one
    };
    constexpr int blocks = 2 * MAX_CTAS;
    auto find = [&](bool is_own) {
        const unsigned i = is_own ? r : lo * a.G + r;  // the row in the list that the item's tiles cut up
        const int tile = i / MT, tiles = is_own ? ws.own_tiles : ws.shared_tiles;
        const int4 at = (is_own ? ws.own_at : ws.shared_at)[((long long)(is_own ? b : 0) * a.c.H_kv + h) * tiles + tile];
        Where x;
        x.row = i % MT;
        if (at.y == 0) {
            x.ml = is_own ? ws.own_ml : ws.shared_ml, x.o = is_own ? ws.own_o : ws.shared_o, x.cap = is_own ? ws.own_cap : MT;
        } else {
            x.ml = ws.slot_ml, x.o = ws.slot_o, x.cap = ws.slot_cap;
        }
        // (calls that overlap on one workspace overwrite each other's: whatever lies there stays within it)
        const unsigned most = at.y == 0 ? (is_own ? a.B : 1) * a.c.H_kv * tiles : blocks;
        const long long blk = min((unsigned)at.x, most - 1);
        x.slot = min((unsigned)((at.z + 1) * 2 * R + tile % R), (unsigned)blocks);
        x.more = at.y == 0 ? 0 : at.y - 1;
        x.ml += blk * x.cap * 2, x.o += blk * x.cap * D;
        return x;
    };
    Join<STEPS> jn;
    const Where at[2] = {find(false), find(true)};
    float2 x[2];
    float4 y[2][STEPS];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[i] = __ldcs(reinterpret_cast<const float2 *>(at[i].ml + 2 * at[i].row));
        load_part<STEPS>(y[i], at[i].o, at[i].cap, at[i].row, c0, cg);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // the prompt, then the sequence's own keys
        jn.add(x[i], y[i]);
#pragma unroll 1
        for (int p = 0, slot = at[i].slot; p < at[i].more && slot < blocks; ++p, slot += 2 * R) {
            const long long blk = (long long)slot * ws.slot_cap;
            const float2 xp = __ldcs(reinterpret_cast<const float2 *>(ws.slot_ml + (blk + at[i].row) * 2));
            float4 yp[STEPS];
            load_part<STEPS>(yp, ws.slot_o + blk * D, ws.slot_cap, at[i].row, c0, cg);
            jn.add(xp, yp);
        }
        if (i == 0 && jn.bad && a.seq_status) atomicOr(&a.seq_status[b], jn.bad);
    }
    const int node = r / a.G;
    jn.store(static_cast<__nv_bfloat16 *>(a.O) + ((long long)(lo + node) * a.H_q + h * a.G + r - node * a.G) * D + c0, cg);
}

struct Plan {
    int R, slot_cap, own_cap, own_tiles, shared_tiles;
    size_t desc, at, slots, own, shared;  // elements; items beside a shared prompt; rows of the three kinds of block
};
Plan plan_of(const AttnArgs &a)
{
    Plan p;
    const long long rows = (long long)a.max_nodes * a.G, tiles = (rows + MT - 1) / MT;
    p.R = (int)(tiles > 4 ? 4 : tiles);
    p.own_cap = rows > MT ? MT : (int)rows, p.own_tiles = (int)tiles;
    p.slot_cap = a.shared_len > 0 ? MT : p.own_cap;
    p.desc = 8 * MAX_CTAS;
    p.slots = 2ull * MAX_CTAS * p.slot_cap;
    p.own = a.shared_len > 0 ? (size_t)a.B * a.c.H_kv * p.own_tiles * p.own_cap : 0;
    p.shared_tiles = (int)(((long long)a.T * a.G + MT - 1) / MT);
    p.shared = a.shared_len > 0 ? (size_t)a.c.H_kv * p.shared_tiles * MT : 0;
    p.at = a.shared_len > 0 ? ((size_t)a.B * p.own_tiles + p.shared_tiles) * a.c.H_kv : 0;
    return p;
}

template <int D> cudaError_t launch_d(AttnArgs a, cudaStream_t stream)
{
    using C = Cfg<D>;
    int dev = 0, sms = 0;
    cudaError_t e = current_device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    const Plan p = plan_of(a);
    const int ctas = (sms < MAX_CTAS ? sms : MAX_CTAS) / p.R * p.R;
    Ws ws;
    unsigned char *at = reinterpret_cast<unsigned char *>(a.ws);
    ws.desc = reinterpret_cast<int *>(at), at += p.desc * 4;
    ws.own_at = reinterpret_cast<int4 *>(at), ws.shared_at = ws.own_at + (size_t)a.B * a.c.H_kv * p.own_tiles, at += p.at * 16;
    ws.slot_o = reinterpret_cast<float *>(at), at += p.slots * D * 4;
    ws.own_o = reinterpret_cast<float *>(at), at += p.own * D * 4;
    ws.shared_o = reinterpret_cast<float *>(at), at += p.shared * D * 4;
    ws.slot_ml = reinterpret_cast<float *>(at), at += p.slots * 8;
    ws.own_ml = reinterpret_cast<float *>(at), at += p.own * 8;
    ws.shared_ml = reinterpret_cast<float *>(at);
    ws.slot_cap = p.slot_cap, ws.own_cap = p.own_cap, ws.own_tiles = p.own_tiles, ws.shared_tiles = p.shared_tiles;
    a.log_page = 0;
    while ((1 << a.log_page) < a.c.page_size) ++a.log_page;

    EncodeTiledFn enc = tma_encode_fn();
    if (!enc) return cudaErrorNotSupported;
    CUtensorMap kc, vc, k, v;
    const CacheView &c = a.c;
    const int box = c.page_size < KT ? c.page_size : KT;
    Layout lay;
    lay.v_rows = box;
    for (lay.log_v_rows = 3; (1 << lay.log_v_rows) < box; ++lay.log_v_rows) {}
    bool by_chunk = false;
    auto lay_k = [&](auto b) { by_chunk = decltype(b)::K_BY_CHUNK, lay.k_chunk = decltype(b)::K_CHUNK, lay.k_group = decltype(b)::K_GROUP; };
    if (box == 8) lay_k(Boxes<D, 8>{});
    else if (box == 16) lay_k(Boxes<D, 16>{});
    else if (box == 32) lay_k(Boxes<D, 32>{});
    else lay_k(Boxes<D, 64>{});
    auto cache_map = [&](CUtensorMap *m, const void *base, int rows, int chunks) {
        const cuuint64_t dims[5] = {64, (cuuint64_t)c.page_size, (cuuint64_t)C::NC, (cuuint64_t)c.H_kv, (cuuint64_t)c.n_pages};
        // (the stride of a dimension of one does not count, but has to be a legal one)
        const cuuint64_t strides[4] = {(cuuint64_t)c.stride_slot * 2, 128, c.H_kv > 1 ? (cuuint64_t)c.stride_head * 2 : 16,
                                       c.n_pages > 1 ? (cuuint64_t)c.stride_page * 2 : 16};
        const cuuint32_t bx[5] = {64, (cuuint32_t)rows, (cuuint32_t)chunks, 1, 1}, es[5] = {1, 1, 1, 1, 1};
        // (128 bytes to L2 at a time: a row of a head of 64 is no longer, and with 256 its neighbour came along from HBM;
        // decoding 64 x 8192 keys, 8 such heads: 132 us instead of 139, other widths the same)
        return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(base), dims, strides, bx, es,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    const uint64_t cols = (uint64_t)c.H_kv * D;
    if (!cache_map(&kc, c.k, by_chunk ? box : 8, by_chunk ? 1 : C::NC) || !cache_map(&vc, c.v, box, C::NC) ||
        !tma_make_map_bf16(enc, &k, a.k, cols, a.T, a.ld_k * 2, 64, 8, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !tma_make_map_bf16(enc, &v, a.v, cols, a.T, a.ld_v * 2, 64, 8, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    const int smem = (C::NK + C::NV) * C::STAGE + 2 * C::P_BYTES + 1024;
    e = ensure_dynamic_smem(reinterpret_cast<const void *>(attn_tc_kernel<D>), smem, dev);
    if (e != cudaSuccess) return e;
    e = launch_dependent(attn_tc_kernel<D>, dim3(ctas), dim3(THREADS), smem, stream, a, p.R, ws, lay, kc, vc, k, v);
    if (e != cudaSuccess) return e;
    if (a.shared_len > 0) {
        constexpr int STEPS = 4;
        const long long warps = ((long long)a.max_nodes * a.G + 7) / 8 * (D / (16 * STEPS));
        return launch_dependent(attn_join_shared_kernel<D, STEPS>, dim3((unsigned)((warps + JOIN_WARPS - 1) / JOIN_WARPS), a.c.H_kv, a.B),
                                dim3(JOIN_WARPS * 32), 0, stream, a, p.R, ws);
    }
    auto cut = [&](auto steps, auto un) {
        constexpr int STEPS = decltype(steps)::value;
        const int warps = (p.slot_cap + 7) / 8 * (D / (16 * STEPS));
        return launch_dependent(attn_join_cut_kernel<D, STEPS, decltype(un)::value>, dim3(ctas, (warps + JOIN_WARPS - 1) / JOIN_WARPS),
                                dim3(JOIN_WARPS * 32), 0, stream, a, p.R, ws);
    };
    // Few rows: many parts to an item and few warps, so little of a row to each and many parts at a time (one sequence 14.0 us
    // instead of 15.4, two of 65537 keys 93.1 instead of 94.6).  Many rows: two or three parts and many warps (32 trees of 32
    // nodes, heads of 256: 87 us instead of 98, of which the join is 6).
    if (p.slot_cap <= 32) return cut(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
    return cut(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
}

}  // namespace

// The units of one sequence, and of the shared prompt, stay below 2^31.
static bool units_fit(const AttnArgs &a)
{
    const long long own = ((long long)a.max_nodes * a.G + MT - 1) / MT *
                          (((long long)a.c.max_pages * a.c.page_size / KT + 2) * MAX_TILE + MAX_START);
    const long long shared = ((long long)a.T * a.G + MT - 1) / MT * ((a.shared_len / KT + 2ll) * MAX_TILE + MAX_START);
    const long long most = 0x7fffffffll / a.c.H_kv;
    return own <= most && shared <= most;
}

bool attn_tc_applies(const AttnArgs &a, treewy_dtype_t io)
{
    const CacheView &c = a.c;
    const bool pow2 = (c.page_size & (c.page_size - 1)) == 0;
    // 8-row groups of the swizzle have to stay whole within a page; the tensor maps want a pool that exists and real strides
    return io == TREEWY_BF16 && (c.d == 64 || c.d == 128 || c.d == 256) && pow2 && c.page_size >= 8 && c.n_pages > 0 &&
           c.max_pages > 0 && c.stride_slot > 0 && (c.H_kv == 1 || c.stride_head > 0) && (c.n_pages == 1 || c.stride_page > 0) &&
           (long long)a.T * a.H_q <= 0x7fffffffll && a.B <= 65535 && a.c.H_kv <= 65535 && units_fit(a);
}

size_t attn_tc_workspace(const AttnArgs &a)
{
    const Plan p = plan_of(a);
    return p.desc * 4 + p.at * 16 + (p.slots + p.own + p.shared) * (a.c.d + 2) * 4;
}

cudaError_t launch_attn_tc(const AttnArgs &a, cudaStream_t stream)
{
    if (a.c.d == 256) return launch_d<256>(a, stream);
    if (a.c.d == 128) return launch_d<128>(a, stream);
    return launch_d<64>(a, stream);
}

}  // namespace treewy
