// treewy_attn_chunk, bf16: new rows over a paged cache on the tensor cores.
//
// Rows.  A row tile is 128 rows of one (sequence, key/value head): the G query heads that read this head, of 128 / G tokens one
// after the other.  A CTA works on two of them at a time (heads of 256: one), each a stream with its own S and O in
// tensor memory and its own warpgroup for the softmax, over the same tiles of keys and values: while one stream's softmax
// runs, the tensor cores have the other's products.  An item with one row tile (decoding, short pieces) gives the two
// streams alternate key tiles instead, and joins their outputs at its end.
// Keys.  Tiles of 64 at multiples of 64: those of the sinks, then from the first row's window to the last
// row.  Tiles that some row does not see whole are masked, those that no row of a stream sees are left out for it.
// One tile of a stream:  S = Q K^T, the softmax step in registers (a row to a thread), P = weights as bf16 over S's
// own columns, O += P V (V read with its rows as the K index).  A stream has two S buffers or more, and its scores are issued as many tiles
// ahead of its products: the next S is there when a softmax step ends.
// Softmax.  o = sum_x 2^{s_x - m} v_x / sum_x 2^{s_x - m} (s in log2) for any reference m.  A row's m is 14 above the maximum of its first
// tile and stays until the weights of one tile add up to 1 (or to NaN); then m becomes 14 above the maximum so far and O and l are scaled.  So
// an ordinary tile has no maximum, no exchange between threads and no pass over O: an fma and an exponential a weight, an addition, half a
// packing.  With weights of less than 1 a tile, rounded to bf16 or not, O overflows nowhere where weights against the true maximum would not make it,
// whatever the values.  (Without the 14 and with a limit of 2^40 m moves less often still, but values from 2^88 on came out infinite.)  And the
// roundings of O among fp32's last numbers, 2^-149, are 2^-135 in the output: less than bf16 tells apart.
//
// What bounds it.  Heads of 128, a prompt of 8192 over 32 / 8 heads (550 GFLOP), 525 us, 1050 TFLOP/s or 0.62 of the measured GEMM rate (up to
// 587 where the power cap has lowered the clock).  Of 541 us 446 are left without the exponentials, 502 without half of Q K^T, 380 without both: three things are about equally long.  The
// tensor cores: an MMA of Q K^T with both operands in shared memory takes 50 cycles for 64 keys where its arithmetic takes 32, since the
// operands are 6 kB at 128 bytes a cycle; with P in tensor memory P V runs at its arithmetic.  The exponentials: 16 a cycle and SM, 1024 of some 2100 cycles a
// tile of both streams.  And the softmax warps' own latency, 2 of them to a scheduler that issues 0.37 a cycle.  Heads of 64: 490 us (561
// TFLOP/s), without exponentials 322.  Heads of 256 (one stream, four S buffers): 508-565 us (1083).  Decoding, 64 sequences
// of 2048 to 8192 tokens: 222 us, 5.9 TB/s, HBM (all of 8192: 335, 6.4); with heads of 64 167-174 us, 3.9 TB/s: four rows of 128 are
// used, four lanes of a warp take a tile's exponentials.  Short items pay their start: eight prompts of up to 512 46 us, window of 256 with heads of 64 154.
//
// Why so.  What else was built and measured on the prompt of 8192, heads of 128 (and 64), against this: a row split over two threads
// 585; key tiles of 128 with one S buffer 773; two warpgroups a stream on alternate tiles, the reference passed between them, 1120 (1080); three S buffers for
// heads of 64 (504 there, window 253 -> 239); one MMA thread for both streams 719; exponentials partly on the FMA pipes 653
// where this form had 606; the next S loaded ahead of the weights' store 714 where this form had 540.
//
// Work.  (sequence, head, item) in one line, an item's length being its start's cost and its keys, cut into equal parts,
// one for each CTA: no CTA waits for a longer neighbour, whatever the lengths and windows.  A cut item leaves unnormalised
// outputs with their m and l in the workspace; a second kernel joins them in the order of the keys.
#include <type_traits>

#include "attn_common.cuh"
#include "chunk_phases.cuh"
#include "ptx_sm100.cuh"
#include "tma_host.cuh"

namespace treewy {
namespace {

constexpr int MT = 128;                // rows of a tile
constexpr int KT = 64;                 // keys of a tile
constexpr int MAX_CTAS = 160;
constexpr int ITEMS = 8;               // ring of work items between the producer and the other roles
constexpr int START = 256;             // cost of an item's start, in keys (128 and 512 cost long prompts 2 %, and 2048 rows 4)
constexpr int MIN_UNITS = 256;         // least units of a part; at least a tile's keys, so that a part inside an item holds the start of one
constexpr int UNSEEN = -0x7fffffff;    // for a page that is not looked up
constexpr float ABOVE = 14.f;          // the reference above the maximum that it was taken from, in log2 (7: prompts behind a window of 256, where a row
                                       // sees little of its first tile, 162 us for 154; 20 loses what bf16 holds of values below 2^-110)
constexpr float LARGE = 1.f;           // a row's weights of one tile add up to less
static_assert(KT < 1 << 14, "a tile's weights add up to less than LARGE behind a new reference");
constexpr float PAGE_BAD = -1.f, NOT_DONE = -2.f;  // l of a row whose part is not there

template <int D> struct Cfg {
    static constexpr int NC = D / 64;                    // 64-column chunks of a row
    static constexpr int STREAMS = D == 256 ? 1 : 2;     // what 512 columns of tensor memory leave
    static constexpr int STAGE = NC * KT * 128;          // bytes of a tile
    static constexpr int NB = D == 256 ? 4 : 2;          // S buffers of a stream
    static constexpr int NK = D == 64 ? 10 : D == 128 ? 5 : 3, NV = D == 64 ? 10 : D == 128 ? 5 : 2;
    static constexpr int Q_TILE = NC * MT * 128;
    static constexpr int TILES = STREAMS * Q_TILE + (NK + NV) * STAGE;  // bytes
    static constexpr int SOFT_WARPS = 4 * STREAMS, MMA = SOFT_WARPS, PRODUCER_K = MMA + 2, PRODUCER_V = MMA + 3;  // (two of MMA)
    static constexpr int THREADS = (SOFT_WARPS + 4) * 32;
    static constexpr int TM_S = 256;                     // columns: O of stream s at s * D, S buffer b of it at 256 + (s * NB + b) * KT
    static constexpr int CAP = STREAMS * MT;             // rows of an item at most
};

// Where the copies put a tile, and in how many pieces.  A box is rows of one page (all of it, or KT of it) and holds the
// chunks of its rows one after the other.  V comes so: rows are its K index, and any 16 of one page make an MMA step.  K
// needs its 8-row groups equally far apart: whole boxes one chunk at a time, or all chunks of 8 rows, whichever makes
// fewer copies.
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
    int b, h, lo, len;          // sequence, key/value head, its first packed row, its context
    int t0, tokens;             // first token of the item among the sequence's rows, tokens
    int pair;                   // two row tiles (else one)
    int j0, tiles, kts;         // first key tile here, tiles here (0: the end), tiles of the whole item
    int sink_tiles, low_tile;   // tile j is tile j of the cache for j < sink_tiles, else low_tile + j - sink_tiles
    int slot;                   // the block of a cut item, else -1
};

struct Seq {
    int lo, n, len, items;
    unsigned long long per;     // units under one head
};
// A CTA's part of the line of work
struct Part {
    long long u0, u1, W;        // its units, and all of the line
    int parts, group;
};
struct Walk {                   // a CTA's way along its part
    int b, h, i;                // the item it is in: sequence, head, item under it
    long long o, u;             // units into the item, and on the line
    Seq s;
};

template <int D> struct Shared {
    using C = Cfg<D>;
    uint64_t k_full[C::NK], k_free[C::NK], v_full[C::NV], v_free[C::NV];
    // Of an S buffer: filled, its weights stored, its product done.  (One to a buffer: a parity names a phase only to who has seen
    // the one before it, and a full S says that the buffer's last product is done.)
    uint64_t s_full[4], p_full[4], pv_done[4], o_free[2], q_full, q_free, item_full[ITEMS], item_empty[ITEMS], ml_full[4], end[2];
    Item items[ITEMS];
    float2 ml[C::STREAMS == 2 ? MT : 1];  // of the second stream's rows, for the first
    unsigned bad_item[8];       // ordinal + 1 of an item that met a page out of range
    unsigned nonfinite[8];      // ordinal + 1 of an item with NaN or infinity among the values of its masked tiles
    long long scan[C::THREADS / 32];
    long long first_off;
    Seq first_seq;              // of sequence first_b
    Part part;
    int first_b;
    unsigned unfinished;        // first of this CTA's items whose output is not all stored, once a wait has run out; else ~0
    unsigned copied[2];         // tiles whose copies of K and of V were issued
    unsigned q_copied;          // items whose queries' copies were
    uint32_t tmem;
};

// The workspace.  A block holds unnormalised outputs of an item's rows, column groups of 4 first: element (row, c) at ((c / 4) *
// cap + row) * 4 + c % 4, so that the rows of a warp are neighbours when its threads write a column group each of their own
// row; (m, l) of the rows beside it.  A part cuts two items at most, the one its start falls into (block 2 g) and one more.
struct Ws {
    int *desc;                  // [MAX_CTAS][8]: the item that a CTA's part cuts at its end
    float *ml, *o;              // [2 * CTAs] blocks
    int cap;                    // rows of a block
};

template <int D> __device__ __forceinline__ int tile_tokens(const ChunkArgs &a) { return MT / a.G; }  // of a row tile

// Units of a sequence's items before item i (under one head): of each its start and its keys, which are its tokens and what
// the first of them sees beside itself, min(p, window + sinks - 1).
template <int D> __device__ __forceinline__ long long units_before(const ChunkArgs &a, int len, int n, long long i)
{
    const long long per = (long long)Cfg<D>::STREAMS * tile_tokens<D>(a), most = (long long)a.window + a.sinks - 1;
    // items whose first token is behind fewer than `most` (all of them where there is no window: no division)
    const long long far = most - len;
    const long long m = far >= i * per ? i : far <= 0 ? 0 : (long long)(((unsigned)far + (unsigned)per - 1) / (unsigned)per);
    const long long tokens = i * per < n ? i * per : n;
    return i * START + tokens + m * len + per * (m * (m - 1) / 2) + (i - m) * most;
}
template <int D> static __device__ __noinline__ Seq load_seq(const ChunkArgs &a, int b, int *status)
{
    Seq s;
    *status = check_rows(a.row_offsets, a.c.context_len, b, a.T, (long long)a.c.max_pages * a.c.page_size, &s.lo, &s.n, &s.len);
    const int per = Cfg<D>::STREAMS * tile_tokens<D>(a);
    s.items = *status ? 0 : (s.n + per - 1) / per;
    s.per = s.items ? units_before<D>(a, s.len, s.n, s.items) : 0;
    return s;
}
// parts: CTAs that get work.  Part g has units g W / parts .. (g + 1) W / parts - 1.  Of an item of START + k units tile t of kts
// begins at START + t k / kts: it belongs to the part that this unit is in.
__device__ __forceinline__ long long part_begin(long long g, long long W, int parts) { return g * W / parts; }
__device__ __forceinline__ int part_of(long long unit, long long W, int parts) { return (int)(((unit + 1) * parts - 1) / W); }
__device__ __forceinline__ int tiles_before(long long o, long long k, int kts)
{
    return o <= START ? 0 : (int)min((long long)kts, ((o - START) * kts + k - 1) / k);
}

// Where a CTA's part begins: unit `off` of sequence b
template <int D> static __device__ __noinline__ Walk walk_from(const ChunkArgs &a, int b, long long off, long long u, const Seq &s)
{
    Walk w{b, 0, 0, 0, u, s};
    if (b < 0) return w;               // (no work)
    w.h = (int)(off / (long long)s.per);
    const long long in_head = off - w.h * (long long)s.per;
    int hi = s.items;
    while (hi - w.i > 1) {
        const int mid = (w.i + hi) >> 1;
        if (units_before<D>(a, s.len, s.n, mid) <= in_head) w.i = mid;
        else hi = mid;
    }
    w.o = in_head - units_before<D>(a, s.len, s.n, w.i);
    return w;
}

// The next item that has tiles here; 0 tiles: the end.  The part that has a cut item's first tile leaves word for the join.  (One thread
// walks while tiles are copied and worked on: divisions only for items that are cut.)
template <int D> static __device__ __noinline__ void next_item(const ChunkArgs &a, const Ws &ws, const Part &p, Walk &w, Item &it, bool describe)
{
    const int tt = tile_tokens<D>(a), per = Cfg<D>::STREAMS * tt;
    it.tiles = 0;
    while (w.u < p.u1 && it.tiles == 0) {
        const Seq &s = w.s;
        if (w.i >= s.items) {          // (a sequence without work has no items)
            w.i = 0;
            if (s.items == 0 || ++w.h >= a.c.H_kv) {
                int st;
                w.h = 0, ++w.b;
                w.s = load_seq<D>(a, w.b, &st);
            }
            continue;
        }
        it.b = w.b, it.h = w.h, it.lo = s.lo, it.len = s.len;
        it.t0 = w.i * per, it.tokens = min(per, s.n - it.t0);
        it.pair = it.tokens > tt;
        const int p0 = s.len + it.t0, p1 = p0 + it.tokens - 1;
        const int low = a.window > p0 ? 0 : p0 - a.window + 1;
        it.low_tile = low / KT;
        it.sink_tiles = min((min(a.sinks, low) + (KT - 1)) / KT, it.low_tile);
        it.kts = it.sink_tiles + p1 / KT - it.low_tile + 1;
        const long long keys = it.tokens + min((long long)p0, (long long)a.window + a.sinks - 1);
        const long long span = min(START + keys - w.o, p.u1 - w.u), begin = w.u - w.o;
        const bool to_end = w.o + span == START + keys;
        it.j0 = w.o <= START ? 0 : tiles_before(w.o, keys, it.kts);
        const int j1 = to_end ? it.kts : tiles_before(w.o + span, keys, it.kts);
        it.tiles = j1 - it.j0;
        const bool cut = it.j0 > 0 || j1 < it.kts;
        it.slot = !cut ? -1 : begin <= p.u0 ? 2 * p.group : 2 * p.group + 1;
        if (describe && cut && it.j0 == 0 && it.tiles > 0) {
            int *d = ws.desc + 8 * p.group;
            const long long last = begin + START + (long long)(it.kts - 1) * keys / it.kts;
            d[1] = it.slot, d[2] = it.lo + it.t0, d[3] = it.h, d[4] = it.tokens, d[5] = it.b, d[6] = p.group;
            d[0] = part_of(last, p.W, p.parts) - p.group + 1;
        }
        w.u += span, w.o += span;
        if (to_end) w.o = 0, ++w.i;
    }
}

// After a wait that ran out: from item `unfinished` on, this CTA's blocks say that they are not there and the sequences are
// flagged.
template <int D> static __device__ __noinline__ void mark_unfinished(const ChunkArgs &a, const Ws &ws, const Part &p, Walk w, unsigned unfinished, int tid, int threads)
{
    Item it;
    for (unsigned ord = 0;; ++ord) {
        next_item<D>(a, ws, p, w, it, false);
        if (it.tiles == 0) return;
        if (ord < unfinished) continue;
        if (it.slot >= 0)
            for (int r = tid; r < ws.cap; r += threads)
                reinterpret_cast<float2 *>(ws.ml)[(long long)it.slot * ws.cap + r] = make_float2(0.f, NOT_DONE);
        if (tid == 0 && a.seq_status) atomicOr(&a.seq_status[it.b], TREEWY_SEQ_TIMEOUT);
    }
}

// What one stream sees of an item: positions of its first and last row.
struct View {
    int p0, p1;
};
__device__ __forceinline__ View view_of(const Item &it, int tt, int s)
{
    const int first = it.pair ? s * tt : 0, last = it.pair && s == 0 ? tt : it.tokens;
    return {it.len + it.t0 + first, it.len + it.t0 + last - 1};
}
// The same for whole tiles kt: some row sees some of one if kt <= high_some and kt >= low_some or kt < sink_some, every row all of it if
// kt < high_all and kt >= low_all or kt < sink_all.
struct Span {
    int sink_some, low_some, high_some, sink_all, low_all, high_all;
};
__device__ __forceinline__ Span span_of(const ChunkArgs &a, const View &v)
{
    const int from0 = a.window > v.p0 ? 0 : v.p0 - a.window + 1, from1 = a.window > v.p1 ? 0 : v.p1 - a.window + 1;
    return {a.sinks > 0 ? (a.sinks - 1) / KT + 1 : 0, from0 / KT, v.p1 / KT, a.sinks / KT, from1 > 0 ? (from1 - 1) / KT + 1 : 0, (v.p0 + 1) / KT};
}
// The cache's tile for tile j of an item's tiles here
struct Tiles {
    int sinks, first, then;
    __device__ __forceinline__ explicit Tiles(const Item &it) : sinks(it.sink_tiles - it.j0), first(it.j0), then(it.low_tile - it.sink_tiles + it.j0) {}
    __device__ __forceinline__ int operator()(int j) const { return j + (j < sinks ? first : then); }
};
// A stream's part in an item's tiles here.  With two row tiles: j < hole (the sinks') and from `on_again` to `end`, else (as far as
// this goes) all.  Those that every row sees whole: j < sinks_whole, and from `whole` to `whole_end`.  (Tiles of the window may be the
// sinks' too.)
struct Turns {
    int hole, on_again, end, sinks_whole, whole, whole_end;
    __device__ __forceinline__ bool some(int j) const { return j < end && (j < hole || j >= on_again); }
    __device__ __forceinline__ bool all(int j) const { return j < sinks_whole || (j >= whole && j < whole_end); }
    __device__ __forceinline__ int at_or_after(int j) const { return j >= hole && j < on_again ? on_again : j; }
};
__device__ __forceinline__ Turns turns_of(const Item &it, const Span &s, bool pair)
{
    const Tiles tiles(it);
    const int n = it.tiles, sink_part = max(min(tiles.sinks, n), 0);
    auto below = [&](int kt) { return kt - tiles.first <= sink_part ? kt - tiles.first : max(sink_part, kt - tiles.then); };  // tiles j before the cache's kt
    Turns t;
    t.end = pair ? min(n, max(sink_part, s.high_some - tiles.then + 1)) : n;
    t.hole = pair ? min(t.end, below(max(s.sink_some, tiles.first + sink_part))) : n;
    t.on_again = pair ? max(t.hole, s.low_some - tiles.then) : n;
    t.sinks_whole = below(min(s.sink_all, s.high_all));
    t.whole = max(sink_part, s.low_all - tiles.then), t.whole_end = s.high_all - tiles.then;
    return t;
}
// Whether some row of the view sees some token of tokens x0 .. x0 + n - 1
__device__ __forceinline__ bool sees_some(const ChunkArgs &a, const View &v, int x0, int n)
{
    return x0 <= v.p1 && ((long long)x0 + n - 1 > (long long)v.p0 - a.window || x0 < a.sinks);
}
// Whether every row sees all of them
__device__ __forceinline__ bool sees_all(const ChunkArgs &a, const View &v, int x0, int n)
{
    return x0 + n - 1 <= v.p0 && ((long long)x0 > (long long)v.p1 - a.window || x0 + n <= a.sinks);
}
__device__ __forceinline__ bool sees(const ChunkArgs &a, int p, int x) { return x <= p && (p - x < a.window || x < a.sinks); }

__device__ __forceinline__ uint32_t low32(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }
__device__ __forceinline__ bool nonfinite2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
// a wait with one outcome for the whole warp: what follows needs all of its lanes
__device__ __forceinline__ bool wait_warp(uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity)); }

template <int D>
__global__ void __launch_bounds__(Cfg<D>::THREADS, 1)
chunk_tc_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ Ws ws, Layout lay, int smem_bytes, const __grid_constant__ CUtensorMap map_q,
                const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using C = Cfg<D>;
    // barriers and the like first, tiles behind them: the bytes that aligning the tiles takes are used so
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Shared<D> &sh = *reinterpret_cast<Shared<D> *>(smem_raw);
    unsigned char *q_tiles = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw + sizeof(Shared<D>)) + 1023) & ~uintptr_t(1023));
    unsigned char *k_ring = q_tiles + C::STREAMS * C::Q_TILE, *v_ring = k_ring + C::NK * C::STAGE;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        ptx::wait_deadline_init(a.wait_cycles);
#pragma unroll 1
        for (int i = 0; i < C::NK; ++i) ptx::mbar_init(&sh.k_full[i], 1), ptx::mbar_init(&sh.k_free[i], C::STREAMS);
#pragma unroll 1
        for (int i = 0; i < C::NV; ++i) ptx::mbar_init(&sh.v_full[i], 1), ptx::mbar_init(&sh.v_free[i], C::STREAMS);
        for (int i = 0; i < 4; ++i) ptx::mbar_init(&sh.s_full[i], 1), ptx::mbar_init(&sh.p_full[i], 4), ptx::mbar_init(&sh.pv_done[i], 1);
        for (int i = 0; i < 2; ++i) ptx::mbar_init(&sh.o_free[i], O_FREE_ARRIVALS);
        ptx::mbar_init(&sh.q_full, 1), ptx::mbar_init(&sh.q_free, C::STREAMS), ptx::mbar_init(&sh.end[0], 1), ptx::mbar_init(&sh.end[1], 1);
        for (int i = 0; i < 4; ++i) ptx::mbar_init(&sh.ml_full[i], 1);
        for (int i = 0; i < ITEMS; ++i) ptx::mbar_init(&sh.item_full[i], 1), ptx::mbar_init(&sh.item_empty[i], C::SOFT_WARPS + 3);
        ptx::fence_barrier_init();
        sh.unfinished = ~0u, sh.first_b = -1;
        sh.copied[0] = sh.copied[1] = sh.q_copied = 0;
        ptx::prefetch_tmap(&map_q), ptx::prefetch_tmap(&map_k), ptx::prefetch_tmap(&map_v);
    }
    if (tid < 8) sh.bad_item[tid] = 0, sh.nonfinite[tid] = 0;
    // (the tiles' end has been allowed for; were the base of shared memory aligned otherwise, nothing may run)
    const bool fits = q_tiles + C::TILES <= smem_raw + smem_bytes;
    if (warp == C::MMA) {
        ptx::tmem_alloc(&sh.tmem, 512);
        ptx::tmem_relinquish();
    }
    grid_dependency_wait();
    grid_dependency_trigger();

    // ---- the line of work and this CTA's part of it
    int st;
    const int chunk = (a.B + C::THREADS - 1) / C::THREADS, b_begin = min(a.B, tid * chunk), b_end = min(a.B, b_begin + chunk);
    long long sum = 0;
    Seq only;                    // a thread's one sequence is not read again
#pragma unroll 1
    for (int b = b_begin; b < b_end; ++b) {
        only = load_seq<D>(a, b, &st);
        sum += (long long)only.per * a.c.H_kv;
        if (!fits && only.items) st |= TREEWY_SEQ_TIMEOUT;
        if (st && blockIdx.x == 0 && a.seq_status) atomicOr(&a.seq_status[b], st);
    }
    long long incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) sh.scan[warp] = incl;
    if (tid == 0) ws.desc[8 * blockIdx.x] = 0;
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    long long before = 0, W = 0;
#pragma unroll
    for (int i = 0; i < C::THREADS / 32; ++i) {
        if (i < warp) before += sh.scan[i];
        W += sh.scan[i];
    }
    before += incl - sum;
    if (!fits) W = 0;
    const int group = blockIdx.x, parts = (int)max(1ll, min((long long)gridDim.x, W / MIN_UNITS));
    const long long u0 = group < parts && W > 0 ? part_begin(group, W, parts) : 0;
    const long long u1 = group < parts && W > 0 ? part_begin(group + 1, W, parts) : 0;
#pragma unroll 1
    for (int b = b_begin; b < b_end; ++b) {
        if (chunk > 1) only = load_seq<D>(a, b, &st);
        const long long units = (long long)only.per * a.c.H_kv;
        if (u1 > u0 && u0 >= before && u0 < before + units) sh.first_b = b, sh.first_off = u0 - before, sh.first_seq = only;
        before += units;
    }
    if (tid == 0) sh.part = {u0, u1, W, parts, group};
    __syncthreads();
    const uint32_t tmem = sh.tmem;
    const int tt = tile_tokens<D>(a);
    if (warp == C::PRODUCER_K || warp == C::PRODUCER_V) {
        // ---------------------------------------------------------------- TMA copies: one thread each; that of V also finds the items
        // (A thread alone takes some 6 cycles for an instruction: what it does for a tile is kept short.)
        if (ptx::elect_one()) {
            const int ps = 1 << a.log_page;
            unsigned filled = 0;    // tiles whose copies were issued
            // (returns early when a wait runs out)
            auto run = [&](auto box_, auto is_v_) {
                constexpr int BOX = decltype(box_)::value;
                constexpr bool IS_V = decltype(is_v_)::value;
                using B = Boxes<D, BOX>;
                const CUtensorMap *map = IS_V ? &map_v : &map_k;
                constexpr int NS = IS_V ? C::NV : C::NK;
                uint64_t *const fulls = IS_V ? sh.v_full : sh.k_full, *const frees = IS_V ? sh.v_free : sh.k_free;
                const uint32_t ring = ptx::smem_u32(IS_V ? v_ring : k_ring);
                unsigned stage = 0, phase = 0;  // of the next tile
                Walk walk = walk_from<D>(a, IS_V ? sh.first_b : -1, sh.first_off, u0, sh.first_seq);
                const Part part{u0, u1, W, parts, group};
                unsigned found = 0;     // items
                auto find = [&]() -> bool {
                    Item it;
                    // (the limit is an item's: a long call's items may take seconds in all)
                    ptx::wait_deadline_init(a.wait_cycles);
                    next_item<D>(a, ws, part, walk, it, true);
                    if (found >= ITEMS && !ptx::mbar_wait(&sh.item_empty[found % ITEMS], (found / ITEMS - 1) & 1)) return false;
                    sh.items[found % ITEMS] = it;
                    ptx::mbar_arrive(&sh.item_full[found % ITEMS]);
                    ++found;
                    return true;
                };
                if (IS_V && !find()) return;
                for (unsigned ord = 0;; ++ord) {
                    const unsigned r = ord % ITEMS;
                    if (!IS_V && !ptx::mbar_wait(&sh.item_full[r], (ord / ITEMS) & 1)) return;
                    const Item it = sh.items[r];
                    if (it.tiles == 0) return;
                    if (IS_V) {             // the next item, ahead of this one's copies
                        if (!find()) return;
                    } else {
                        ptx::mbar_arrive(&sh.item_empty[r]);
                    }
                    if (it.b * a.c.H_kv + it.h == a.skip_item) return;  // (test hook)
                    if constexpr (!IS_V) {  // the queries of the item
                        if (ord > 0 && !ptx::mbar_wait(&sh.q_free, (ord - 1) & 1)) return;
                        const int streams = C::STREAMS == 2 && it.pair ? 2 : 1;
                        sh.q_copied = ord + 1;
                        ptx::mbar_arrive_expect_tx(&sh.q_full, (uint32_t)(streams * C::NC * tt * a.G * 128));
                        for (int s = 0; s < streams; ++s)
#pragma unroll
                            for (int c = 0; c < C::NC; ++c)
                                ptx::tma_load_5d(q_tiles + s * C::Q_TILE + c * MT * 128, &map_q, 0, 0, it.lo + it.t0 + s * tt, c, it.h, &sh.q_full);
                    }
                    const int32_t *table = a.c.page_table + (size_t)it.b * a.c.max_pages;
                    const View all{it.len + it.t0, it.len + it.t0 + it.tokens - 1};
                    const Tiles tiles(it);
                    const int n = it.tiles, h = it.h;
                    // tiles of the cache of which every page is seen: what is needed of others is looked at page by page
                    const int low = a.window > all.p0 ? 0 : all.p0 - a.window + 1;
                    const int low_whole = low > 0 ? (low - 1) / KT + 1 : 0, high_whole = (all.p1 + 1) / KT, sinks_whole = a.sinks / KT;
                    auto look = [&](int j, int (&to)[B::P]) {
                        const int kt = tiles(j), x0 = kt * KT;
                        const int32_t *t = table + (x0 >> a.log_page);
                        if (kt < high_whole && (kt >= low_whole || kt < sinks_whole)) {
#pragma unroll
                            for (int i = 0; i < B::P; ++i) to[i] = t[i];
                        } else {
#pragma unroll
                            for (int i = 0; i < B::P; ++i) {
                                to[i] = UNSEEN;
                                if (sees_some(a, all, x0 + i * BOX, BOX)) {
                                    to[i] = t[i];
                                    if (to[i] == UNSEEN) to[i] = -1;
                                }
                            }
                        }
                    };
                    bool bad = false;
                    int next[B::P];
                    look(0, next);
#pragma unroll 1
                    for (int j = 0; j < n; ++j) {
                        int pages[B::P];
                        uint32_t bytes = BOX * C::NC * 128 * B::P;
                        bool odd = false;
#pragma unroll
                        for (int i = 0; i < B::P; ++i) pages[i] = next[i], odd |= (unsigned)pages[i] >= (unsigned)a.c.n_pages;
                        if (odd) {          // pages that no row sees, and such as there are not
#pragma unroll
                            for (int i = 0; i < B::P; ++i) {
                                if (pages[i] == UNSEEN) bytes -= BOX * C::NC * 128;
                                else if ((unsigned)pages[i] >= (unsigned)a.c.n_pages) bad = true, pages[i] = a.c.n_pages;  // (one past the pool reads as zeros)
                            }
                            if (bad && !IS_V) {
                                sh.bad_item[ord % 8] = ord + 1;
                                if (a.seq_status) atomicOr(&a.seq_status[it.b], TREEWY_SEQ_BAD_PAGE);
                            }
                        }
                        const int slot = BOX < KT ? 0 : tiles(j) * KT & (ps - 1);
                        if (j + 1 < n) look(j + 1, next);
                        if (!ptx::mbar_wait(&frees[stage], phase ^ 1)) return;  // (the first time round: the phase before the first)
                        ++filled;
                        const uint32_t dst = ring + stage * C::STAGE, full = ptx::smem_u32(&fulls[stage]);
                        ptx::mbar_arrive_expect_tx(full, bytes);
#pragma unroll
                        for (int i = 0; i < B::P; ++i) {
                            if (pages[i] == UNSEEN) continue;  // (left as it is, never used)
                            if constexpr (IS_V) {
                                ptx::tma_load_5d(dst + i * (BOX * C::NC * 128), map, 0, slot, 0, h, pages[i], full);
                            } else if constexpr (B::K_BY_CHUNK) {
#pragma unroll
                                for (int c = 0; c < C::NC; ++c) ptx::tma_load_5d(dst + i * (BOX * 128) + c * B::K_CHUNK, map, 0, slot, c, h, pages[i], full);
                            } else {
#pragma unroll
                                for (int g = 0; g < BOX / 8; ++g)
                                    ptx::tma_load_5d(dst + (i * (BOX / 8) + g) * B::K_GROUP, map, 0, slot + 8 * g, 0, h, pages[i], full);
                            }
                        }
                        if (++stage == NS) stage = 0, phase ^= 1;
                    }
                }
            };
            auto run_box = [&](auto box_) { return warp == C::PRODUCER_V ? run(box_, std::true_type{}) : run(box_, std::false_type{}); };
            if (lay.v_rows == 64) run_box(std::integral_constant<int, 64>{});
            else if (lay.v_rows == 32) run_box(std::integral_constant<int, 32>{});
            else if (lay.v_rows == 8) run_box(std::integral_constant<int, 8>{});
            else run_box(std::integral_constant<int, 16>{});
            sh.copied[warp == C::PRODUCER_V] = filled;
        }
        __syncwarp();
    } else if (warp >= C::MMA) {
        // ---------------------------------------------------------------- MMAs: a thread to each stream; of one stream, one to Q K^T and
        // one to P V (a single thread for all was the slowest role: what it does between two MMAs alone took as long as a tile)
        if (ptx::elect_one()) {
            constexpr uint32_t idesc_qk = ptx::umma_idesc_bf16_f32(MT, KT), idesc_pv = ptx::umma_idesc_bf16_f32_bmn(MT, D);
            const int me = warp - C::MMA, strm = C::STREAMS == 2 ? me : 0;
            // Descriptors: stages, streams and steps only add to the address, 16 bytes a unit in the low bits
            const uint64_t qd = ptx::umma_desc_k_sw128(ptx::smem_u32(q_tiles)), kd = ptx::umma_desc_k_sw128(ptx::smem_u32(k_ring), lay.k_group);
            const uint64_t q_hi = qd & ~0xffffffffull, k_hi = kd & ~0xffffffffull;
            const uint32_t q_lo = (uint32_t)qd, k_lo = (uint32_t)kd, k_chunk = lay.k_chunk / 16;
            uint64_t v_hi = 0;
            uint32_t v_lo[KT / 16];
#pragma unroll
            for (int s = 0; s < KT / 16; ++s) {  // a step of V is 16 rows
                const uint32_t off = ((16 * s) >> lay.log_v_rows) * (lay.v_rows * C::NC * 128) + ((16 * s) & (lay.v_rows - 1)) * 128;
                const uint64_t vd = ptx::umma_desc_mn_sw128(ptx::smem_u32(v_ring) + off, lay.v_rows * 128, lay.v_rows == 8 ? C::NC * 1024 : 1024);
                v_hi = vd & ~0xffffffffull, v_lo[s] = (uint32_t)vd;
            }
            const uint32_t tm_o = tmem + strm * D, tm_s = tmem + C::TM_S + strm * C::NB * KT;
            uint64_t *const s_full = sh.s_full + strm * C::NB, *const p_full = sh.p_full + strm * C::NB, *const pv_done = sh.pv_done + strm * C::NB;
            // stages of the rings and S buffers, and their phases
            unsigned k_stage = 0, k_phase = 0, v_stage = 0, v_phase = 0, made = 0, made_phase = 0, used = 0, used_phase = 0;
            unsigned uses = 0;             // items with products here: phases of o_free
            auto next_k = [&]() { if (++k_stage == C::NK) k_stage = 0, k_phase ^= 1; };
            auto next_v = [&]() { if (++v_stage == C::NV) v_stage = 0, v_phase ^= 1; };
            // scores of the next tile; ql: low word of the queries' descriptor
            auto scores = [&](uint32_t ql) -> bool {
                // (the buffer's last product is done; in the other case the same thread has issued it before)
                if (C::STREAMS == 1 && !ptx::mbar_wait(&pv_done[made], made_phase ^ 1)) return false;
                if (!ptx::mbar_wait(&sh.k_full[k_stage], k_phase)) return false;
                ptx::tc_fence_after_sync();
                const uint32_t lo = k_lo + k_stage * (C::STAGE / 16), to = tm_s + made * KT;
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
                    ptx::umma_bf16(to, q_hi | (ql + (c / 4) * (MT * 128 / 16) + (c % 4) * 2), k_hi | (lo + (c / 4) * k_chunk + (c % 4) * 2), idesc_qk, c > 0);
                ptx::umma_commit(&s_full[made]);
                ptx::umma_commit(&sh.k_free[k_stage]);
                if (++made == C::NB) made = 0, made_phase ^= 1;
                next_k();
                return true;
            };
            // output of the next tile
            auto product = [&](bool onto) -> bool {
                if (!onto) {               // the output of the use before this one has been read
                    if (uses > 0 && !ptx::mbar_wait(&sh.o_free[strm], (uses - 1) & 1)) return false;
                    ++uses;
                }
                if (!ptx::mbar_wait(&sh.v_full[v_stage], v_phase)) return false;
                if (!ptx::mbar_wait(&p_full[used], used_phase)) return false;
                ptx::tc_fence_after_sync();
                const uint32_t at = v_stage * (C::STAGE / 16), from = tm_s + used * KT;
#pragma unroll
                for (int c = 0; c < KT / 16; ++c) ptx::umma_bf16_ts(tm_o, from + c * 8, v_hi | (v_lo[c] + at), idesc_pv, onto || c > 0);
                ptx::umma_commit(&pv_done[used]);
                ptx::umma_commit(&sh.v_free[v_stage]);
                if (++used == C::NB) used = 0, used_phase ^= 1;
                next_v();
                return true;
            };
            // a tile that this stream takes no part in: its stages are free as far as this thread goes (once they are filled: an
            // arrival ahead of that would count for the tile before)
            auto pass_k = [&]() -> bool {
                if (!ptx::mbar_wait(&sh.k_full[k_stage], k_phase)) return false;
                ptx::mbar_arrive(&sh.k_free[k_stage]);
                next_k();
                return true;
            };
            auto pass_v = [&]() -> bool {
                if (!ptx::mbar_wait(&sh.v_full[v_stage], v_phase)) return false;
                ptx::mbar_arrive(&sh.v_free[v_stage]);
                next_v();
                return true;
            };
            auto run = [&]() -> bool {
                for (unsigned ord = 0;; ++ord) {
                    const unsigned r = ord % ITEMS;
                    if (!ptx::mbar_wait(&sh.item_full[r], (ord / ITEMS) & 1)) return false;
                    const Item it = sh.items[r];
                    if (it.tiles == 0) return true;
                    ptx::mbar_arrive(&sh.item_empty[r]);
                    const int n = it.tiles;
                    const bool pair = C::STREAMS == 2 && it.pair;
                    // Scores run `ahead` tiles ahead of the products: as many as there are S buffers for.
                    const int ahead = pair || C::STREAMS == 1 ? C::NB : 2 * C::NB;
                    const Turns turns = turns_of(it, span_of(a, view_of(it, tt, strm)), pair);
                    // whether this stream takes part in tile j: with two row tiles as far as it sees some of it, else in turn
                    auto on = [&](int j) { return C::STREAMS == 1 || (pair ? turns.some(j) : (j & 1) == strm); };
                    const uint32_t ql = q_lo + (pair ? strm : 0) * (C::Q_TILE / 16);
                    const bool does_qk = C::STREAMS == 2 || me == 0, does_pv = C::STREAMS == 2 || me == 1;
                    if (does_qk && !ptx::mbar_wait(&sh.q_full, ord & 1)) return false;
                    bool onto = false;
#pragma unroll 1
                    for (int t = 0; t < n + ahead; ++t) {  // scores of tile t, products of tile j
                        const int j = t - ahead;
                        if (does_pv && j >= 0) {
                            if (on(j)) {
                                if (!product(onto)) return false;
                                onto = true;
                            } else if (!pass_v()) {
                                return false;
                            }
                        }
                        if (does_qk && t < n) {
                            if (on(t)) {
                                if (!scores(ql)) return false;
                            } else if (!pass_k()) {
                                return false;
                            }
                            if (t + 1 == n) ptx::umma_commit(&sh.q_free);
                        }
                    }
                }
            };
            if (!run()) {  // MMAs in flight have to end before the CTA may leave: a commit behind all of them, on a barrier of its own
                ptx::umma_commit(&sh.end[me]);
                for (int t = 0; t < 100000 && !ptx::mbar_try_wait(&sh.end[me], 0); ++t) __nanosleep(20);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- softmax, epilogue
        const int strm = C::STREAMS == 1 ? 0 : warp >> 2, w4 = warp & 3, row = w4 * 32 + lane;  // this warpgroup's stream; a row to a thread
        const uint32_t lane_base = (uint32_t)(w4 * 32) << 16;
        const float sl2 = a.scale * 1.4426950408889634f;
        const int tok = row / a.G;    // this row's token in a row tile
        unsigned count = 0;           // the stream's tiles so far
        unsigned g0 = 0, ord = 0, singles = 0;
        auto wait_product = [&](unsigned i) { return wait_warp(&sh.pv_done[strm * C::NB + i % C::NB], (i / C::NB) & 1); };  // of this stream's tile i
        auto run = [&]() -> bool {
            for (;; ++ord) {
                if (!wait_warp(&sh.item_full[ord % ITEMS], (ord / ITEMS) & 1)) return false;
                const Item &it = sh.items[ord % ITEMS];
                const int n = it.tiles;
                if (n == 0) return true;
                const bool pair = C::STREAMS == 2 && it.pair;
                const View v = view_of(it, tt, pair ? strm : 0), all{it.len + it.t0, it.len + it.t0 + it.tokens - 1};
                const Tiles tiles(it);
                const int rows = (v.p1 - v.p0 + 1) * a.G;
                const bool warp_on = w4 * 32 < rows, on = row < rows;
                const int p = v.p0 + (on ? tok : 0);  // this row's position
                const int step = pair || C::STREAMS == 1 ? 1 : 2;
                const Turns turns = turns_of(it, span_of(a, v), pair);
                float m = -INFINITY, l = 0.f;
                int taken = 0;             // tiles of this stream
                uint32_t x[KT];            // a row of S
                bool loaded = false;       // (its next tile's is on its way there)
                for (int j = turns.at_or_after(step == 1 ? 0 : strm), next; j < turns.end; j = next) {
                    const int buf = strm * C::NB + count % C::NB;
                    const bool masked = !turns.all(j);
                    const uint32_t ts = tmem + lane_base + C::TM_S + buf * KT;
                    auto load = [&](uint32_t from) {
#pragma unroll
                        for (int c = 0; c < KT; c += 32) ptx::tmem_ld32(from + c, *reinterpret_cast<uint32_t(*)[32]>(&x[c]));
                    };
                    if (!loaded) {
                        if (!wait_warp(&sh.s_full[buf], (count / C::NB) & 1)) return false;
                        ptx::tc_fence_after_sync();
                        if (warp_on) load(ts);
                    }
                    next = turns.at_or_after(j + step);
                    loaded = false;
                    bool ready = false;
                    if (warp_on) {
                        ptx::tmem_wait_ld();
                        if (masked) {
                            __syncwarp();  // (a branch, not predicated instructions for every tile)
                            const int x0 = tiles(j) * KT;
                            const int hi = min(p - x0, KT) + 1, from = (int)max((long long)p - a.window + 1 - x0, -1ll), sk = (int)max((long long)a.sinks - x0, -1ll);
#pragma unroll
                            for (int c = 0; c < KT; c += 32) {
                                const uint32_t bits = low32(hi - c) & (~low32(from - c) | low32(sk - c));
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (!(bits & (1u << i))) x[c + i] = 0xff800000u;
                            }
                        }
                        // Weights against the reference as it is; if they come out too large, or there is none yet, it becomes the maximum.
                        bool anew = __any_sync(0xffffffffu, on && m == -INFINITY);
                        float2 acc[2];
                        uint32_t w[KT / 2];
#pragma unroll 1
                        for (;;) {
                            if (anew) {
                                float t[2] = {-INFINITY, -INFINITY};
#pragma unroll
                                for (int i = 0; i < KT; i += 2) t[(i >> 1) & 1] = ptx::max3_nan(t[(i >> 1) & 1], __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
                                const float top = ptx::max3_nan(t[0], t[1], t[1]) * sl2 + ABOVE, m0 = m;
                                // (a NaN or plus infinity there makes the row NaN, by its sum)
                                m = top > m0 || top != top ? top : m0;
                                const float f = m == m0 ? 1.f : ptx::ex2(m0 - m);
                                l *= f;
                                if (taken > 0) {
                                    // O at rest: the stream's product before this one is done, and the next one waits for these weights
                                    if (!wait_product(count - 1)) return false;
                                    ptx::tc_fence_after_sync();
#pragma unroll 1
                                    for (int c = 0; c < D; c += 16) {
                                        uint32_t o[16];
                                        const uint32_t to = tmem + lane_base + strm * D + c;
                                        ptx::tmem_ld16(to, o);
                                        ptx::tmem_wait_ld();
#pragma unroll
                                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                        ptx::tmem_st16(to, o);
                                    }
                                }
                            }
                            const float ref = m == -INFINITY ? 0.f : m;
                            const float2 scale2 = make_float2(sl2, sl2), ref2 = make_float2(-ref, -ref);
                            acc[0] = acc[1] = make_float2(0.f, 0.f);
#pragma unroll
                            for (int i = 0; i < KT; i += 2) {
                                float2 y = ptx::fma2(make_float2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), scale2, ref2);
                                y.x = ptx::ex2(y.x), y.y = ptx::ex2(y.y);
                                acc[(i >> 1) & 1] = ptx::add2(acc[(i >> 1) & 1], y);
                                // weights as bf16: at most 2^-8 of each, independent from key to key
                                w[i / 2] = pack_bf16(y.x, y.y);
                            }
                            acc[0] = ptx::add2(acc[0], acc[1]);
                            acc[0].x += acc[0].y;
                            if (anew || !__any_sync(0xffffffffu, on && !(acc[0].x < LARGE))) break;
                            anew = true;
                        }
#pragma unroll
                        for (int c = 0; c < KT / 2; c += 16) ptx::tmem_st16(ts + c, *reinterpret_cast<const uint32_t(*)[16]>(&w[c]));
                        l += acc[0].x;
                        const unsigned nc = count + 1;
                        ready = next < turns.end && ptx::mbar_try_wait(&sh.s_full[strm * C::NB + nc % C::NB], (nc / C::NB) & 1);
                        ready = __all_sync(0xffffffffu, ready);
                        ptx::tmem_wait_st();
                    }
                    if (masked) {
                        // Values that a zero weight may not meet: tokens that no row of the item sees (not copied, or the page's unused
                        // slots) become zeros, and NaN and infinity in those that only some rows see are taken out; the
                        // epilogue adds them where they are seen.
                        const unsigned g = g0 + j, sidx = g % C::NV;
                        const int x0 = tiles(j) * KT;
                        // (where S runs further ahead than V's ring, the stage's last tile has to be done for its phase to mean this one)
                        if (C::NV < C::NB && count >= C::NV && !wait_product(count - C::NV)) return false;
                        if (!wait_warp(&sh.v_full[sidx], (g / C::NV) & 1)) return false;
                        unsigned char *vt = v_ring + sidx * C::STAGE;
                        constexpr int VR = C::NC * 8;  // 16-byte vectors of a row
                        // of the tile's keys: every row of this stream sees those up to `up` from `from` on or below `sk`, some row of the item
                        // those up to `up_any` from `from_any` on or below `sk`
                        const int up = v.p0 - x0, up_any = all.p1 - x0, sk = (int)max((long long)a.sinks - x0, -1ll);
                        const int from = (int)max((long long)v.p1 - a.window + 1 - x0, -1ll), from_any = (int)max((long long)all.p0 - a.window + 1 - x0, -1ll);
#pragma unroll 1
                        for (int i = w4 * 32 + lane; i < KT * VR; i += 128) {
                            const int key = i / VR, cc = i - key * VR;
                            if (key <= up && (key >= from || key < sk)) continue;
                            uint4 *at = reinterpret_cast<uint4 *>(vt + (key >> lay.log_v_rows) * (lay.v_rows * C::NC * 128) +
                                                                  ((cc >> 3) * lay.v_rows + (key & (lay.v_rows - 1))) * 128 + (cc & 7) * 16);
                            if (key > up_any || (key < from_any && key >= sk)) {
                                *at = make_uint4(0, 0, 0, 0);
                                continue;
                            }
                            uint4 y = *at;
                            if (nonfinite2(y.x) || nonfinite2(y.y) || nonfinite2(y.z) || nonfinite2(y.w)) {
                                sh.nonfinite[ord % 8] = ord + 1;  // (ahead of the value's going: who finds it gone finds this)
                                __threadfence_block();
                                uint32_t *yw = reinterpret_cast<uint32_t *>(&y);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if ((yw[e] & 0x7f80u) == 0x7f80u) yw[e] &= 0xffff0000u;
                                    if ((yw[e] & 0x7f800000u) == 0x7f800000u) yw[e] &= 0x0000ffffu;
                                }
                                *at = y;
                            }
                        }
                        ptx::fence_proxy_async();
                    }
                    // every warp's part of the values has to be clean before any of them is used: p_full counts all four
                    ptx::tc_fence_before_sync();
                    ptx::mbar_arrive_warp(&sh.p_full[buf]);
                    ++taken, ++count;
                    if (ready) {           // (behind the store: ahead of it the load holds that up)
                        loaded = true;
                        ptx::tc_fence_after_sync();
                        load(tmem + lane_base + C::TM_S + (strm * C::NB + count % C::NB) * KT);
                    }
                }
                // ---- end of the item
                if (taken > 0 && !wait_product(count - 1)) return false;
                ptx::tc_fence_after_sync();
                const int slot = it.slot;
                const long long orow = ((long long)it.lo + it.t0 + (p - all.p0)) * a.H_q + it.h * a.G + (row - tok * a.G);
                const int brow = (pair ? strm * MT : 0) + row;  // in the block
                // Alone in an item with one row tile, the first warpgroup joins both streams' outputs.
                bool second = false;       // the second stream's O counts
                float f0 = 1.f, f1 = 0.f;
                if (C::STREAMS == 2 && !pair && n > 1) {
                    // (the next item's m and l are written behind a product of that item, and so behind this use's o_free)
                    second = true;
                    if (strm == 1) {       // (its products are done, then)
                        sh.ml[row] = make_float2(m, l);
                        ptx::tc_fence_before_sync();
                        ptx::mbar_arrive_warp(&sh.ml_full[w4]);
                    } else {
                        if (!wait_warp(&sh.ml_full[w4], singles & 1)) return false;
                        ptx::tc_fence_after_sync();
                    }
                    ++singles;
                    if (strm == 0) {
                        const float2 x = sh.ml[row];
                        const float mn = fmaxf(m, x.x), ref = mn == -INFINITY ? 0.f : mn;
                        f0 = ptx::ex2(m - ref), f1 = ptx::ex2(x.x - ref);
                        l = l * f0 + x.y * f1, m = mn;
                    }
                }
                // (behind the wait for the other stream, whose tiles may be the ones that met something)
                const bool bad = sh.bad_item[ord % 8] == ord + 1, fix = sh.nonfinite[ord % 8] == ord + 1;
                const bool writes = C::STREAMS == 1 || pair || strm == 0;
                const float inv = l == 0.f ? 0.f : 1.f / l;  // (a row that saw nothing has 0 everywhere)
                __nv_bfloat16 *const out_row = static_cast<__nv_bfloat16 *>(a.O) + orow * D;
                float *const blk = ws.o + (long long)slot * ws.cap * D;
                const bool wide = (reinterpret_cast<uintptr_t>(a.O) & 31) == 0;
                if (writes && warp_on) {
                    if (slot >= 0 && on) reinterpret_cast<float2 *>(ws.ml)[(long long)slot * ws.cap + brow] = make_float2(m, bad ? PAGE_BAD : l);
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        if (taken > 0) {
                            ptx::tmem_ld32(tmem + lane_base + (pair ? strm : 0) * D + c, o);
                            ptx::tmem_wait_ld();
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = 0;
                        }
                        if (second) {
                            uint32_t o1[32];
                            ptx::tmem_ld32(tmem + lane_base + D + c, o1);
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f0 + __uint_as_float(o1[i]) * f1);
                        }
                        if (!on) continue;
                        if (slot < 0) {
                            if (!bad) {
#pragma unroll
                                for (int i = 0; i < 32; i += 2) o[i / 2] = pack_bf16(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv);
                                if (wide) {  // whole sectors
                                    ptx::st_global_32(out_row + c, *reinterpret_cast<const uint32_t(*)[8]>(&o[0]));
                                    ptx::st_global_32(out_row + c + 16, *reinterpret_cast<const uint32_t(*)[8]>(&o[8]));
                                } else {
#pragma unroll
                                    for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4 *>(out_row + c + 2 * i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                                }
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                *reinterpret_cast<uint4 *>(blk + ((long long)((c + i) / 4) * ws.cap + brow) * 4) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                        }
                    }
                    __syncwarp();
                }
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {  // all read: the next products may overwrite it
                    const bool apart = C::STREAMS == 1 || pair;
#pragma unroll
                    for (int s = 0; s < C::STREAMS; ++s)
                        if (frees_output(apart, strm, s, apart ? taken > 0 : s < n)) ptx::mbar_arrive(&sh.o_free[s]);
                }
                if (writes && warp_on && fix && on && !bad) {
                    // Values with NaN or infinity in masked tiles: those elements, onto what was stored.  (Of two streams either may have
                    // taken them out: what not every row of both sees.)
                    const int32_t *table = a.c.page_table + (size_t)it.b * a.c.max_pages;
#pragma unroll 1
                    for (int j = 0; j < n; ++j) {
                        const int x0 = tiles(j) * KT;
                        if (sees_all(a, all, x0, KT)) continue;
#pragma unroll 1
                        for (int x = x0; x < x0 + KT; ++x) {
                            if (!sees(a, p, x) || sees_all(a, all, x, 1)) continue;
                            const __nv_bfloat16 *vr = static_cast<const __nv_bfloat16 *>(a.c.v) + table[x >> a.log_page] * a.c.stride_page +
                                                      (x & ((1 << a.log_page) - 1)) * a.c.stride_slot + it.h * a.c.stride_head;
#pragma unroll 1
                            for (int c = 0; c < D; ++c) {
                                const float y = to_f32(vr[c]);
                                if (isfinite(y)) continue;
                                if (slot < 0) out_row[c] = __float2bfloat16_rn(to_f32(out_row[c]) + y);
                                else blk[((long long)(c / 4) * ws.cap + brow) * 4 + c % 4] += y;
                            }
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sh.item_empty[ord % ITEMS]);
                g0 += n;
            }
        };
        if (!run()) {
            ptx::tmem_wait_st();
            if (lane == 0) atomicMin(&sh.unfinished, ord);
        }
        __syncwarp();
        ptx::tc_fence_before_sync();
        ptx::named_arrive(1, C::THREADS);
        return;
    }
    // ---- what is left when all have come to their end: the other warpgroup's work
    ptx::tc_fence_before_sync();
    ptx::named_sync(1, C::THREADS);
    ptx::tc_fence_after_sync();
    const int rest = tid - C::SOFT_WARPS * 32;
    if (sh.unfinished != ~0u) {
        if (rest < 2) {  // copies in flight have to land before the CTA may leave
            const unsigned filled = sh.copied[rest], ns = rest ? C::NV : C::NK;
            uint64_t *fulls = rest ? sh.v_full : sh.k_full;
            for (unsigned i = filled > ns ? filled - ns : 0; i < filled; ++i)
                for (int t = 0; t < 100000 && !ptx::mbar_try_wait(&fulls[i % ns], (i / ns) & 1); ++t) __nanosleep(20);
            if (rest == 0 && sh.q_copied > 0)
                for (int t = 0; t < 100000 && !ptx::mbar_try_wait(&sh.q_full, (sh.q_copied - 1) & 1); ++t) __nanosleep(20);
        }
        mark_unfinished<D>(a, ws, sh.part, walk_from<D>(a, sh.first_b, sh.first_off, sh.part.u0, sh.first_seq), sh.unfinished, rest, 128);
    }
    ptx::named_sync(2, 128);
    if (warp == C::MMA) ptx::tmem_dealloc(tmem, 512);
}

// The join: o = sum_p 2^{m_p - m} o_p / sum_p 2^{m_p - m} l_p over the parts p of an item in the order of its keys.  A warp
// takes 8 rows and 16 STEPS columns of them: lane = row + 8 * column group, 4 groups of 4 columns a step, so that both the
// blocks (8 rows of a group are 128 bytes) and the output (4 groups of a row are 32) move in whole sectors.  UN parts are loaded
// at a time.  A part with a bad page, or one that was not worked out, has a negative l: the row is left.
constexpr int JOIN_WARPS = 8;
template <int D, int STEPS, int UN>
__global__ void __launch_bounds__(JOIN_WARPS * 32) chunk_tc_join_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ Ws ws)
{
    constexpr int CW = D / (16 * STEPS);         // warps that share a row
    const int w = blockIdx.y * JOIN_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31, cg = lane >> 3;
    const int row = w / CW * 8 + (lane & 7), c0 = w % CW * (16 * STEPS);
    grid_dependency_wait();
    grid_dependency_trigger();
    const int4 d0 = *reinterpret_cast<const int4 *>(ws.desc + 8 * blockIdx.x), d1 = *reinterpret_cast<const int4 *>(ws.desc + 8 * blockIdx.x + 4);
    const int pieces = min(d0.x, MAX_CTAS), tt = MT / a.G;  // (calls that overlap on one workspace overwrite each other's: whatever lies there stays within it)
    const int first = row / MT * tt, in_tile = row % MT, token = first + in_tile / a.G;
    if (pieces <= 0 || token >= d1.x || in_tile >= tt * a.G || d1.z != (int)blockIdx.x || (unsigned)d0.y >= 2u * gridDim.x || d1.z + pieces > (int)gridDim.x) return;
    float m = -INFINITY, l = 0.f;
    int bad = 0;
    float4 acc[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int p0 = 0; p0 < pieces; p0 += UN) {
        float2 x[UN];
        float4 y[UN][STEPS];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int p = min(p0 + i, pieces - 1);
            const long long blk = (long long)(p == 0 ? d0.y : 2 * (d1.z + p)) * ws.cap;
            x[i] = __ldcs(reinterpret_cast<const float2 *>(ws.ml) + blk + row);
#pragma unroll
            for (int e = 0; e < STEPS; ++e) y[i][e] = __ldcs(reinterpret_cast<const float4 *>(ws.o + blk * D + ((long long)(c0 / 4 + 4 * e + cg) * ws.cap + row) * 4));
        }
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            if (p0 + i >= pieces) continue;
            if (x[i].y < 0.f) bad = 1;
            if (x[i].y == 0.f) continue;  // saw nothing
            const float mn = fmaxf(m, x[i].x), ref = mn == -INFINITY ? 0.f : mn;
            const float f0 = ptx::ex2(m - ref), f1 = ptx::ex2(x[i].x - ref);
            m = mn, l = l * f0 + x[i].y * f1;
#pragma unroll
            for (int e = 0; e < STEPS; ++e) {
                acc[e].x = acc[e].x * f0 + y[i][e].x * f1, acc[e].y = acc[e].y * f0 + y[i][e].y * f1;
                acc[e].z = acc[e].z * f0 + y[i][e].z * f1, acc[e].w = acc[e].w * f0 + y[i][e].w * f1;
            }
        }
    }
    if (bad) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const long long orow = ((long long)d0.z + token) * a.H_q + (long long)d0.w * a.G + in_tile % a.G;
    __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(a.O) + orow * D + c0;
#pragma unroll
    for (int e = 0; e < STEPS; ++e)
        *reinterpret_cast<uint2 *>(out + 16 * e + 4 * cg) =
            make_uint2(pack_bf16(acc[e].x * inv, acc[e].y * inv), pack_bf16(acc[e].z * inv, acc[e].w * inv));
}

// rows of a block: an item's, as far as the batch can have them
template <int D> int cap_of(const ChunkArgs &a)
{
    const long long rows = ((long long)a.T * a.G + 7) / 8 * 8;
    // (a second row tile starts at row 128 of the block whatever the first one holds)
    return (int)(a.T <= MT / a.G ? (rows < MT ? rows : MT) : Cfg<D>::CAP);
}
size_t desc_bytes() { return (size_t)MAX_CTAS * 8 * sizeof(int); }
template <int D> size_t workspace_of(const ChunkArgs &a) { return desc_bytes() + 2ull * MAX_CTAS * cap_of<D>(a) * (D + 2) * sizeof(float); }

template <int D> cudaError_t launch_d(ChunkArgs a, cudaStream_t stream)
{
    using C = Cfg<D>;
    int dev = 0, sms = 0;
    cudaError_t e = current_device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    const int ctas = sms < MAX_CTAS ? sms : MAX_CTAS;
    Ws ws;
    ws.cap = cap_of<D>(a);
    ws.desc = reinterpret_cast<int *>(a.ws);
    ws.o = reinterpret_cast<float *>(reinterpret_cast<unsigned char *>(a.ws) + desc_bytes());
    ws.ml = ws.o + 2ull * MAX_CTAS * ws.cap * D;
    a.log_page = 0;
    while ((1 << a.log_page) < a.c.page_size) ++a.log_page;

    EncodeTiledFn enc = tma_encode_fn();
    if (!enc) return cudaErrorNotSupported;
    CUtensorMap q, k, v;
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
    auto map5 = [&](CUtensorMap *m, const void *base, const cuuint64_t (&dims)[5], const cuuint64_t (&strides)[4], const cuuint32_t (&bx)[5]) {
        const cuuint32_t es[5] = {1, 1, 1, 1, 1};
        return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(base), dims, strides, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    // (the stride of a dimension of one does not count, but has to be a legal one)
    const cuuint64_t cache_dims[5] = {64, (cuuint64_t)c.page_size, (cuuint64_t)C::NC, (cuuint64_t)c.H_kv, (cuuint64_t)c.n_pages};
    const cuuint64_t cache_strides[4] = {(cuuint64_t)c.stride_slot * 2, 128, c.H_kv > 1 ? (cuuint64_t)c.stride_head * 2 : 16,
                                         c.n_pages > 1 ? (cuuint64_t)c.stride_page * 2 : 16};
    const cuuint32_t k_box[5] = {64, (cuuint32_t)(by_chunk ? box : 8), (cuuint32_t)(by_chunk ? 1 : C::NC), 1, 1};
    const cuuint32_t v_box[5] = {64, (cuuint32_t)box, (cuuint32_t)C::NC, 1, 1};
    const cuuint64_t q_dims[5] = {64, (cuuint64_t)a.G, (cuuint64_t)a.T, (cuuint64_t)C::NC, (cuuint64_t)c.H_kv};
    const cuuint64_t q_strides[4] = {D * 2, (cuuint64_t)a.ld_q * 2, 128, (cuuint64_t)a.G * D * 2};
    const cuuint32_t q_box[5] = {64, (cuuint32_t)a.G, (cuuint32_t)(MT / a.G), 1, 1};
    if (!map5(&k, c.k, cache_dims, cache_strides, k_box) || !map5(&v, c.v, cache_dims, cache_strides, v_box) || !map5(&q, a.q, q_dims, q_strides, q_box))
        return cudaErrorInvalidValue;
    // (the kernel's static shared memory, a deadline, comes first; the tiles start at the next multiple of 1024 behind `Shared`)
    const int smem = (16 + (int)sizeof(Shared<D>) + 1023) / 1024 * 1024 - 16 + C::TILES;
    static_assert((16 + sizeof(Shared<D>) + 1023) / 1024 * 1024 + C::TILES <= 227 * 1024, "shared memory of a CTA");
    e = ensure_dynamic_smem(reinterpret_cast<const void *>(chunk_tc_kernel<D>), smem, dev);
    if (e != cudaSuccess) return e;
    e = launch_dependent(chunk_tc_kernel<D>, dim3(ctas), dim3(C::THREADS), smem, stream, a, ws, lay, smem, q, k, v);
    if (e != cudaSuccess) return e;
    auto join = [&](auto steps, auto un) {
        constexpr int STEPS = decltype(steps)::value;
        const int warps = (ws.cap + 7) / 8 * (D / (16 * STEPS));
        return launch_dependent(chunk_tc_join_kernel<D, STEPS, decltype(un)::value>, dim3(ctas, (warps + JOIN_WARPS - 1) / JOIN_WARPS), dim3(JOIN_WARPS * 32),
                                0, stream, a, ws);
    };
    return join(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
}

}  // namespace

// The line's units times the parts stay within 63 bits.
static bool units_fit(const ChunkArgs &a)
{
    const double items = (double)a.T * a.G / 64 + a.B, keys = (double)a.c.max_pages * a.c.page_size + START;
    return items * keys * a.c.H_kv * MAX_CTAS < 4e18;
}

bool chunk_tc_applies(const ChunkArgs &a, treewy_dtype_t io)
{
    const CacheView &c = a.c;
    const bool pow2 = (c.page_size & (c.page_size - 1)) == 0;
    // 8-row groups of the swizzle have to stay whole within a page; the tensor maps want a pool that exists and real strides
    return io == TREEWY_BF16 && (c.d == 64 || c.d == 128 || c.d == 256) && pow2 && c.page_size >= 8 && c.n_pages > 0 && c.max_pages > 0 &&
           c.stride_slot > 0 && (c.H_kv == 1 || c.stride_head > 0) && (c.n_pages == 1 || c.stride_page > 0) && a.G <= MT && units_fit(a);
}

size_t chunk_tc_workspace(const ChunkArgs &a)
{
    if (a.G > MT) return 0;
    return a.c.d == 256 ? workspace_of<256>(a) : a.c.d == 128 ? workspace_of<128>(a) : a.c.d == 64 ? workspace_of<64>(a) : 0;
}

cudaError_t launch_chunk_tc(const ChunkArgs &a, cudaStream_t stream)
{
    if (a.c.d == 256) return launch_d<256>(a, stream);
    if (a.c.d == 128) return launch_d<128>(a, stream);
    return launch_d<64>(a, stream);
}

}  // namespace treewy
