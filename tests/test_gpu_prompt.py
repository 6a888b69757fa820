"""The calls that take new rows through an attention layer, on the GPU against the operators in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import attn_util as au
from tests import prompt_util as pu

pytestmark = pytest.mark.gpu

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DEV = "cuda:0"


# ------------------------------------------------------------------------------------------ attention

CHUNKS = {
    "one row, nothing before": dict(L=[0], N=[1]),
    "one row behind one token": dict(L=[1], N=[1]),
    "no rows among others": dict(L=[5, 70, 0], N=[3, 0, 2]),
    "lengths around a tile": dict(L=[0, 1, 63, 64, 65, 127, 128], N=[128, 127, 65, 64, 1, 2, 129]),
    "decode": dict(L=[300, 1, 777, 0], N=[1, 1, 1, 1], Hq=16, Hkv=2),
    "five heads a group": dict(L=[200, 33], N=[40, 77], Hq=5, Hkv=1),
    "no grouping": dict(L=[40, 0], N=[150, 290], Hq=3, Hkv=3),
    "a wide group": dict(L=[10, 3], N=[9, 40], Hq=48, Hkv=1),
    "several row tiles": dict(L=[100, 0], N=[300, 257], Hq=8, Hkv=2),
    "head 128, page 8": dict(L=[150, 9], N=[70, 150], D=128, page=8),
    "head 128, page 64": dict(L=[150, 256], N=[200, 6], D=128, page=64),
    "head 256, page 32": dict(L=[321, 17], N=[130, 7], D=256, page=32, Hq=8, Hkv=1),
    "head 256, page 128": dict(L=[500, 129], N=[3, 200], D=256, page=128, Hq=4, Hkv=2),
    "page 256": dict(L=[700, 255, 256], N=[2, 30, 4], page=256),
    "odd page, odd head": dict(L=[50, 11], N=[30, 140], page=5, D=72),
    "long context": dict(L=[5000], N=[3], Hq=4, Hkv=1, D=128),
    "many short sequences": dict(L=[(7 * b) % 50 for b in range(150)], N=[b % 4 for b in range(150)], Hq=4, Hkv=2),
    "window": dict(L=[200, 0, 60], N=[100, 150, 5], window=50),
    "window and sinks": dict(L=[400, 0, 60], N=[100, 150, 5], window=64, sinks=4, D=128),
    "window of one": dict(L=[30, 0], N=[40, 140], window=1),
    "window of one, one sink": dict(L=[30, 0], N=[40, 140], window=1, sinks=1),
    "sinks past a tile": dict(L=[600, 150], N=[60, 90], window=100, sinks=130, D=128),
    "sinks wider than all": dict(L=[60, 0], N=[60, 9], window=10, sinks=1000),
    "sinks without a window": dict(L=[60], N=[60], sinks=4),
    "window wider than all": dict(L=[60, 0], N=[60, 9], window=1 << 20, sinks=3),
    "window, decode": dict(L=[3000, 70, 0, 513], N=[1, 1, 1, 1], window=512, sinks=4, Hq=16, Hkv=2, D=128),
    "window, head 256": dict(L=[900, 64], N=[150, 300], window=200, sinks=3, D=256, Hq=4, Hkv=1),
    "steep softmax": dict(L=[400, 64], N=[80, 5], q_scale=30.0),
}


def _case(name, dtype, seed=0):
    return pu.make_case(dtype=dtype, seed=seed, **CHUNKS[name])


def _check(c, O, generic, rows=None, steep=False):
    ref, size = pu.chunk_reference(c)
    if steep:  # scores 30 times as large: their rounding, and so the weights', grows with them
        size = size * 30
    pu.assert_chunk(c, O, ref, size, tensor_cores=c.dtype == BF16 and not generic, rows=rows)


@pytest.mark.parametrize("name", list(CHUNKS))
@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)], ids=["bf16", "bf16-generic", "f32"])
def test_chunk_matches_64_bits(name, dtype, generic):
    c = _case(name, dtype)
    O, status = pu.run_chunk(c, generic=generic)
    assert not any(status)
    _check(c, O, generic, steep="steep" in name)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts_agree(dtype):
    c = pu.make_case([150, 128, 333], [70, 1, 120], Hq=8, Hkv=2, D=128, dtype=dtype, window=200, sinks=5, seed=3)
    O, _ = pu.run_chunk(c)
    P, status = pu.run_chunk(c, layout="heads")
    assert not any(status) and torch.equal(O, P)


@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_what_a_row_may_not_see_never_spreads(dtype, generic, D):
    """NaN and infinities in the keys and values of some tokens: rows ahead of them, and rows whose window has left them, do
    not change."""
    c = pu.make_case([70, 3], [180, 20], Hq=4, Hkv=2, D=D, dtype=dtype, window=40, sinks=2, seed=5)
    bad = [(0, 75, math.nan), (0, 140, math.inf), (0, 200, -math.inf), (0, 249, math.nan), (1, 20, math.nan)]
    for b, x, y in bad:
        at = (int(c.table[b, x // c.page]), x % c.page)
        c.kc[at], c.vc[at] = y, y
    O, status = pu.run_chunk(c, generic=generic)
    assert not any(status)
    clean = torch.tensor([not any(bb == b and x in c.seen(c.L[b] + i) for bb, x, _ in bad) for b in range(2) for i in range(c.N[b])])
    assert clean.any() and not clean.all()
    _check(c, O, generic, rows=clean)
    assert not torch.isfinite(O[~clean]).all(-1).any(), "a row that sees NaN keys or values has to say so"


@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)])
def test_infinite_values_that_are_seen_come_through(dtype, generic):
    """Infinity in a value row alone: exactly its columns, in exactly the rows that see it."""
    c = pu.make_case([70], [100], Hq=4, Hkv=2, D=64, dtype=dtype, window=60, seed=6)
    for x, h, col, y in ((75, 1, 7, math.inf), (120, 0, 9, -math.inf), (169, 1, 3, math.inf)):
        c.vc[int(c.table[0, x // c.page]), x % c.page, h, col] = y
    O, _ = pu.run_chunk(c, generic=generic)
    want = torch.zeros(c.T, c.Hq, c.D)
    want[5:65, 2:, 7] = math.inf                     # positions 75 .. 134; heads 2, 3 read key/value head 1
    want[50:100, :2, 9] = -math.inf
    want[99:, 2:, 3] = math.inf
    inf = ~torch.isfinite(want)
    assert torch.equal(O[inf].float(), want[inf]) and torch.isfinite(O[~inf]).all()


@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)])
def test_bad_sequences_are_flagged_and_the_others_are_right(dtype, generic):
    c = pu.make_case([40, 50, 60, 30, 20], [20, 30, 9, 5, 6], Hq=4, Hkv=2, D=128, dtype=dtype, seed=8, poison=False)
    clean = torch.ones(c.T, dtype=torch.bool)
    lens = list(c.L)
    c.table[1, 2] = c.kc.shape[0]                    # a page past the pool
    c.table[2, 0] = -1
    c.L[3] = -1
    c.offsets = torch.cat([c.offsets[:-1], torch.tensor([c.T + 5], dtype=torch.int32)])   # the last range leaves the rows
    for b in (1, 2, 3, 4):
        clean[int(c.offsets[b]):int(c.offsets[b]) + c.N[b]] = False
    O, status = pu.run_chunk(c, generic=generic)
    assert status == [0, 64, 64, 128, 32]
    c.L, c.table[1, 2], c.table[2, 0] = lens, 0, 0   # (for the reference; those rows are not compared)
    _check(c, O, generic, rows=clean)


@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)])
def test_rows_of_no_sequence_are_left(dtype, generic):
    c = pu.make_case([40], [200], Hq=4, Hkv=2, D=128, dtype=dtype, seed=9, gaps=[5, 11])
    O, status = pu.run_chunk(c, generic=generic)
    assert not any(status) and (O[:5] == 7.25).all() and (O[205:] == 7.25).all()
    rows = torch.zeros(c.T, dtype=torch.bool)
    rows[5:205] = True
    _check(c, O, generic, rows=rows)


def test_more_sequences_than_threads_that_look_them_up():
    c = pu.make_case([b % 7 for b in range(1100)], [1 if b % 5 else 0 for b in range(1100)], Hq=2, Hkv=1, seed=10)
    for generic in (False, True):
        O, status = pu.run_chunk(c, generic=generic)
        assert not any(status)
        _check(c, O, generic)


# ------------------------------------------------------------------------------------------ norms

def _rope(T, rot, axes, interleaved, gen, top=300):
    table = au.rope_table(rot, top)
    positions = torch.randint(top, (axes, T), generator=gen, dtype=torch.int32)
    pair_axis = (torch.arange(rot // 2) * axes // (rot // 2)).to(torch.uint8) if axes > 1 else None
    return table, positions, pair_axis, interleaved


def _handle(rope):
    from paper_2608_20961_b200 import attention as at
    if rope is None:
        return None
    return at.Rope(*(None if r is None else r.to(DEV) for r in rope[:3]), interleaved=rope[3])


# T, H, d, rot (0: no rotation), axes, interleaved
NORMS = [(1, 1, 64, 64, 1, False), (7, 3, 128, 128, 1, False), (33, 24, 128, 64, 3, False), (5, 4, 256, 64, 3, True),
         (300, 5, 80, 48, 1, True), (9, 2, 72, 72, 2, False), (4, 8, 250, 128, 1, False), (2, 72, 2, 2, 1, False), (50, 6, 96, 0, 1, False),
         (1201, 8, 64, 32, 1, False), (6, 2, 252, 126, 1, True), (3, 5, 16, 0, 1, False)]


def _strided(x, pad):
    """x [T, H, d] as a column range of wider rows."""
    T, H, d = x.shape
    wide = torch.full((T, H * d + pad), 9.0, dtype=x.dtype, device=DEV)
    wide[:, :H * d] = x.reshape(T, H * d).to(DEV)
    return wide[:, :H * d].view(T, H, d)


def _norm_case(i, dtype, wdtype):
    T, H, d, rot, axes, inter = NORMS[i]
    gen = torch.Generator().manual_seed(i)
    x = (torch.randn(T, H, d, generator=gen) * torch.randn(T, H, 1, generator=gen).exp()).to(dtype)
    dy = torch.randn(T, H, d, generator=gen).to(dtype)
    w = (1 + 0.3 * torch.randn(d, generator=gen)).to(wdtype)
    return x, dy, w, _rope(T, rot, axes, inter, gen) if rot else None


# Errors: a sum of d <= 256 squares is at most 16 additions in a lane and 5 exchanges, so r is off by 11 steps of 2^-24 and its
# function's 2; three products and the rotation's three roundings more: below 2^-19 of |a| + |b| of a pair in all.  The
# result is rounded once.
@pytest.mark.parametrize("i", range(len(NORMS)))
@pytest.mark.parametrize("dtype,wdtype,plus_one", [(BF16, BF16, False), (BF16, F32, True), (F32, F32, False), (F32, BF16, True)])
def test_norm_rope_matches_64_bits(i, dtype, wdtype, plus_one):
    from paper_2608_20961_b200 import attention as at
    x, _, w, rope = _norm_case(i, dtype, wdtype)
    ref = pu.norm_reference(x, w, 1e-6, rope, plus_one)
    plain = pu.norm_reference(x, w, 1e-6, None, plus_one)
    tol = 2.0 ** -19 * pu.pair_size(plain, rope) + pu.HALF_STEP[dtype] * 1.01 * ref.abs()
    norm, xs = at.HeadNorm(w.to(DEV), 1e-6, plus_one), _strided(x, 32)
    y = torch.empty(x.shape, dtype=dtype, device=DEV)
    at.treewy_norm_rope(norm, _handle(rope), xs, y)
    assert ((y.cpu().to(F64) - ref).abs() <= tol).all()
    at.treewy_norm_rope(norm, _handle(rope), xs, xs)          # in place
    assert torch.equal(xs, y)


# dx: as above, relative to the sizes of both of its terms.  dw: a lane adds its rows one after the other (at most 64 of them
# here), then 5 exchanges, 3 warps, 37 parts and 4 levels: below 2^-17 of the sum of absolute terms.
@pytest.mark.parametrize("i", range(len(NORMS)))
@pytest.mark.parametrize("dtype,wdtype,plus_one", [(BF16, BF16, False), (BF16, F32, True), (F32, F32, False), (F32, BF16, True)])
def test_norm_rope_backward_matches_64_bits(i, dtype, wdtype, plus_one):
    from paper_2608_20961_b200 import attention as at
    x, dy, w, rope = _norm_case(i, dtype, wdtype)
    eps, d = 1e-5, x.shape[-1]
    dx_ref, dw_ref = pu.norm_backward_reference(x, w, eps, dy, rope, plus_one)
    X, W = x.to(F64), (w.to(F64) + (1 if plus_one else 0)).abs()
    r = (X.square().mean(-1, keepdim=True) + eps) ** -0.5
    g = pu.pair_size(dy.to(F64), rope)
    size = r * W * g + X.abs() * r ** 3 * (W * g * X.abs()).mean(-1, keepdim=True)
    norm, xs, dys = at.HeadNorm(w.to(DEV), eps, plus_one), _strided(x, 16), _strided(dy, 64)
    dx, dw = torch.full(x.shape, 7.0, dtype=dtype, device=DEV), torch.full((d,), 7.0, device=DEV)
    ws = at.norm_rope_workspace(xs)
    ws.fill_(0xff)
    at.treewy_norm_rope_backward(norm, _handle(rope), xs, dys, dx, dw, ws)
    assert ((dx.cpu().to(F64) - dx_ref).abs() <= 2.0 ** -18 * size + pu.HALF_STEP[dtype] * 1.01 * dx_ref.abs()).all()
    assert ((dw.cpu().to(F64) - dw_ref).abs() <= 2.0 ** -17 * (g * X.abs() * r).sum((0, 1))).all()
    for _ in range(2):                                       # the order of its sums is fixed; dx may be dy
        dw2, at_dy = torch.empty_like(dw), dys.clone()
        at.treewy_norm_rope_backward(norm, _handle(rope), xs, at_dy, at_dy, dw2, ws)
        assert torch.equal(dw2, dw) and torch.equal(at_dy, dx)


def test_norm_backward_of_no_rows_and_of_a_bad_position():
    from paper_2608_20961_b200 import attention as at
    norm = at.HeadNorm(torch.ones(64, device=DEV))
    z = lambda T: torch.ones((T, 2, 64), device=DEV)
    ws, dw = at.norm_rope_workspace(z(1)), torch.full((64,), 7.0, device=DEV)
    at.treewy_norm_rope_backward(norm, None, z(0), z(0), z(0), dw, ws)
    assert (dw == 0).all()
    rope = at.Rope(au.rope_table(64, 8).to(DEV), torch.tensor([1, 8, 2], dtype=torch.int32, device=DEV))
    status, dx = torch.zeros(1, dtype=torch.int32, device=DEV), torch.full((3, 2, 64), 7.0, device=DEV)
    at.treewy_norm_rope_backward(norm, rope, z(3), z(3), dx, dw, ws, status)
    assert int(status) == 256 and (dx[1] == 7).all() and not (dx[0] == 7).any()
    two = at.Rope(au.rope_table(64, 8).to(DEV), torch.tensor([1, 2], dtype=torch.int32, device=DEV))
    dw2 = torch.empty_like(dw)
    at.treewy_norm_rope_backward(norm, two, z(2), z(2), torch.empty_like(z(2)), dw2, ws)
    assert torch.allclose(dw, dw2, rtol=0, atol=1e-5)


def test_norm_rope_flags_the_rows_sequence():
    from paper_2608_20961_b200 import attention as at
    norm = at.HeadNorm(torch.ones(64, device=DEV))
    rope = at.Rope(au.rope_table(64, 8).to(DEV), torch.tensor([1, 3, -1, 2, 9], dtype=torch.int32, device=DEV))
    x, y = torch.ones((5, 2, 64), device=DEV), torch.full((5, 2, 64), 7.0, device=DEV)
    status = torch.zeros(3, dtype=torch.int32, device=DEV)
    at.treewy_norm_rope(norm, rope, x, y, torch.tensor([0, 2, 4, 5], dtype=torch.int32, device=DEV), status)
    assert status.tolist() == [0, 256, 256] and [(y[t] == 7).all().item() for t in range(5)] == [False, False, True, False, True]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,rot,page", [(128, 128, 16), (256, 64, 32), (72, 72, 5), (64, 0, 8)])
def test_append_norm_is_norm_then_append(dtype, d, rot, page):
    """One pass against the norm's own call and the plain append: the same arithmetic, so the same bits."""
    from paper_2608_20961_b200 import attention as at
    gen = torch.Generator().manual_seed(d)
    N, L, Hq, Hkv = [1, 0, 40, 3], [5, 9, 0, 77], 8, 2
    T, B = sum(N), len(N)
    qkv = torch.randn(T, (Hq + 2 * Hkv) * d, generator=gen).to(dtype).to(DEV)
    q, k, v = (x.view(T, -1, d) for x in qkv.split([Hq * d, Hkv * d, Hkv * d], 1))
    wq, wk = (at.HeadNorm((1 + 0.2 * torch.randn(d, generator=gen)).to(dtype).to(DEV), 1e-6, one) for one in (False, True))
    rope = _handle(_rope(T, rot, 1, False, gen)) if rot else None
    n = max(-(-(a + b) // page) for a, b in zip(L, N))
    table = torch.randperm(B * n, generator=gen).int().view(B, n).to(DEV)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(N)]), dtype=torch.int32, device=DEV)
    lens = torch.tensor(L, dtype=torch.int32, device=DEV)

    def caches():
        return at.KVCache(*(torch.full((B * n, page, Hkv, d), 3.0, dtype=dtype, device=DEV) for _ in range(2)), table, lens)

    one, two = caches(), caches()
    q1, q2, k2 = (torch.empty((T, h, d), dtype=dtype, device=DEV) for h in (Hq, Hq, Hkv))
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    at.treewy_kv_append_norm(one, offsets, k, v, wk, rope, q, q1, wq, status)
    at.treewy_norm_rope(wq, rope, q, q2)
    at.treewy_norm_rope(wk, rope, k, k2)
    at.treewy_kv_append(two, offsets, k2, v)
    assert not status.any()
    assert torch.equal(q1, q2) and torch.equal(one.k, two.k) and torch.equal(one.v, two.v)
    # without norms: the plain append
    at.treewy_kv_append_norm(one, offsets, k, v, None, rope, q, q1)
    at.treewy_kv_append(two, offsets, k, v, rope, q, q2)
    assert torch.equal(q1, q2) and torch.equal(one.k, two.k) and torch.equal(one.v, two.v)


# ------------------------------------------------------------------------------------------ pages

def _pool(p: pu.Pages):
    from paper_2608_20961_b200 import attention as at
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    return at.PagePool(i(p.table).view(len(p.table), -1), p.page, p.n_pages, i(p.free), i([p.count]))


def _same_pages(pool, p):
    assert pool.page_table.tolist() == p.table and int(pool.free_count) == p.count and pool.free_pages.tolist() == p.free


def _reserve(pool, p, L, off, T, expect=None):
    from paper_2608_20961_b200 import attention as at
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    status = torch.zeros(len(L), dtype=torch.int32, device=DEV)
    position = torch.full((T + 1,), -5, dtype=torch.int32, device=DEV)
    slots = torch.full((T + 1,), -5, dtype=torch.int64, device=DEV)
    at.treewy_pages_reserve(pool, i(L), i(off), T, position, slots, status)
    want, pos, slot = p.reserve(L, off, T)
    left = lambda x: [-5 if y is None else y for y in x] + [-5]
    assert status.tolist() == want and (expect is None or want == expect)
    assert position.tolist() == left(pos) and slots.tolist() == left(slot)
    _same_pages(pool, p)


def _release(pool, p, first, end, expect=None):
    from paper_2608_20961_b200 import attention as at
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    status = torch.zeros(len(first), dtype=torch.int32, device=DEV)
    at.treewy_pages_release(pool, i(first), i(end), status)
    want = p.release(first, end)
    assert status.tolist() == want and (expect is None or want == expect)
    _same_pages(pool, p)


@pytest.mark.parametrize("B,most,page,pages", [(1, 1, 16, 4), (5, 40, 8, 60), (64, 9, 16, 300), (3, 5000, 24, 700), (2100, 6, 4, 6000), (40, 700, 1, 40000)])
def test_pages_over_many_steps(B, most, page, pages):
    """Sequences grow, some of what they reserved is not kept, windows leave pages behind, sequences end; the pool may run out."""
    rng = np.random.default_rng(B)
    max_pages = min(pages, -(-12 * most // page) + 2, (1 << 20) // B)
    p = pu.Pages([[-1] * max_pages for _ in range(B)], rng.permutation(pages).tolist(), pages, page, pages)
    pool, L = _pool(p), [0] * B
    for step in range(6):
        N = [int(n) if l + n <= max_pages * page else 0 for n, l in zip(rng.integers(0, most + 1, B), L)]
        off = np.concatenate([[0], np.cumsum(N)]).tolist()
        _reserve(pool, p, L, off, off[-1])
        keep = [int(rng.integers(0, n + 1)) for n in N]
        # (sequences that have got no pages keep their length)
        L = [l + k if all(p.table[b][x] >= 0 for x in range(l // page, -(-(l + k) // page))) else l for b, (l, k) in enumerate(zip(L, keep))]
        _release(pool, p, L, [1 << 30] * B)                   # the drafts that were not kept
        if step == 3:
            ends = [int(l) if rng.random() < 0.3 else 0 for l in L]
            _release(pool, p, [0] * B, ends)
            L = [0 if e and e % page == 0 else l for e, l in zip(ends, L)]


def test_pages_run_out_in_order_and_bad_entries_are_flagged():
    p = pu.Pages([[-1] * 4, [-1] * 4, [-1] * 4, [-1] * 4], list(range(6)), 5, 8, 6)
    pool = _pool(p)
    _reserve(pool, p, [0, 0, 0, 0], [0, 16, 16, 40, 41], 41, [0, 0, 0, 512])     # 2 + 0 + 3 of 5
    _release(pool, p, [0, 0, 9, 0], [8, 0, 24, 0], [0, 0, 0, 0])                 # one page each
    # a partly used page that is gone; a full pool of wishes that does not fit; a range that leaves the rows
    _reserve(pool, p, [3, 0, 16, 0], [0, 2, 30, 31, 99], 31, [64, 512, 512, 32])
    p.table[1][0], p.free[p.count - 1] = 9, 77                                   # out of range: held, and on the stack
    pool = _pool(p)
    _reserve(pool, p, [8, 0, 0, 33], [0, 0, 9, 9, 10], 10, [0, 64, 0, 128])
    _release(pool, p, [-3, 0, 0, 0], [0, 16, 8, -1], [0, 64, 0, 0])


def test_a_page_that_is_released_twice_is_flagged():
    p = pu.Pages([[0, 1, 0], [2, 3, 1]], [0, 0, 0, 0], 0, 4, 4)
    pool = _pool(p)
    _release(pool, p, [0, 0], [12, 12])
    assert p.count == 4


@pytest.mark.parametrize("count", [-1, 7])
def test_a_stack_that_is_no_stack_hands_out_nothing(count):
    from paper_2608_20961_b200 import attention as at
    pool = at.PagePool.empty(2, 3, 8, 6, DEV)
    pool.free_count.fill_(count)
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    at.treewy_pages_reserve(pool, i(0, 0), i(0, 3, 5), 5, seq_status=status)
    assert status.tolist() == [512, 512] and (pool.page_table == -1).all() and int(pool.free_count) == count
