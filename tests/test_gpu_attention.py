"""The attention-layer calls on the GPU against the operators in 64 bits (tests/attn_util.py states the error
bounds and where they come from)."""
import math

import numpy as np
import pytest
import torch

from tests import attn_util as au

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"


# ------------------------------------------------------------------------------------------ attention

CASES = {
    # one token, one cached token, none at all
    "one node, no context": dict(L=[0], N=[1]),
    "one node, one token": dict(L=[1], N=[1]),
    "lengths around a tile": dict(L=[63, 64, 65, 127, 128, 129], N=[1, 2, 3, 1, 2, 3]),
    "decode, eight heads a group": dict(L=[300, 1, 777], N=[1, 1, 1], Hq=16, Hkv=2),
    "decode, five heads a group": dict(L=[200, 33], N=[1, 1], Hq=5, Hkv=1),
    "no grouping": dict(L=[40, 90], N=[4, 9], Hq=3, Hkv=3),
    "a tree of 64": dict(L=[100, 10], N=[64, 37], Hq=8, Hkv=2),
    "many rows a head": dict(L=[130], N=[64], Hq=16, Hkv=2),
    "a chain of 64": dict(L=[70], N=[64], chain=True),
    "forests": dict(L=[5, 80], N=[20, 33], forest=True),
    "head 128, page 8": dict(L=[150, 9, 0], N=[5, 1, 17], D=128, page=8),
    "head 128, page 64": dict(L=[150, 256], N=[5, 6], D=128, page=64),
    "head 256, page 32": dict(L=[321, 17], N=[32, 7], D=256, page=32, Hq=8, Hkv=1),
    "head 256, page 128": dict(L=[500, 129], N=[3, 64], D=256, page=128, Hq=4, Hkv=2),
    "page 256": dict(L=[700, 255, 256], N=[2, 3, 4], page=256),
    "odd page, odd head": dict(L=[50, 11], N=[3, 4], page=5, D=72),
    "long context": dict(L=[5000], N=[3], Hq=4, Hkv=1, D=128),
    "short contexts in a large batch": dict(L=[(7 * b) % 50 for b in range(150)], N=[1 + b % 3 for b in range(150)], Hq=4, Hkv=2),
    "shared prompt": dict(L=[200, 128, 140], N=[4, 1, 9], shared=128),
    "shared prompt, many rows": dict(L=[300] * 9, N=[16] * 9, shared=256, Hq=16, Hkv=2, D=128),
    "shared prompt, head 256": dict(L=[64, 100, 65], N=[30, 2, 5], shared=64, D=256, Hq=10, Hkv=2),
    "nothing but a shared prompt": dict(L=[96, 96], N=[1, 1], shared=96, page=32),
    "steep softmax": dict(L=[400, 64], N=[8, 5], q_scale=30.0),
}


def _case(name, dtype, seed=0):
    return au.make_case(dtype=dtype, seed=seed, **CASES[name])


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)], ids=["bf16", "bf16-generic", "f32"])
def test_attention_matches_64_bits(name, dtype, generic):
    c = _case(name, dtype)
    ref, size = au.attn_reference(c)
    O, status = au.run_attn(c, generic=generic)
    assert not any(status)
    if "steep" in name:  # scores 30 times as large: their rounding, and so the weights', grows with them
        size = size * 30
    au.assert_attn(c, O, ref, size, tensor_cores=dtype == BF16 and not generic)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_hint_layout_and_forms_agree(dtype):
    """A tight max_nodes, heads-first pages and a shared prompt handed over as plain pages change nothing but
    the order of sums."""
    c = au.make_case([150, 128, 333], [7, 1, 12], Hq=8, Hkv=2, D=128, dtype=dtype, shared=128, seed=3)
    ref, size = au.attn_reference(c)
    tc = dtype == BF16
    for kw in (dict(max_nodes=12), dict(layout="heads"), dict(max_nodes=64, layout="heads")):
        O, status = au.run_attn(c, **kw)
        assert not any(status)
        au.assert_attn(c, O, ref, size, tc)
    c.table[:, :128 // c.page] = c.shared_pages
    c.shared, c.shared_pages = 0, None
    O, status = au.run_attn(c)
    assert not any(status)
    au.assert_attn(c, O, ref, size, tc)


@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)])
def test_what_a_node_may_not_see_never_spreads(dtype, generic):
    """NaN and infinities in rows of other branches, of other sequences and in unused slots."""
    c = au.make_case([70, 0, 64], [20, 9, 3], Hq=4, Hkv=2, D=128, dtype=dtype, seed=5)
    bad = [5, 19, 20 + 4, 31]                       # packed rows that are poisoned
    for t, x in zip(bad, (math.nan, math.inf, -math.inf, math.nan)):
        c.k[t], c.v[t] = x, x
    c.v[bad[0], :, ::2] = math.inf
    ref, size = au.attn_reference(c)
    O, status = au.run_attn(c, generic=generic)
    assert not any(status)
    masks = c.mask.numpy().view(np.uint64)
    clean = torch.ones(c.T, dtype=torch.bool)
    for b in range(c.B):
        lo = int(c.offsets[b])
        for t in range(lo, lo + c.N[b]):
            clean[t] = not any(lo <= x < lo + c.N[b] and (int(masks[t]) >> (x - lo)) & 1 for x in bad)
    assert clean.any() and not clean.all()
    au.assert_attn(c, O, ref, size, dtype == BF16 and not generic, rows=clean)
    assert not torch.isfinite(O[~clean]).all(-1).any(), "a node that sees NaN keys or values has to say so"


@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)])
def test_infinite_values_that_are_seen_come_through(dtype, generic):
    """Infinity in a value row alone: exactly its columns, in exactly the rows that see it."""
    c = au.make_case([70, 5], [6, 5], Hq=4, Hkv=2, D=64, dtype=dtype, seed=6, chain=True)
    c.v[2, 1, 7], c.v[3, 1, 7], c.v[4, 0, 9] = math.inf, math.inf, -math.inf
    O, _ = au.run_attn(c, generic=generic)
    want = torch.zeros(c.T, c.Hq, c.D)
    want[2:6, 2:, 7] = math.inf                     # heads 2, 3 read key/value head 1
    want[4:6, :2, 9] = -math.inf
    inf = ~torch.isfinite(want)
    assert torch.equal(O[inf].float(), want[inf]) and torch.isfinite(O[~inf]).all()


@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)])
def test_nodes_that_see_nothing_get_zero(dtype, generic):
    c = au.make_case([0, 40, 0], [5, 4, 2], dtype=dtype, seed=7)
    c.mask[1], c.mask[6], c.mask[9] = 0, 0, -1 << 40   # no bit, no bit but a context, bits past the tree alone
    ref, size = au.attn_reference(c)
    O, status = au.run_attn(c, generic=generic)
    assert not any(status) and not O[1].any() and not O[9].any() and O[6].any()
    au.assert_attn(c, O, ref, size, dtype == BF16 and not generic)


@pytest.mark.parametrize("dtype,generic", [(BF16, False), (BF16, True), (F32, False)])
@pytest.mark.parametrize("shared", [0, 32])
def test_malformed_sequences_are_flagged_and_skipped(dtype, generic, shared):
    from paper_2608_20961_b200 import attention as at, binding as tw
    c = au.make_case([100, 90, 300, 70, 80, 64], [3, 4, 5, 2, 6, 3], dtype=dtype, seed=8, shared=shared)
    ref, size = au.attn_reference(c)
    c.table[2, 300 // c.page] = int(c.kc.shape[0])     # one past the pool, in the last page that is read
    c.table[1, 90 // c.page + 1:] = -1                 # never read
    good_len = list(c.L)
    c.L[3] = -1 if not shared else shared - 1          # negative, or shorter than the shared prompt
    c.L[4] = c.table.shape[1] * c.page + 1             # longer than its table
    O, status = au.run_attn(c, generic=generic, max_nodes=5)
    assert status == [0, 0, at.SEQ_BAD_PAGE, at.SEQ_BAD_LENGTH, tw.SEQ_TOO_MANY_NODES, 0]
    good = torch.zeros(c.T, dtype=torch.bool)
    for b in (0, 1, 5):
        good[int(c.offsets[b]):int(c.offsets[b + 1])] = True
    assert (O[~good] == 7.25).all()
    au.assert_attn(c, O, ref, size, dtype == BF16 and not generic, rows=good)
    c.L[4] = good_len[4]
    c.L[5] = c.table.shape[1] * c.page + 1
    c.offsets[1] = 200                                 # sequences 0 and 1 leave the packed rows
    O, status = au.run_attn(c, generic=generic)
    assert status[0] == status[1] == tw.SEQ_BAD_OFFSETS and status[5] == at.SEQ_BAD_LENGTH and status[4] == 0


def test_a_bad_shared_page_skips_every_sequence():
    from paper_2608_20961_b200 import attention as at
    for generic in (False, True):
        c = au.make_case([100, 90], [3, 4], dtype=BF16, seed=9, shared=64)
        c.shared_pages[2] = -1
        O, status = au.run_attn(c, generic=generic)
        assert status == [at.SEQ_BAD_PAGE] * 2 and (O == 7.25).all()


def test_calls_repeat_bit_for_bit_and_on_another_stream():
    from paper_2608_20961_b200 import attention as at
    c = au.make_case([3000, 17, 900], [12, 1, 30], Hq=16, Hkv=2, D=128, seed=10)
    g = au.on_gpu(c)
    ws = at.attn_workspace(g["cache"], g["tree"], c.Hq)
    call = lambda O, stream=None: at.treewy_attn_verify(g["cache"], g["tree"], g["q"], g["k"], g["v"], c.scale, O, ws, stream=stream)
    outs = [torch.empty((c.T, c.Hq, c.D), dtype=c.dtype, device=DEV) for _ in range(3)]
    call(outs[0])
    call(outs[1])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    call(outs[2], s)
    s.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    graph = torch.cuda.CUDAGraph()
    O = torch.empty_like(outs[0])
    with torch.cuda.graph(graph):
        call(O)
    O.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, outs[0])


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(seed):
    rng = np.random.default_rng(100 + seed)
    B = int(rng.integers(1, 12))
    Hkv = int(rng.choice([1, 2, 4]))
    page = int(rng.choice([8, 16, 32, 64]))
    shared = int(rng.choice([0, 1, 3])) * page
    most = int(rng.choice([3, 9, 64]))
    c = au.make_case([shared + int(x) for x in rng.integers(0, rng.choice([5, 70, 600]), B)],
                     [int(x) for x in rng.integers(1, most + 1, B)], Hq=Hkv * int(rng.choice([1, 3, 4, 8])), Hkv=Hkv,
                     D=int(rng.choice([64, 128, 256])), page=page, seed=seed, shared=shared, forest=bool(seed & 1))
    ref, size = au.attn_reference(c)
    O, status = au.run_attn(c, max_nodes=max(c.N) if seed % 3 else 0)
    assert not any(status)
    au.assert_attn(c, O, ref, size, tensor_cores=True)


@pytest.mark.parametrize("D,page,nodes,Hkv,shared", [(64, 16, 1, 8, 0), (128, 8, 3, 4, 0), (128, 32, 64, 2, 640), (256, 16, 16, 2, 0),
                                                     (256, 64, 5, 4, 0), (256, 8, 24, 1, 512), (256, 128, 64, 1, 0)])
def test_long_runs_of_tiles(D, page, nodes, Hkv, shared):
    """Batches that keep every CTA at work for dozens of tiles and several items, against the SIMT kernel (which the
    tests above tie to 64 bits): both are within their bounds of the same value."""
    from paper_2608_20961_b200 import attention as at, binding as tw
    B, G = 12, 4
    rng = np.random.default_rng(D + page)
    gen = torch.Generator(device=DEV).manual_seed(D + page)
    L = [int(x) for x in rng.integers(shared, 9000, B)]
    N = [int(x) for x in rng.integers((nodes + 1) // 2, nodes + 1, B)]
    T = sum(N)
    need = [-(-n // page) for n in L]
    n_pages = sum(need) + 1
    table = torch.zeros((B, max(need)), dtype=torch.int32)
    order, k0 = torch.from_numpy(rng.permutation(n_pages).astype(np.int32)), 0
    for b, n in enumerate(need):
        table[b, :n] = order[k0:k0 + n]
        k0 += n
    table[:, :shared // page] = table[0, :shared // page].clone()
    rand = lambda *s: torch.randn(s, generator=gen, device=DEV, dtype=BF16)
    cache = at.KVCache(rand(n_pages, page, Hkv, D), rand(n_pages, page, Hkv, D), table.to(DEV), torch.tensor(L, dtype=torch.int32, device=DEV))
    trees = [au.random_tree(n, rng) for n in N]
    off = torch.tensor(np.concatenate([[0], np.cumsum(N)]), dtype=torch.int32, device=DEV)
    tree = tw.Tree.empty(off, torch.tensor(sum((t[0] for t in trees), []), dtype=torch.int32, device=DEV), 1, nodes)
    tree.anc_mask = torch.from_numpy(np.array(sum((t[1] for t in trees), []), np.uint64).view(np.int64)).to(DEV)
    q, k, v = rand(T, Hkv * G, D), rand(T, Hkv, D), rand(T, Hkv, D)
    ws = at.attn_workspace(cache, tree, Hkv * G, shared)
    pages = table[0, :shared // page].contiguous().to(DEV) if shared else None
    outs = []
    for generic in (False, False, True):
        O = torch.zeros((T, Hkv * G, D), dtype=BF16, device=DEV)
        status = torch.zeros(B, dtype=torch.int32, device=DEV)
        at.treewy_attn_verify(cache, tree, q, k, v, D ** -0.5, O, ws, pages, shared, status, generic=generic)
        assert not status.any()
        outs.append(O.double())
    assert torch.equal(outs[0], outs[1])
    # the weights' rounding is independent from key to key, so it adds up as a square root: per row, 2^-8 of the output's
    # own size twice over (weights, store) and once for the SIMT kernel's store
    err = (outs[0] - outs[2]).norm(dim=-1) / outs[2].norm(dim=-1)
    assert float(err.max()) <= 3 * au.BF16_HALF_ULP, float(err.max())


def test_cache_offsets_past_32_bits():
    """A pool of more than 2^32 elements (and bytes), the sequences' pages at its far end."""
    from paper_2608_20961_b200 import attention as at
    page, Hkv, D = 64, 8, 128
    n_pages = (1 << 32) // (page * Hkv * D) + 40      # 8 GB each for k and v
    c = au.make_case([500, 77], [6, 2], Hq=16, Hkv=Hkv, D=D, page=page, seed=11)
    ref, size = au.attn_reference(c)
    have = c.kc.shape[0]
    c2 = dict(k=torch.empty((n_pages, page, Hkv, D), dtype=BF16, device=DEV), v=torch.empty((n_pages, page, Hkv, D), dtype=BF16, device=DEV))
    c2["k"][-have:], c2["v"][-have:] = c.kc.to(DEV), c.vc.to(DEV)
    g = au.on_gpu(c)
    table = torch.where(c.table >= 0, c.table + (n_pages - have), c.table).to(DEV)
    cache = at.KVCache(c2["k"], c2["v"], table, g["cache"].context_len)
    for generic in (False, True):
        O = torch.zeros((c.T, c.Hq, D), dtype=BF16, device=DEV)
        at.treewy_attn_verify(cache, g["tree"], g["q"], g["k"], g["v"], c.scale, O, at.attn_workspace(cache, g["tree"], c.Hq),
                              generic=generic)
        au.assert_attn(c, O.cpu(), ref, size, tensor_cores=not generic)
    # append and commit write there
    k, v = g["k"], g["v"]
    table2 = torch.full((2, 10), n_pages - 1, dtype=torch.int32, device=DEV)
    table2[0, 8], table2[1, 1] = n_pages - 1, n_pages - 2
    cache = at.KVCache(c2["k"], c2["v"], table2, torch.tensor([8 * page + 3, page], dtype=torch.int32, device=DEV))
    at.treewy_kv_append(cache, g["tree"].node_offsets, k, v)
    assert torch.equal(c2["k"][-1, 3:9], k[:6]) and torch.equal(c2["v"][-2, 0:2], v[6:8])
    c2["k"][-2:].zero_()
    at.treewy_kv_commit(cache, g["tree"], k, v, torch.tensor([0, 1], dtype=torch.int32, device=DEV))
    assert torch.equal(c2["k"][-1, 3], k[0]) and not c2["k"][-1, 4:].any()


# --------------------------------------------------------------------------------------- rope, append

def _bound_rope(ref, x, dtype):
    """Two products and a sum in fp32 (each rounded to 2^-24 of at most |x| + |y|), then one store."""
    size = x.to(torch.float64).abs().amax(-1, keepdim=True) * 2
    tol = 3 * 2.0 ** -24 * size
    return tol + (au.BF16_HALF_ULP * (ref.abs() + tol) if dtype == BF16 else 2.0 ** -24 * ref.abs())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,rot,axes", [(1, 1, 64, 64, 1), (7, 3, 128, 128, 3), (33, 5, 80, 48, 2), (5, 2, 256, 64, 3),
                                            (9, 4, 24, 20, 2), (3, 70, 8, 2, 1), (260, 2, 128, 32, 4), (2, 3, 512, 512, 3)])
def test_rope_and_its_inverse(dtype, interleaved, T, H, D, rot, axes):
    from paper_2608_20961_b200 import attention as at
    gen = torch.Generator().manual_seed(T)
    pad = 8
    x = torch.randn((T, H * D + pad), generator=gen).to(dtype)
    pos = torch.randint(0, 4000, (axes, T), generator=gen, dtype=torch.int32)
    pair_axis = torch.randint(0, axes, (rot // 2,), generator=gen, dtype=torch.uint8)
    table = au.rope_table(rot, 4000)
    rope = at.Rope(table.to(DEV), pos.to(DEV), pair_axis.to(DEV), interleaved)
    for inverse in (False, True):
        xg = x.to(DEV)
        y = torch.full((T, H, D), 7.25, dtype=dtype, device=DEV)
        at.treewy_rope(rope, xg[:, :H * D].unflatten(1, (H, D)), y, inverse)
        xin = x[:, :H * D].unflatten(1, (H, D))
        ref = au.rope_reference(xin, table, pos, pair_axis, interleaved, inverse)
        err = (y.cpu().double() - ref).abs()
        assert (err <= _bound_rope(ref, xin, dtype)).all(), float(err.max())
        assert torch.equal(y.cpu()[..., rot:], xin[..., rot:])
        in_place = xg[:, :H * D].unflatten(1, (H, D))
        at.treewy_rope(rope, in_place, in_place, inverse)
        assert torch.equal(in_place, y) and torch.equal(xg[:, H * D:].cpu(), x[:, H * D:])


def test_rope_backward_is_the_gradient():
    """The inverse of the output's gradient, against the formula's derivative by central differences."""
    from paper_2608_20961_b200 import attention as at
    T, H, D, rot = 4, 2, 32, 24
    gen = torch.Generator().manual_seed(1)
    pos = torch.randint(0, 100, (2, T), generator=gen, dtype=torch.int32)
    pair_axis = torch.tensor([0, 1] * 6, dtype=torch.uint8)
    table = au.rope_table(rot, 100)
    rope = at.Rope(table.to(DEV), pos.to(DEV), pair_axis.to(DEV))
    x, dy = (torch.randn((T, H, D), generator=gen) for _ in range(2))
    dx = torch.empty((T, H, D), device=DEV)
    at.treewy_rope(rope, dy.to(DEV), dx, inverse=True)
    f = lambda z: float((au.rope_reference(z, table, pos, pair_axis) * dy).sum())
    for idx in [(0, 0, 0), (1, 1, 5), (2, 0, 12), (3, 1, 23), (3, 0, 31)]:
        e = torch.zeros(T, H, D, dtype=torch.float64)
        e[idx] = 0.5                                   # (linear: the step does not matter)
        diff = f(x.double() + e) - f(x.double() - e)
        assert abs(diff - float(dx.cpu()[idx])) <= 1e-5 * (1 + abs(diff))


def test_rope_skips_and_flags_positions_out_of_range():
    from paper_2608_20961_b200 import attention as at
    pos = torch.tensor([[0, 50, 3, -1, 9], [1, 2, 49, 4, 1]], dtype=torch.int32, device=DEV)
    x = torch.randn(5, 2, 64, device=DEV)
    table = au.rope_table(64, 50).to(DEV)
    axes = torch.tensor([0, 1] * 16, dtype=torch.uint8, device=DEV)
    y, st = torch.full_like(x, 7.25), torch.zeros(1, dtype=torch.int32, device=DEV)
    at.treewy_rope(at.Rope(table, pos, axes), x, y, row_status=st)
    assert int(st) == at.SEQ_BAD_POSITION
    assert (y[[1, 3]] == 7.25).all() and (y[[0, 2, 4]] != 7.25).all()
    axes[7] = 2                                        # an axis there is not: no row can be rotated
    y.fill_(7.25)
    at.treewy_rope(at.Rope(table, pos, axes), x, y)
    assert (y == 7.25).all()


def _append_reference(kc, vc, table, L, offsets, k, v, page):
    """Row by row; rows are placed where their sequence's table says."""
    kc, vc = kc.clone(), vc.clone()
    for b in range(len(L)):
        for i, t in enumerate(range(int(offsets[b]), int(offsets[b + 1]))):
            s = L[b] + i
            kc[int(table[b, s // page]), s % page], vc[int(table[b, s // page]), s % page] = k[t], v[t]
    return kc, vc


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,Hq,Hkv,D,page,rot", [([1] * 9, 8, 2, 128, 16, 128), ([0, 5, 0, 40, 1, 0], 4, 4, 64, 8, 16),
                                                   ([130, 3], 16, 2, 256, 32, 64), ([7], 0, 1, 72, 5, 6), ([2, 0, 3], 3, 3, 8, 1, 4)])
def test_append(dtype, new, Hq, Hkv, D, page, rot):
    from paper_2608_20961_b200 import attention as at
    gen = torch.Generator().manual_seed(len(new))
    rng = np.random.default_rng(len(new))
    L = [int(x) for x in rng.integers(0, 50, len(new))]
    c = au.make_case(L, [1] * len(new), Hq=max(Hq, Hkv), Hkv=Hkv, D=D, page=page, dtype=dtype, poison=False,
                     room=-(-max(new) // page) + 1)
    T = sum(new)
    off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
    fused = torch.randn((T, (Hq + 2 * Hkv) * D), generator=gen).to(dtype)
    cut = lambda x: (x[:, :Hq * D].unflatten(1, (Hq, D)) if Hq else None, x[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D)),
                     x[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D)))
    q, k, v = cut(fused)
    qg, kg, vg = cut(fused.to(DEV))
    table = au.rope_table(rot, 99)
    pos = torch.randint(0, 99, (2, T), generator=gen, dtype=torch.int32)
    pair_axis = torch.randint(0, 2, (rot // 2,), generator=gen, dtype=torch.uint8)
    for rope in (None, at.Rope(table.to(DEV), pos.to(DEV), pair_axis.to(DEV))):
        for layout in ("slots", "heads"):
            g = au.on_gpu(c, layout=layout)
            q_out = torch.full((T, Hq, D), 7.25, dtype=dtype, device=DEV) if Hq else None
            status = torch.zeros(len(new), dtype=torch.int32, device=DEV)
            at.treewy_kv_append(g["cache"], off.to(DEV), kg, vg, rope, qg, q_out, status)
            assert not status.any()
            turn = lambda x: au.rope_reference(x, table, pos, pair_axis) if rope else x.double()
            kc, vc = _append_reference(c.kc.double(), c.vc, c.table, L, off, turn(k), v, page)
            assert torch.equal(g["cache"].v.cpu(), vc)
            err = (g["cache"].k.cpu().double() - kc).abs()
            bound = _bound_rope(kc, kc, dtype) if rope else torch.zeros_like(kc)
            assert (err <= bound * 2).all()              # (the bound takes the rotated row's own size: up to sqrt 2 less)
            untouched = (_append_reference(torch.zeros_like(c.vc), torch.zeros_like(c.vc), c.table, L, off, torch.ones_like(k),
                                           torch.ones_like(v), page)[0] == 0)
            assert torch.equal(g["cache"].k.cpu()[untouched], c.kc[untouched])
            if Hq:
                ref = turn(q)
                assert ((q_out.cpu().double() - ref).abs() <= (_bound_rope(ref, q, dtype) if rope else 0)).all()


def test_append_flags_and_skips():
    from paper_2608_20961_b200 import attention as at, binding as tw
    c = au.make_case([10, 20, 30, 5], [4, 4, 4, 4], Hkv=1, Hq=1, poison=False, room=1)
    g = au.on_gpu(c)
    c.table[2, 30 // 16] = 999
    g["cache"].page_table.copy_(c.table)
    g["cache"].context_len.copy_(torch.tensor([10, c.table.shape[1] * 16 - 3, 30, 5], dtype=torch.int32))
    before = g["cache"].k.clone()
    status = torch.zeros(4, dtype=torch.int32, device=DEV)
    pos = torch.zeros(16, dtype=torch.int32, device=DEV)
    pos[13] = 8                                          # row 1 of sequence 3
    q_out = torch.full_like(g["q"], 7.25)
    at.treewy_kv_append(g["cache"], g["tree"].node_offsets, g["k"], g["v"], at.Rope(au.rope_table(64, 8).to(DEV), pos), g["q"], q_out, status)
    # sequence 2: rows 30, 31 meet the bad page, rows 32, 33 do not
    assert status.tolist() == [0, at.SEQ_BAD_LENGTH, at.SEQ_BAD_PAGE, at.SEQ_BAD_POSITION]
    written = (g["cache"].k != before).flatten(2).any(2).nonzero().tolist()
    where = lambda b, s: [int(c.table[b, s // 16]), s % 16]
    assert sorted(written) == sorted([where(0, s) for s in range(10, 14)] + [where(2, 32), where(2, 33)] + [where(3, s) for s in (5, 7, 8)])
    assert (q_out[[4, 5, 6, 7, 8, 9, 13]] == 7.25).all() and (q_out[[0, 1, 2, 3, 10, 11, 12, 14, 15]] != 7.25).any(-1).all()
    off = g["tree"].node_offsets.clone()
    off[4] = 99
    status.zero_()
    at.treewy_kv_append(g["cache"], off, g["k"], g["v"], seq_status=status)
    assert status.tolist() == [0, at.SEQ_BAD_LENGTH, at.SEQ_BAD_PAGE, tw.SEQ_BAD_OFFSETS]


# --------------------------------------------------------------------------------------------- commit

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,Hkv,D,page,chain", [([1], 1, 64, 16, False), ([32, 7, 64, 1], 2, 256, 8, False),
                                                ([64, 64, 5], 8, 128, 16, True), ([9] * 70, 3, 72, 5, False)])
def test_commit(dtype, N, Hkv, D, page, chain):
    from paper_2608_20961_b200 import attention as at
    rng = np.random.default_rng(len(N))
    L = [int(x) for x in rng.integers(0, 60, len(N))]
    c = au.make_case(L, N, Hq=Hkv, Hkv=Hkv, D=D, page=page, dtype=dtype, chain=chain, poison=False, room=-(-64 // page) + 1)
    acc = [int(rng.integers(-1, n)) for n in N]
    acc[0] = N[0] - 1
    kc, vc, want = c.kc.clone(), c.vc.clone(), []
    for b, a in enumerate(acc):
        lo, path = int(c.offsets[b]), []
        while a >= 0:
            path.insert(0, a)
            a = int(c.parent[lo + a])
        for r, i in enumerate(path):
            s = L[b] + r
            kc[int(c.table[b, s // page]), s % page], vc[int(c.table[b, s // page]), s % page] = c.k[lo + i], c.v[lo + i]
        want.append(L[b] + len(path))
    for layout in ("slots", "heads"):
        g = au.on_gpu(c, layout=layout)
        new = torch.full((c.B,), -5, dtype=torch.int32, device=DEV)
        status = torch.zeros(c.B, dtype=torch.int32, device=DEV)
        at.treewy_kv_commit(g["cache"], g["tree"], g["k"], g["v"], torch.tensor(acc, dtype=torch.int32, device=DEV), new, status)
        assert not status.any() and new.tolist() == want
        assert torch.equal(g["cache"].k.cpu(), kc) and torch.equal(g["cache"].v.cpu(), vc)


def test_commit_flags_and_skips():
    from paper_2608_20961_b200 import attention as at, binding as tw
    c = au.make_case([10, 20, 30, 5, 6, 7], [4] * 6, Hkv=1, Hq=1, poison=False, room=1, chain=True)
    c.table[2, 1] = -1                                    # token 30 is on it, tokens 32, 33 are not
    g = au.on_gpu(c)
    g["cache"].context_len[1] = c.table.shape[1] * 16 - 3  # three of four rows would fit
    g["cache"].context_len[5] = -1
    before = g["cache"].k.clone()
    acc = torch.tensor([3, 3, 3, 4, -2, 0], dtype=torch.int32, device=DEV)
    new, status = torch.full((6,), -5, dtype=torch.int32, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
    at.treewy_kv_commit(g["cache"], g["tree"], g["k"], g["v"], acc, new, status)
    assert status.tolist() == [0, at.SEQ_BAD_LENGTH, at.SEQ_BAD_PAGE, tw.SEQ_BAD_ACCEPTED, tw.SEQ_BAD_ACCEPTED, at.SEQ_BAD_LENGTH]
    assert new.tolist() == [14, -5, -5, -5, -5, -5]
    written = (g["cache"].k != before).flatten(2).any(2).nonzero().tolist()
    assert sorted(written) == [[int(c.table[0, 0]), s] for s in range(10, 14)]


# ------------------------------------------------------------------------- the round of a hybrid's layer

def test_rounds_of_a_layer_equal_attention_over_the_accepted_tokens():
    """Prompt appended, then rounds of rotate -> verify -> commit: the outputs of every round's accepted node equal
    plain causal attention over the prompt and the accepted tokens."""
    from paper_2608_20961_b200 import attention as at
    Hq, Hkv, D, page, B = 4, 2, 64, 16, 3
    rng = np.random.default_rng(4)
    gen = torch.Generator().manual_seed(4)
    randn = lambda *s: torch.randn(s, generator=gen).to(BF16)
    table = torch.arange(B * 8, dtype=torch.int32).view(B, 8).to(DEV)
    kc = torch.full((B * 8, page, Hkv, D), math.nan, dtype=BF16, device=DEV)
    cache = at.KVCache(kc, kc.clone(), table, torch.zeros(B, dtype=torch.int32, device=DEV))
    wave = au.rope_table(D, 200)
    prompt = [20, 1, 33]
    off = torch.tensor([0, 20, 21, 54], dtype=torch.int32)
    pos = torch.tensor([i for n in prompt for i in range(n)], dtype=torch.int32)
    k, v = randn(54, Hkv, D), randn(54, Hkv, D)
    at.treewy_kv_append(cache, off.to(DEV), k.to(DEV), v.to(DEV), at.Rope(wave.to(DEV), pos.to(DEV)))
    cache.context_len.copy_(torch.tensor(prompt, dtype=torch.int32))
    turned = au.rope_reference(k, wave, pos[None], None).to(BF16)
    seen = [(turned[off[b]:off[b + 1]], v[off[b]:off[b + 1]]) for b in range(B)]
    for rnd in range(3):
        c = au.make_case([0] * B, [9, 5, 16], Hq=Hq, Hkv=Hkv, D=D, seed=50 + rnd)
        lens = cache.context_len.tolist()
        depth = [bin(int(m)).count("1") - 1 for m in c.mask.numpy().view(np.uint64)]
        seq = [b for b in range(B) for _ in range(c.N[b])]
        pos = torch.tensor([lens[b] + d for b, d in zip(seq, depth)], dtype=torch.int32)
        rope = at.Rope(wave.to(DEV), pos.to(DEV))
        g = au.on_gpu(c)
        for x in (g["q"], g["k"]):
            at.treewy_rope(rope, x, x)
        O = torch.empty((c.T, Hq, D), dtype=BF16, device=DEV)
        at.treewy_attn_verify(cache, g["tree"], g["q"], g["k"], g["v"], c.scale, O, at.attn_workspace(cache, g["tree"], Hq))
        acc = [int(rng.integers(0, n)) for n in c.N]
        new_len = torch.empty_like(cache.context_len)
        at.treewy_kv_commit(cache, g["tree"], g["k"], g["v"], torch.tensor(acc, dtype=torch.int32, device=DEV), new_len)
        cache.context_len.copy_(new_len)
        q, k = g["q"].cpu(), g["k"].cpu()
        for b in range(B):
            lo = int(c.offsets[b])
            m = int(c.mask[lo + acc[b]].item())
            rows = [lo + j for j in range(c.N[b]) if (m >> j) & 1]
            seen[b] = (torch.cat([seen[b][0], k[rows]]), torch.cat([seen[b][1], c.v[rows]]))
            one = au.make_case([0], [1], Hq=Hq, Hkv=Hkv, D=D)
            n = seen[b][0].shape[0]
            one.kc, one.vc, one.L, one.page = seen[b][0][None, :n - 1], seen[b][1][None, :n - 1], [n - 1], max(n - 1, 1)
            one.table = torch.zeros((1, 1), dtype=torch.int32)
            one.q, one.k, one.v = q[lo + acc[b]][None], seen[b][0][n - 1:], seen[b][1][n - 1:]
            ref, size = au.attn_reference(one)
            au.assert_attn(one, O.cpu()[lo + acc[b]][None], ref, size, tensor_cores=True)
    assert new_len.tolist() == [s[0].shape[0] for s in seen]


def test_hybrid_example_decodes_the_same_tokens_with_and_without_trees():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_decode.py")
    spec = importlib.util.spec_from_file_location("hybrid_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(["--sequences", "3", "--tokens", "20", "--nodes", "9"]) == 0
    assert example.main(["--sequences", "2", "--tokens", "30", "--nodes", "40"]) == 0


@pytest.mark.parametrize("D,skip", [(64, 0), (128, 5), (256, 3)])
def test_a_wait_that_runs_out_raises_timeout_and_leaves_the_stream_usable(D, skip):
    """One item's copies are never issued (nothing is in flight for it) and the waits get about a millisecond: the call has
    to return, say so in the status, and leave the stream fit for the next call."""
    from paper_2608_20961_b200 import binding as tw
    c = au.make_case([500, 700, 90], [3, 9, 1], Hq=8, Hkv=2, D=D, seed=12)
    ref, size = au.attn_reference(c)
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    try:
        tw.treewy_debug_inject(2_000_000, skip)
        t0.record()
        _, status = au.run_attn(c)
        t1.record()
        torch.cuda.synchronize()
    finally:
        tw.treewy_debug_inject(0, -1)
    assert t0.elapsed_time(t1) < 2000.0
    assert any(s & tw.SEQ_TIMEOUT for s in status) and not any(s & ~tw.SEQ_TIMEOUT for s in status)
    O, status = au.run_attn(c)
    assert not any(status)
    au.assert_attn(c, O, ref, size, tensor_cores=True)


@pytest.mark.parametrize("skip", [0, 3])
def test_a_wait_that_runs_out_beside_a_shared_prompt(skip):
    """The same with a shared prompt: items that were never worked on leave nothing to join, which has to be harmless, and
    the next call on the same workspace is right."""
    from paper_2608_20961_b200 import binding as tw
    c = au.make_case([700, 500, 590], [3, 9, 1], Hq=8, Hkv=2, D=128, seed=13, shared=480)
    ref, size = au.attn_reference(c)
    try:
        tw.treewy_debug_inject(2_000_000, skip)
        _, status = au.run_attn(c)
        torch.cuda.synchronize()
    finally:
        tw.treewy_debug_inject(0, -1)
    assert any(s & tw.SEQ_TIMEOUT for s in status)
    O, status = au.run_attn(c)
    assert not any(status)
    au.assert_attn(c, O, ref, size, tensor_cores=True)
