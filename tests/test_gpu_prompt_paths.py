"""The calls that take new rows through an attention layer, as they are used: a layer's steps, long contexts that are cut
up, captured graphs, other streams, waits that run out, and caches past 2^31 elements."""
import math

import numpy as np
import pytest
import torch

from tests import attn_util as au
from tests import prompt_util as pu

pytestmark = pytest.mark.gpu

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
DEV = "cuda:0"


def _int(*x):
    return torch.tensor(x, dtype=I32, device=DEV)


# ------------------------------------------------------------------------------------------ larger cases

BIG = {
    "cut items, two row tiles": dict(L=[6000, 20000], N=[300, 90], Hq=8, Hkv=2),
    "cut items, one row tile": dict(L=[30000], N=[5], Hq=8, Hkv=1),
    "a prompt": dict(L=[0], N=[2500], Hq=4, Hkv=1),
    "window and sinks over long contexts": dict(L=[9000, 100, 4000], N=[700, 1500, 1], Hq=8, Hkv=2, window=1500, sinks=200),
    "prompts among sequences that decode": dict(L=[2000, 5, 900, 4000, 0, 70], N=[1, 600, 1, 1, 1000, 1], Hq=8, Hkv=2),
    "odd groups": dict(L=[1500, 0], N=[333, 800], Hq=21, Hkv=3),
}


@pytest.mark.parametrize("name", list(BIG))
@pytest.mark.parametrize("D,page", [(64, 16), (128, 16), (128, 128), (256, 32), (256, 8)])
def test_larger_cases_match_64_bits(name, D, page):
    c = pu.make_case(D=D, page=page, seed=31, poison=False, **BIG[name])
    ref, size = pu.chunk_reference_gpu(c)
    O, status = pu.run_chunk(c)
    assert not any(status)
    pu.assert_chunk(c, O, ref, size, tensor_cores=True)


def test_scores_that_grow_without_bound():
    """Later keys whose scores are above all before by more than fp32's exponents reach: the weights so far become nothing, and do not
    overflow on the way."""
    for D in (64, 128, 256):
        c = pu.make_case([0], [700], Hq=2, Hkv=1, D=D, seed=32, poison=False)
        x = torch.arange(700) / 40.0                          # scores grow along the sequence, by hundreds (in log2) a tile
        c.kc[c.table[0, torch.arange(700) // c.page].long(), torch.arange(700) % c.page] = (torch.ones(700, 1, D) * x[:, None, None]).to(BF16)
        c.q = (torch.ones_like(c.q) * 4.0)
        c.scale = 1.0
        ref, size = pu.chunk_reference(c)
        for generic in (False, True):
            O, status = pu.run_chunk(c, generic=generic)
            assert not any(status)
            # (a score is a sum of D equal products here and exact in fp32; exp of differences of hundreds is 0 or of few bits)
            pu.assert_chunk(c, O, ref, size, tensor_cores=not generic)


def test_a_cache_past_2_31_elements():
    from paper_2608_20961_b200 import attention as at
    Hkv, D, page = 8, 128, 64
    n_pages = (1 << 31) // (Hkv * D * page) + 40
    k, v = (torch.empty((n_pages, page, Hkv, D), dtype=BF16, device=DEV) for _ in range(2))
    gen = torch.Generator().manual_seed(1)
    L, N = [500, 130], [70, 200]
    need = [-(-(a + b) // page) for a, b in zip(L, N)]
    pages = n_pages - 1 - torch.randperm(sum(need), generator=gen)          # the last ones
    table = torch.full((2, max(need)), -1, dtype=I32)
    table[0, :need[0]], table[1, :need[1]] = pages[:need[0]].int(), pages[need[0]:].int()
    small = pu.make_case(L, N, Hq=16, Hkv=Hkv, D=D, page=page, seed=33, poison=False)
    for b in range(2):
        for e in range(need[b]):
            for big, src in ((k, small.kc), (v, small.vc)):
                big[int(table[b, e])] = src[int(small.table[b, e])].to(DEV)
    ref, size = pu.chunk_reference_gpu(small)
    lens, off, q = _int(*L), small.offsets.to(DEV), small.q.to(DEV)
    cache = at.KVCache(k, v, table.to(DEV), lens)
    # the rows are written once more by the append, rotated by nothing: the same values
    row_k, row_v = (torch.cat([torch.stack([x[int(small.table[b, p // page]), p % page] for p in range(L[b], L[b] + N[b])]) for b in range(2)]).to(DEV)
                    for x in (small.kc, small.vc))
    norm = at.HeadNorm(torch.ones(D, device=DEV), 1e-6)
    at.treewy_kv_append_norm(cache, off, torch.zeros_like(row_k), row_v, norm)
    assert not cache.k[int(table[0, L[0] // page]), L[0] % page].any()
    at.treewy_kv_append(cache, off, row_k, row_v)
    for generic in (False, True):
        O = torch.empty_like(q)
        at.treewy_attn_chunk(cache, off, q, small.scale, O, at.attn_chunk_workspace(cache, small.T, 16), generic=generic)
        pu.assert_chunk(small, O.cpu(), ref, size, tensor_cores=not generic)


# ------------------------------------------------------------------------------------------ many pages

@pytest.mark.parametrize("short", [0, 1, 70001])
def test_pages_of_more_entries_than_are_taken_at_a_time(short):
    """Lines of 2^17 entries and more: one long sequence among short ones, more sequences than threads; and a pool that ends within."""
    from tests.test_gpu_prompt import _pool, _release, _reserve
    rng = np.random.default_rng(short)
    N = [3, 140000, 0, 1, 20000, 5, 5]
    n_pages = sum(N) - short
    p = pu.Pages([[-1] * 140010 for _ in N], rng.permutation(n_pages).tolist(), n_pages, 1, n_pages)
    pool, off = _pool(p), np.concatenate([[0], np.cumsum(N)]).tolist()
    _reserve(pool, p, [0] * len(N), off, off[-1])
    _release(pool, p, [1, 7, 0, 0, 3, 0, 0], [3, 139990, 5, 0, 20000, 5, 1 << 30])
    _reserve(pool, p, [1, 7, 0, 1, 3, 0, 0], off, off[-1])
    many = 3000
    p = pu.Pages([[-1] * 9 for _ in range(many)], rng.permutation(many * 4).tolist(), many * 4, 8, many * 4)
    pool = _pool(p)
    for most in (10, 60):                               # (the second time the pool ends)
        N = rng.integers(0, most, many).tolist()
        off = np.concatenate([[0], np.cumsum(N)]).tolist()
        L = [8 * sum(x >= 0 for x in r) for r in p.table]
        L = [l if l + n <= 72 else 0 for l, n in zip(L, N)]
        _reserve(pool, p, L, off, off[-1])
    _release(pool, p, [8] * many, [40] * many)


# ------------------------------------------------------------------------------------------ a layer's steps

def _layer(dtype, window, sinks, normed, B=3, Hq=8, Hkv=2, D=128, page=16, max_pages=40, seed=0):
    from paper_2608_20961_b200 import attention as at
    gen = torch.Generator().manual_seed(seed)
    n_pages = B * max_pages
    pool = at.PagePool.empty(B, max_pages, page, n_pages, DEV)
    kv = lambda: torch.full((n_pages, page, Hkv, D), math.nan, dtype=dtype, device=DEV)
    cache = at.KVCache(kv(), kv(), pool.page_table, torch.zeros(B, dtype=I32, device=DEV))
    norm = lambda: at.HeadNorm((1 + 0.2 * torch.randn(D, generator=gen)).to(dtype).to(DEV)) if normed else None
    layer = at.AttentionLayer(cache, Hq, au.rope_table(D, max_pages * page).to(DEV), q_norm=norm(), k_norm=norm(), window=window, sinks=sinks)
    return layer, pool


def _qkv(layer, T, gen):
    c = layer.cache
    x = torch.randn(T, (layer.H_q + 2 * c.H_kv) * c.d_head, generator=gen).to(c.dtype).to(DEV)
    return (y.unflatten(1, (-1, c.d_head)) for y in x.split([layer.H_q * c.d_head, c.H_kv * c.d_head, c.H_kv * c.d_head], 1))


def _reference(layer, b, q_pos, q):
    """Attention of queries q (already normalised and rotated, 64 bits) at positions q_pos over what the cache holds of sequence b."""
    c, G = layer.cache, layer.H_q // layer.cache.H_kv
    n = int(max(q_pos)) + 1
    x = torch.arange(n, device=DEV)
    pages = c.page_table[b].long()[x // c.page_size]
    k, v = (s[pages, x % c.page_size].to(F64).repeat_interleave(G, 1) for s in (c.k, c.v))
    p = torch.tensor(q_pos, device=DEV)[:, None]
    seen = x <= p
    if layer.window:
        seen &= (p - x < layer.window) | (x < layer.sinks)
    v = torch.where(seen.any(0)[:, None, None], v, 0.0)           # (pages that went back hold anything)
    s = (torch.einsum("nhd,xhd->nhx", q, k) * layer.scale).masked_fill_(~seen[:, None], -math.inf)
    w = torch.softmax(s, -1)
    return torch.einsum("nhx,xhd->nhd", w, v), torch.einsum("nhx,xhd->nhd", w, v.abs())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
@pytest.mark.parametrize("normed", [False, True])
def test_a_layer_over_prompts_pieces_and_single_tokens(dtype, window, sinks, normed):
    run_layer_steps(dtype, window, sinks, normed)


def run_layer_steps(dtype, window, sinks, normed):
    """Pages are reserved, rows written and attended, lengths advanced: prompts in pieces, then a token each; beside a window the pages that
    it has left go back to the pool."""
    from paper_2608_20961_b200 import attention as at, binding as tw
    layer, pool = _layer(dtype, window, sinks, normed)
    c, gen, B = layer.cache, torch.Generator().manual_seed(5), 3
    lens, status = [0] * B, torch.zeros(B, dtype=I32, device=DEV)
    for N in ([200, 1, 0], [130, 300, 5], [1, 1, 1], [1, 1, 1], [70, 0, 64], [1, 1, 1]):
        T, off = sum(N), _int(*np.concatenate([[0], np.cumsum(N)]).tolist())
        positions, slots = torch.empty(T, dtype=I32, device=DEV), torch.empty(T, dtype=torch.int64, device=DEV)
        at.treewy_pages_reserve(pool, c.context_len, off, T, positions, slots, status)
        q, k, v = _qkv(layer, T, gen)
        if N == [1, 1, 1]:
            tree = tw.Tree.empty(off, torch.full((B,), -1, dtype=I32, device=DEV), 1, 1)
            O = layer.append_and_attend(tree, positions, q, k, v, status)
        else:
            O = layer.prefill(off, positions, q, k, v, status)
        assert not status.any(), status.tolist()
        rope = (layer.cos_sin.cpu(), positions[None].cpu(), None, False)
        turn = lambda x, n: (pu.norm_reference(x.cpu(), n.weight.cpu(), n.eps, rope) if n else au.rope_reference(x.cpu(), *rope[:3])).to(DEV)
        qt, kt = turn(q, layer.q_norm), turn(k, layer.k_norm)
        # what was written, where the slots say
        flat = lambda s: s.flatten(0, 1)[slots]
        assert torch.equal(flat(c.v), v)
        assert ((flat(c.k).to(F64) - kt).abs() <= 2.0 ** -19 * pu.pair_size(kt, rope) * 2 + pu.HALF_STEP[dtype] * 1.01 * kt.abs()).all()
        at_rows = 0
        for b in range(B):
            if N[b]:
                pos = list(range(lens[b], lens[b] + N[b]))
                ref, size = _reference(layer, b, pos, qt[at_rows:at_rows + N[b]])
                # the kernels' bound, and queries that were rounded: a score of |q||k| / sqrt(d), about 11 at the most here, is off by half a
                # step of it in bf16, and its weight by as much of itself
                slack = (0.1 if dtype == BF16 else 2.0 ** -17) * size
                err = (O[at_rows:at_rows + N[b]].to(F64) - ref).abs() - slack
                case = type("C", (), dict(dtype=dtype))
                assert (err <= au.attn_bound(case, ref, size, dtype == BF16)).all()
            at_rows += N[b]
        lens = [a + n for a, n in zip(lens, N)]
        assert c.context_len.tolist() == lens
        if window:
            # what no later token sees: from behind the sinks' page to the window of the next token
            first = _int(*[sinks] * B)
            at.treewy_pages_release(pool, first, _int(*[max(0, n - window + 1) for n in lens]), status)
            assert not status.any()
    held = sum(len([e for e in range(-(-n // 16)) if not window or e * 16 < sinks or (e + 1) * 16 > n - window + 1]) for n in lens)
    assert int(pool.free_count) == pool.n_pages - held


def test_a_layers_steps_are_its_calls():
    """prefill and append_and_attend beside a window against the calls themselves: the same bits."""
    from paper_2608_20961_b200 import attention as at
    layer, pool = _layer(BF16, 60, 3, True, seed=3)
    other, pool2 = _layer(BF16, 60, 3, True, seed=3)
    gen, N = torch.Generator().manual_seed(6), [90, 3, 150]
    off, T = _int(0, 90, 93, 243), 243
    q, k, v = _qkv(layer, T, gen)
    positions = torch.empty(T, dtype=I32, device=DEV)
    for p, l in ((pool, layer), (pool2, other)):
        at.treewy_pages_reserve(p, l.cache.context_len, off, T, positions)
    O = layer.prefill(off, positions, q, k, v)
    c = other.cache
    q_out, P = torch.empty_like(O), torch.empty_like(O)
    at.treewy_kv_append_norm(c, off, k, v, other.k_norm, at.Rope(other.cos_sin, positions), q, q_out, other.q_norm)
    at.treewy_attn_chunk(c, off, q_out, other.scale, P, at.attn_chunk_workspace(c, T, 8, 60, 3), 60, 3)
    assert torch.equal(O, P) and layer.cache.context_len.tolist() == N and torch.equal(layer.cache.v.nan_to_num(), c.v.nan_to_num())


def test_flagged_sequences_keep_their_length():
    from paper_2608_20961_b200 import attention as at, binding as tw
    layer, pool = _layer(BF16, 0, 0, False, max_pages=4)
    gen = torch.Generator().manual_seed(7)
    off, T = _int(0, 10, 80, 85), 85                              # the second does not fit 4 pages of 16
    positions = torch.full((T,), 3, dtype=I32, device=DEV)
    status = torch.zeros(3, dtype=I32, device=DEV)
    at.treewy_pages_reserve(pool, layer.cache.context_len, off, T, positions, seq_status=status)
    assert status.tolist() == [0, 128, 0] and (positions[10:80] == 3).all()
    layer.prefill(off, positions, *_qkv(layer, T, gen), status)
    assert status.tolist() == [0, 128, 0] and layer.cache.context_len.tolist() == [10, 0, 5]
    layer.window = 20                                             # one token each is wanted there
    tree = tw.Tree.empty(_int(0, 2, 2, 3), torch.full((3,), -1, dtype=I32, device=DEV), 1, 2)
    layer.append_and_attend(tree, positions[:3], *_qkv(layer, 3, gen))
    assert layer.cache.context_len.tolist() == [10, 0, 6]


def test_trees_behind_norms_are_the_rows_one_after_another():
    """A chain verified and committed against the same tokens as new rows: keys of the same bits, outputs within both kernels' bounds."""
    from paper_2608_20961_b200 import attention as at, binding as tw
    outs, caches = [], []
    for chain in (True, False):
        layer, pool = _layer(BF16, 0, 0, True, seed=9)
        gen = torch.Generator().manual_seed(10)
        prompt, off, T = _int(0, 40, 41, 141), _int(0, 9, 14, 20), 20
        positions = torch.empty(141, dtype=I32, device=DEV)
        at.treewy_pages_reserve(pool, layer.cache.context_len, prompt, 141, positions)
        layer.prefill(prompt, positions, *_qkv(layer, 141, gen))
        at.treewy_pages_reserve(pool, layer.cache.context_len, off, T, positions)
        q, k, v = _qkv(layer, T, gen)
        if chain:
            parent = _int(*[i - 1 for n in (9, 5, 6) for i in range(n)])
            tree = tw.Tree.empty(off, parent, 1, 9)
            status = torch.zeros(3, dtype=I32, device=DEV)
            tw.treewy_tree_prepare(tree, torch.ones(T, 1, device=DEV), status)
            O = layer.verify(tree, positions[:T], q, k, v, status)
            layer.commit(tree, k, v, _int(8, 4, 5), status)
            assert not status.any()
        else:
            O = layer.prefill(off, positions[:T], q, k, v)
        outs.append(O.to(F64)), caches.append(layer.cache)
    assert caches[0].context_len.tolist() == caches[1].context_len.tolist() == [49, 6, 106]
    for a, b in ((caches[0].k, caches[1].k), (caches[0].v, caches[1].v)):
        assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
    # |v| is at most 5 here; either kernel is off by at most 2^-7 of the weighted sum of |v| (weights and output rounded to bf16)
    assert (outs[0] - outs[1]).abs().max() <= 2 * 2.0 ** -7 * float(caches[0].v.nan_to_num(0.0).abs().max())


def test_the_example_with_prompts_and_norms():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_decode.py")
    spec = importlib.util.spec_from_file_location("hybrid_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model = example.Hybrid(3, torch.device(DEV), head_norms=True)
    prompts = [[1, 8, 15, 22] * 10, [5], [7, 7, 9] * 5]
    plain = example.one_by_one(model, prompts, 12)
    assert model.cache.context_len.tolist() == [len(p) + 12 for p in prompts]
    again, rounds = example.speculative(model, prompts, 12, 9, plain)
    assert [len(a) for a in again] == [12] * 3 and rounds <= 12
    assert int(model.pool.free_count) == model.pool.n_pages - int((model.pool.page_table >= 0).sum())


def test_layer_refusals():
    from paper_2608_20961_b200 import attention as at, binding as tw
    layer, _ = _layer(BF16, 60, 3, True)
    with pytest.raises(ValueError):
        at.AttentionLayer(layer.cache, 8, layer.cos_sin, window=-1)
    with pytest.raises(ValueError):
        at.AttentionLayer(layer.cache, 8, layer.cos_sin, q_norm=at.HeadNorm(torch.ones(64, device=DEV)))
    gen = torch.Generator().manual_seed(8)
    tree = tw.Tree.empty(_int(0, 1, 2, 3), torch.full((3,), -1, dtype=I32, device=DEV), 1, 1)
    pos = torch.zeros(3, dtype=I32, device=DEV)
    with pytest.raises(ValueError):
        layer.verify(tree, pos, *_qkv(layer, 3, gen))
    with pytest.raises(ValueError):
        layer.append_and_attend(tree, pos, *_qkv(layer, 3, gen), shared_pages=pos, shared_len=16)
    with pytest.raises(ValueError):
        layer.prefill(_int(0, 1, 2), pos, *_qkv(layer, 3, gen))


# ------------------------------------------------------------------------------------------ streams, graphs, waits

def _step(dtype=BF16, seed=11):
    """A step over all calls on buffers of its own; returns the function and what it writes."""
    from paper_2608_20961_b200 import attention as at
    layer, pool = _layer(dtype, 50, 2, True, seed=seed)
    c, gen = layer.cache, torch.Generator().manual_seed(seed)
    off, T = _int(0, 150, 151, 300), 300
    q, k, v = (x.contiguous() for x in _qkv(layer, T, gen))
    w = dict(positions=torch.zeros(T, dtype=I32, device=DEV), slots=torch.zeros(T, dtype=torch.int64, device=DEV), q_out=torch.zeros_like(q),
             O=torch.zeros_like(q), y=torch.zeros_like(q), dx=torch.zeros_like(q), dw=torch.zeros(c.d_head, device=DEV),
             status=torch.zeros(3, dtype=I32, device=DEV), table=pool.page_table, free=pool.free_pages, count=pool.free_count, k=c.k, v=c.v)
    lens, none, end = c.context_len, torch.zeros(3, dtype=I32, device=DEV), _int(10000, 10000, 10000)
    rope = at.Rope(layer.cos_sin, w["positions"])
    ws, nws = at.attn_chunk_workspace(c, T, 8, 50, 2), at.norm_rope_workspace(q)

    def run():
        at.treewy_pages_release(pool, none, end, w["status"])
        at.treewy_pages_reserve(pool, lens, off, T, w["positions"], w["slots"], w["status"])
        at.treewy_kv_append_norm(c, off, k, v, layer.k_norm, rope, q, w["q_out"], layer.q_norm, w["status"])
        at.treewy_attn_chunk(c, off, w["q_out"], layer.scale, w["O"], ws, 50, 2, w["status"])
        at.treewy_norm_rope(layer.q_norm, rope, q, w["y"], off, w["status"])
        at.treewy_norm_rope_backward(layer.q_norm, rope, q, w["O"], w["dx"], w["dw"], nws, w["status"])

    return run, w


def _same(a, b):
    for name in a:
        assert torch.equal(a[name].nan_to_num(7.0), b[name].nan_to_num(7.0)), name


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_step_captured_and_on_another_stream_is_the_eager_one(dtype):
    eager, want = _step(dtype)
    eager()
    assert not want["status"].any()
    side = torch.cuda.Stream()
    on_side, got = _step(dtype)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side()
    side.synchronize()
    _same(want, got)
    captured, got = _step(dtype)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured()
        captured()                                                # (releases what it had reserved and takes the same again)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    _same(want, got)


def test_a_captured_prefill_keeps_its_workspace():
    """A longer prompt makes the layer take a larger workspace; a graph that was captured ahead of that still has its own."""
    from paper_2608_20961_b200 import attention as at
    layer, pool = _layer(BF16, 0, 0, True, B=1, max_pages=400, seed=4)
    gen = torch.Generator().manual_seed(4)
    first = _qkv(layer, 5000, gen)
    first = [x.contiguous() for x in first]
    pos, off = torch.empty(5000, dtype=I32, device=DEV), _int(0, 5000)
    at.treewy_pages_reserve(pool, layer.cache.context_len, off, 5000, pos)
    layer.prefill(off, pos, *first)
    layer._rows_ws, layer._rows_for = None, 0
    q, k, v = (x.contiguous() for x in _qkv(layer, 3, gen))
    pos, off = torch.empty(3, dtype=I32, device=DEV), _int(0, 3)
    at.treewy_pages_reserve(pool, layer.cache.context_len, off, 3, pos)
    want = layer.prefill(off, pos, q, k, v, advance=False).clone()     # (sizes the workspace outside the graph)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer.prefill(off, pos, q, k, v, advance=False)
    small = layer._rows_ws.numel()
    layer.prefill(_int(0, 700), torch.arange(5000, 5700, dtype=I32, device=DEV), *_qkv(layer, 700, gen), advance=False)
    assert layer._rows_ws.numel() > small
    held = [torch.full((small,), 0x5a, dtype=torch.uint8, device=DEV) for _ in range(4)]    # whoever is given freed memory
    layer.prefill(off, pos, q, k, v, advance=False)                    # (the rows that the graph writes are there again)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(bool((h == 0x5a).all()) for h in held)


def test_a_long_call_does_not_run_out_of_time():
    """The limit of the waits is for an item's work: a call of many items may take longer (here: a limit of a millisecond, a call of two)."""
    from paper_2608_20961_b200 import binding as tw
    c = pu.make_case([0], [16384], Hq=32, Hkv=8, D=128, seed=13, poison=False)
    want, status = pu.run_chunk(c)
    assert not any(status)
    try:
        tw.treewy_debug_inject(2_000_000, -1)
        O, status = pu.run_chunk(c)
    finally:
        tw.treewy_debug_inject(0, -1)
    assert not any(status) and torch.equal(O, want)


def test_one_row_of_an_odd_size():
    """Its distance to the next is nobody's business."""
    from paper_2608_20961_b200 import attention as at
    norm, gen = at.HeadNorm(torch.ones(30, device=DEV)), torch.Generator().manual_seed(1)
    x = torch.randn(1, 3, 30, generator=gen).to(BF16)
    xs, y, dw = x.to(DEV), torch.empty((1, 3, 30), dtype=BF16, device=DEV), torch.empty(30, device=DEV)
    at.treewy_norm_rope(norm, None, xs, y)
    ref = pu.norm_reference(x, torch.ones(30), 1e-6)
    assert ((y.cpu().to(F64) - ref).abs() <= (2.0 ** -19 + pu.HALF_STEP[BF16] * 1.01) * ref.abs()).all()
    at.treewy_norm_rope_backward(norm, None, xs, y, y, dw, at.norm_rope_workspace(xs))
    with pytest.raises(ValueError):
        at.treewy_norm_rope(norm, None, xs[:, :2], y)


def test_nothing_to_do():
    from paper_2608_20961_b200 import attention as at
    layer, pool = _layer(BF16, 30, 2, True)
    off, none = _int(0, 0, 0, 0), torch.empty(0, dtype=I32, device=DEV)
    at.treewy_pages_reserve(pool, layer.cache.context_len, off, 0, none)
    O = layer.prefill(off, none, *_qkv(layer, 0, torch.Generator().manual_seed(0)))
    assert O.shape == (0, 8, 128) and not layer.cache.context_len.any() and int(pool.free_count) == pool.n_pages


@pytest.mark.parametrize("Hq,D", [(127, 64), (128, 128), (128, 256), (129, 64), (200, 128)])
def test_many_query_heads_to_one(Hq, D):
    """Up to a whole row tile to a token, and beyond it (the SIMT kernel)."""
    c = pu.make_case([300, 0], [3, 20], Hq=Hq, Hkv=1, D=D, page=16, window=90, sinks=5, seed=14)
    ref, size = pu.chunk_reference(c)
    O, status = pu.run_chunk(c)
    assert not any(status)
    pu.assert_chunk(c, O, ref, size, tensor_cores=Hq <= 128)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_outputs_on_any_16_bytes(D):
    from paper_2608_20961_b200 import attention as at
    c = pu.make_case([100, 3000], [200, 2], Hq=4, Hkv=2, D=D, seed=15, poison=False)
    want, g = pu.run_chunk(c)[0].to(DEV), pu.on_gpu(c)
    ws = at.attn_chunk_workspace(g["cache"], c.T, c.Hq)
    wide = torch.full((want.numel() + 24,), 7.0, dtype=BF16, device=DEV)
    O = wide[8:8 + want.numel()].view_as(want)                    # 16 bytes past a boundary of 32
    at.treewy_attn_chunk(g["cache"], g["offsets"], g["q"], c.scale, O, ws)
    assert torch.equal(O, want) and (wide[:8] == 7).all() and (wide[8 + want.numel():] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_sequences_than_a_grid_has_rows(dtype):
    from paper_2608_20961_b200 import attention as at
    B, D, page = 70000, 64, 16
    gen = torch.Generator().manual_seed(16)
    where = {3: 2, 65536: 1, 69999: 4}
    N = torch.zeros(B, dtype=I32)
    for b, n in where.items():
        N[b] = n
    off = torch.cat([torch.zeros(1, dtype=I32), N.cumsum(0).to(I32)]).to(DEV)
    T, L = 7, 1000
    pages = -(-(L + 4) // page)
    table = torch.arange(pages, dtype=I32, device=DEV).repeat(B, 1)              # all read the same tokens
    k, v = (torch.randn(pages, page, 1, D, generator=gen).to(dtype).to(DEV) for _ in range(2))
    q = torch.randn(T, 2, D, generator=gen).to(dtype).to(DEV)
    lens = torch.full((B,), L, dtype=I32, device=DEV)
    cache = at.KVCache(k, v, table, lens)
    O, status = torch.empty_like(q), torch.zeros(B, dtype=I32, device=DEV)
    at.treewy_attn_chunk(cache, off, q, 0.125, O, at.attn_chunk_workspace(cache, T, 2), seq_status=status)
    assert not status.any()
    one = at.KVCache(k, v, table[:1], lens[:1])
    lo = 0
    for n in where.values():
        P = torch.empty_like(q[lo:lo + n])
        at.treewy_attn_chunk(one, _int(0, n), q[lo:lo + n], 0.125, P, at.attn_chunk_workspace(one, n, 2))
        # (cut in other places: each is within its bound of the sum, |v| at most 5)
        assert (O[lo:lo + n].to(F64) - P.to(F64)).abs().max() <= (2 * 2.0 ** -7 if dtype == BF16 else 2.0 ** -17) * 5
        lo += n
    x, y = torch.randn(T, 1, D, generator=gen).to(dtype).to(DEV), torch.randn(T, 1, D, generator=gen).to(dtype).to(DEV)
    at.treewy_kv_append_norm(cache, off, x, y, at.HeadNorm(torch.ones(D, device=DEV)), seq_status=status)
    assert not status.any()


def test_two_graphs_on_one_workspace():
    """One after the other; what a call leaves there is nothing that the other reads."""
    from paper_2608_20961_b200 import attention as at
    cases = [pu.make_case([4000, 50], [3, 200], Hq=8, Hkv=2, D=128, seed=s, poison=False) for s in (1, 2)]
    cases.append(pu.make_case([100] * 20, [1] * 20, Hq=8, Hkv=2, D=128, seed=3, poison=False))
    gs = [pu.on_gpu(c) for c in cases]
    ws = max((at.attn_chunk_workspace(g["cache"], c.T, c.Hq) for g, c in zip(gs, cases)), key=lambda w: w.numel())
    outs = [torch.empty((c.T, c.Hq, c.D), dtype=BF16, device=DEV) for c in cases]
    want = [pu.run_chunk(c)[0] for c in cases]
    graphs = []
    for c, g, O in zip(cases, gs, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            at.treewy_attn_chunk(g["cache"], g["offsets"], g["q"], c.scale, O, ws)
        graphs.append(graph)
    for i in (0, 2, 1, 0, 1, 2):
        outs[i].zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i].cpu(), want[i])


def test_two_calls_at_once_with_a_workspace_each():
    from paper_2608_20961_b200 import attention as at
    c = pu.make_case([4000, 50], [3, 200], Hq=8, Hkv=2, D=128, seed=1, poison=False)
    want, g = pu.run_chunk(c)[0].to(DEV), pu.on_gpu(c)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(want) for _ in range(2)]
    spaces = [at.attn_chunk_workspace(g["cache"], c.T, c.Hq) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, O, ws in zip(streams, outs, spaces):
            at.treewy_attn_chunk(g["cache"], g["offsets"], g["q"], c.scale, O, ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(O, want) for O in outs)


def test_a_workspace_for_more_rows_is_enough_for_fewer():
    from paper_2608_20961_b200 import attention as at
    for dtype, D in ((F32, 64), (BF16, 72), (BF16, 128)):
        c = pu.make_case([3000], [1], Hq=8, Hkv=2, D=D, dtype=dtype, seed=4, poison=False)
        g = pu.on_gpu(c)
        sizes = [at.attn_chunk_workspace(g["cache"], T, c.Hq).numel() for T in (1, 2, 3, 5, 17, 64, 200, 1000, 5000, 100000)]
        assert sizes == sorted(sizes)
        O = torch.empty((1, 8, D), dtype=dtype, device=DEV)
        at.treewy_attn_chunk(g["cache"], g["offsets"], g["q"], c.scale, O, at.attn_chunk_workspace(g["cache"], 5000, c.Hq))
        assert torch.equal(O.cpu(), pu.run_chunk(c)[0])


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("skip", [0, 3])
@pytest.mark.parametrize("kind", ["prompt", "decode", "cut"])
def test_a_wait_that_runs_out_is_flagged(D, skip, kind):
    """One item's copies are never issued (nothing is in flight for it) and the waits get about a millisecond: what the call leaves
    unwritten is flagged, the rest is right, and the next call is."""
    from paper_2608_20961_b200 import binding as tw
    sizes = dict(prompt=dict(L=[50, 300, 0, 7], N=[200, 150, 300, 90]), decode=dict(L=[60, 900, 33, 400], N=[1, 1, 1, 1]),
                 cut=dict(L=[9000, 12000], N=[4, 3]))[kind]
    c = pu.make_case(Hq=4, Hkv=2, D=D, seed=12, poison=False, **sizes)
    ref, size = pu.chunk_reference_gpu(c)
    try:
        tw.treewy_debug_inject(2_000_000, skip)
        O, status = pu.run_chunk(c)
    finally:
        tw.treewy_debug_inject(0, -1)
    b = skip // c.Hkv
    assert status[b] == tw.SEQ_TIMEOUT and all(s in (0, tw.SEQ_TIMEOUT) for s in status)
    good = torch.zeros(c.T, dtype=torch.bool)
    for i, s in enumerate(status):
        good[int(c.offsets[i]):int(c.offsets[i + 1])] = s == 0
    if good.any():
        pu.assert_chunk(c, O, ref, size, tensor_cores=True, rows=good)
    O, status = pu.run_chunk(c)
    assert not any(status)
    pu.assert_chunk(c, O, ref, size, tensor_cores=True)
