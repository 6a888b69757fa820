"""AttentionLayer under flags, beside other layers, and with a shared prompt: lengths, caches and outputs against plain causal
attention in 64 bits (tests/attn_util.py states the error bounds)."""
import numpy as np
import pytest
import torch

from tests import attn_util as au

pytestmark = pytest.mark.gpu

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
DEV = "cuda:0"
HQ, HKV, D, PAGE, TOP = 4, 2, 64, 16, 400
i32 = lambda *x: torch.tensor(x, dtype=I32, device=DEV)


def random_case(L, N, seed, **kw):
    return au.make_case(L, N, Hq=HQ, Hkv=HKV, D=D, page=PAGE, poison=False, room=2, seed=seed, **kw)


def layer_of(c, context_len=None):
    """The case's cache as a layer (its keys count as rotated already), its tree, and its draft rows on the device."""
    from paper_2608_20961_b200 import attention as at
    g = au.on_gpu(c)
    cache = g["cache"] if context_len is None else at.KVCache(g["cache"].k, g["cache"].v, g["cache"].page_table, context_len)
    return at.AttentionLayer(cache, HQ, au.rope_table(D, TOP).to(DEV)), g


def positions_of(c):
    depth = [bin(int(m)).count("1") - 1 for m in c.mask.numpy().view(np.uint64)]
    seq = [b for b in range(c.B) for _ in range(c.N[b])]
    return torch.tensor([c.L[b] + d for b, d in zip(seq, depth)], dtype=I32)


def rotated(c, pos):
    """The case with its queries and keys rotated as the layer does it."""
    table = au.rope_table(D, TOP)
    c.q, c.k = (au.rope_reference(x, table, pos[None], None).to(c.dtype) for x in (c.q, c.k))
    return c


def rows_of(c, good):
    out = torch.zeros(c.T, dtype=torch.bool)
    for b in good:
        out[int(c.offsets[b]):int(c.offsets[b + 1])] = True
    return out


@pytest.mark.parametrize("words", ["both", "verify", "commit", "none"])
def test_a_position_out_of_range_is_flagged_and_not_committed(words):
    """words: which of the round's calls get the caller's status words."""
    from paper_2608_20961_b200 import attention as at
    c = random_case([30, 70, 5], [4, 6, 3], seed=1)
    layer, g = layer_of(c)
    pos = positions_of(c)
    pos[7] = TOP                                        # a node of sequence 1
    status = i32(0, 0, 0)
    O = layer.verify(g["tree"], pos.to(DEV), g["q"], g["k"], g["v"], status if words in ("both", "verify") else None)
    if words in ("both", "verify"):
        assert status.tolist() == [0, at.SEQ_BAD_POSITION, 0]
    pos[7] = 0
    ref, size = au.attn_reference(rotated(c, pos))
    au.assert_attn(c, O.cpu(), ref, size, tensor_cores=True, rows=rows_of(c, (0, 2)))
    layer.commit(g["tree"], g["k"], g["v"], i32(3, 5, 0), status if words in ("both", "commit") else None)
    if words != "none":
        assert status.tolist() == [0, at.SEQ_BAD_POSITION, 0]
    path = [bin(int(c.mask[t])).count("1") for t in (3, 10)]
    assert layer.cache.context_len.tolist() == [30 + path[0], 70, 5 + path[1]]
    # the next round has nothing left of it
    if words in ("both", "verify"):
        status.zero_()
    layer.commit(g["tree"], g["k"], g["v"], i32(-1, 0, -1))
    assert layer.cache.context_len.tolist() == [30 + path[0], 71, 5 + path[1]]


def test_rotation_flags_the_sequence_of_the_row():
    from paper_2608_20961_b200 import attention as at
    for B in (3, 70, 1100):                            # one, two and three rounds of the search for a row's sequence
        n = [b % 3 for b in range(B)]
        off = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=I32)
        T = int(off[-1])
        pos = torch.arange(T, dtype=I32) % 50
        bad = sorted({1, T // 2, T - 1})
        pos[bad] = torch.tensor([-1, 50, 1 << 30], dtype=I32)[:len(bad)]
        x = torch.randn(T, 2, 64, device=DEV)
        y, want = torch.full_like(x, 7.25), torch.full_like(x, 7.25)
        rope = at.Rope(au.rope_table(64, 50).to(DEV), pos.to(DEV))
        status = torch.zeros(B, dtype=I32, device=DEV)
        at.treewy_rope_rows(rope, off.to(DEV), x, y, seq_status=status)
        at.treewy_rope(rope, x, want)
        owner = [max(b for b in range(B) if off[b] <= t and n[b]) for t in bad]
        assert torch.equal(y, want) and (y[bad] == 7.25).all()
        assert status.tolist() == [at.SEQ_BAD_POSITION if b in owner else 0 for b in range(B)]


def decode_reference(c, pos):
    """One token a sequence: its own case, which sees the context and itself."""
    one = rotated(c, pos)
    one.mask = torch.ones(c.T, dtype=torch.int64)
    return one, *au.attn_reference(one)


def test_decoding_leaves_flagged_sequences_where_they_are():
    """Beside two good sequences: a position out of range, a page out of range, and a table that is full."""
    from paper_2608_20961_b200 import attention as at
    c = random_case([20, 33, 48, 15, 40], [1] * 5, seed=2)
    c.table[2, 3] = -1                                  # where token 48 would go
    c.table = c.table[:, :4].contiguous()
    c.L[3] = 4 * PAGE                                   # no slot left (what the table holds there does not matter)
    layer, g = layer_of(c)
    pos = torch.tensor(c.L, dtype=I32)
    pos[1] = -1
    before = layer.cache.k.clone()
    status = i32(*[0] * 5)
    O = layer.append_and_attend(g["tree"], pos.to(DEV), g["q"], g["k"], g["v"], status)
    assert status.tolist() == [0, at.SEQ_BAD_POSITION, at.SEQ_BAD_PAGE, at.SEQ_BAD_LENGTH, 0]
    assert layer.cache.context_len.tolist() == [21, 33, 48, 4 * PAGE, 41]
    changed = (layer.cache.k != before).flatten(2).any(2).nonzero().tolist()
    assert sorted(changed) == sorted([int(c.table[b, n // PAGE]), n % PAGE] for b, n in ((0, 20), (4, 40)))
    pos[1], c.L[3] = 0, 0
    one, ref, size = decode_reference(c, pos)
    au.assert_attn(one, O.cpu(), ref, size, tensor_cores=True, rows=rows_of(c, (0, 4)))
    # the position mended, the same token again: now it counts, and nothing of the first try is seen
    g2 = au.on_gpu(random_case([20, 33, 48, 15, 40], [1] * 5, seed=2))
    pos[0], pos[4] = 21, 41
    pos[1] = 33
    status.zero_()
    layer.append_and_attend(g2["tree"], pos.to(DEV), g2["q"], g2["k"], g2["v"], status)
    assert status.tolist()[:2] == [0, 0] and layer.cache.context_len.tolist() == [22, 34, 48, 4 * PAGE, 42]


def test_decoding_without_status_words_keeps_lengths_as_well():
    c = random_case([20, 33], [1, 1], seed=3)
    layer, g = layer_of(c)
    layer.append_and_attend(g["tree"], i32(20, TOP), g["q"], g["k"], g["v"])
    assert layer.cache.context_len.tolist() == [21, 33]
    layer.append_and_attend(g["tree"], i32(21, 33), g["q"], g["k"], g["v"])
    assert layer.cache.context_len.tolist() == [22, 34]


@pytest.mark.parametrize("hint", [0, 2])
def test_decoding_flags_sequences_without_exactly_one_token(hint):
    """As many rows as sequences, but two of one and none of another."""
    from paper_2608_20961_b200 import binding as tw
    c = random_case([20, 33, 9], [1, 1, 1], seed=4)
    layer, g = layer_of(c)
    tree = tw.Tree.empty(i32(0, 2, 2, 3), i32(-1, 0, -1), 1, hint)
    status = i32(0, 0, 0)
    layer.append_and_attend(tree, i32(20, 21, 9), g["q"], g["k"], g["v"], status)
    assert status.tolist() == [tw.SEQ_TOO_MANY_NODES, tw.SEQ_TOO_MANY_NODES, 0]
    assert layer.cache.context_len.tolist() == [20, 33, 10]


def test_a_tree_for_another_number_of_sequences_is_refused_before_anything_is_rotated():
    from paper_2608_20961_b200 import binding as tw
    c = random_case([20, 33], [1, 1], seed=5)
    layer, g = layer_of(c)
    q, k = g["q"].clone(), g["k"].clone()
    tree = tw.Tree.empty(i32(0, 1), i32(-1), 1)
    for call in (layer.verify, layer.append_and_attend):
        with pytest.raises(ValueError):
            call(tree, i32(20), q[:1], k[:1], g["v"][:1])
    assert torch.equal(q, g["q"]) and layer.cache.context_len.tolist() == [20, 33]


def two_layers(seed, L, N, **kw):
    """Two cases with one context_len array."""
    cases = [random_case(L, N, seed=seed + i, **kw) for i in range(2)]
    cases[1].offsets, cases[1].parent, cases[1].mask = cases[0].offsets, cases[0].parent, cases[0].mask
    context_len = i32(*L)
    layers, gs = zip(*(layer_of(c, context_len) for c in cases))
    return cases, layers, gs, context_len


def test_two_layers_on_one_length_array_decode():
    cases, layers, gs, context_len = two_layers(30, [20, 33, 64], [1, 1, 1])
    status = i32(0, 0, 0)
    for step in range(3):
        pos = torch.tensor([n + step for n in (20, 33, 64)], dtype=I32)
        gen = torch.Generator().manual_seed(step)
        for i, (c, layer, g) in enumerate(zip(cases, layers, gs)):
            c.q, c.k, c.v = (torch.randn(x.shape, generator=gen).to(BF16) for x in (c.q, c.k, c.v))
            O = layer.append_and_attend(g["tree"], pos.to(DEV), c.q.to(DEV), c.k.to(DEV), c.v.to(DEV), status, advance=i == 1)
            c.L = pos.tolist()
            one, ref, size = decode_reference(c, pos)
            au.assert_attn(one, O.cpu(), ref, size, tensor_cores=True)
            for b, n in enumerate(c.L):                 # what the next step finds
                at_ = int(c.table[b, n // PAGE]), n % PAGE
                c.kc[at_], c.vc[at_] = layer.cache.k.cpu()[at_], c.v[b]
                assert torch.equal(layer.cache.v.cpu()[at_], c.v[b])
                assert (layer.cache.k.cpu()[at_].double() - c.k[b].double()).abs().max() <= 2 * au.BF16_HALF_ULP * c.k.double().abs().max()
            assert context_len.tolist() == [n + step + i for n in (20, 33, 64)]
    assert not status.any()


@pytest.mark.parametrize("speculative", [False, True])
def test_what_one_layer_flags_the_last_one_does_not_advance(speculative):
    from paper_2608_20961_b200 import attention as at
    cases, layers, gs, context_len = two_layers(40, [20, 32, 48], [1, 1, 1])
    layers[0].cache.page_table[1, 2] = -1               # where token 32 goes, in the first layer alone
    status, pos = i32(0, 0, 0), i32(20, 32, 48)
    for i, (layer, g) in enumerate(zip(layers, gs)):
        if speculative:
            layer.verify(g["tree"], pos, g["q"], g["k"], g["v"], status)
        else:
            layer.append_and_attend(g["tree"], pos, g["q"], g["k"], g["v"], status, advance=i == 1)
    if speculative:
        for i, (layer, g) in enumerate(zip(layers, gs)):
            layer.commit(g["tree"], g["k"], g["v"], i32(0, 0, 0), status, advance=i == 1)
    assert status.tolist() == [0, at.SEQ_BAD_PAGE, 0]
    assert context_len.tolist() == [21, 32, 49]


def test_decoding_beside_a_shared_prompt():
    """The page tables' entries for the prompt are not valid pages: neither call may read them."""
    from paper_2608_20961_b200 import attention as at
    c = random_case([70, 64, 90], [1, 1, 1], seed=6, shared=64)
    layer, g = layer_of(c)
    assert (c.table[:, :4] < 0).all()
    pos, status = torch.tensor(c.L, dtype=I32), i32(0, 0, 0)
    O = layer.append_and_attend(g["tree"], pos.to(DEV), g["q"], g["k"], g["v"], status, shared_pages=g["shared_pages"], shared_len=64)
    assert not status.any() and layer.cache.context_len.tolist() == [71, 65, 91]
    one, ref, size = decode_reference(c, pos)
    au.assert_attn(one, O.cpu(), ref, size, tensor_cores=True)
    layer.cache.context_len[1] = 63                     # shorter than the prompt, with a page of its own there
    layer.cache.page_table[1, 3] = layer.cache.page_table[1, 4]
    layer.append_and_attend(g["tree"], i32(71, 63, 91), g["q"], g["k"], g["v"], status, shared_pages=g["shared_pages"], shared_len=64)
    assert status.tolist() == [0, at.SEQ_BAD_LENGTH, 0]
    assert layer.cache.context_len.tolist() == [72, 63, 92]
