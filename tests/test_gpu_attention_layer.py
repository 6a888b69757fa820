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
