"""Paths of the attention-layer calls that need a batch of their own to be reached (tests/attn_util.py states the error bounds)."""
import pytest
import torch

from tests import attn_util as au

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"


@pytest.mark.parametrize("D", [64, 128, 256])
def test_items_of_one_and_two_tiles(D):
    """Contexts of 0 to 64 tokens: every item is the draft rows, or one tile and the draft rows, hundreds in a row for each CTA."""
    L = [(13 * b) % 65 for b in range(180)]
    c = au.make_case(L, [1 + b % 4 for b in range(180)], Hq=8, Hkv=8, D=D, seed=20)
    ref, size = au.attn_reference(c)
    for _ in range(3):
        O, status = au.run_attn(c)
        assert not any(status)
        au.assert_attn(c, O, ref, size, tensor_cores=True)


def _rows_of(c, b):
    return slice(int(c.offsets[b]), int(c.offsets[b + 1]))


@pytest.mark.parametrize("limit,skip", [(2_000_000, 0), (2_000_000, 7), (2_000_000, 61), (40_000, -1), (12_000, -1)])
@pytest.mark.parametrize("D,shared", [(64, 0), (128, 0), (256, 0), (128, 192), (256, 64)])
def test_what_a_wait_that_ran_out_left_is_flagged(D, shared, limit, skip):
    """Waits with a short limit, with one item whose copies are never issued or with work for longer: a sequence without a
    flag is right, and what was not worked out is not written, whatever the workspace held."""
    from paper_2608_20961_b200 import attention as at, binding as tw
    B, Hkv = 160, 2
    long = 9000 if skip < 0 else 300
    c = au.make_case([shared + (97 * b) % long for b in range(B)], [1 + b % 5 for b in range(B)], Hq=16, Hkv=Hkv, D=D, seed=21, shared=shared,
                     poison=False)
    g = au.on_gpu(c)
    ws = at.attn_workspace(g["cache"], g["tree"], c.Hq, shared)

    def call(fill):
        O = torch.full((c.T, c.Hq, D), 7.25, dtype=BF16, device=DEV)
        status = torch.zeros(B, dtype=torch.int32, device=DEV)
        ws.view(torch.float32)[:] = fill
        at.treewy_attn_verify(g["cache"], g["tree"], g["q"], g["k"], g["v"], c.scale, O, ws, g["shared_pages"], shared, status)
        torch.cuda.synchronize()
        return O.cpu(), status.cpu().tolist()

    good, status = call(1.0)
    assert not any(status)
    try:
        tw.treewy_debug_inject(limit, skip)
        O, status = call(1.0)
    finally:
        tw.treewy_debug_inject(0, -1)
    assert all(s in (0, tw.SEQ_TIMEOUT) for s in status) and any(status)
    if skip >= 0:
        assert status[skip // Hkv] == tw.SEQ_TIMEOUT and not all(status)
    for b in range(B):
        got, want = O[_rows_of(c, b)], good[_rows_of(c, b)]
        assert (torch.equal(got, want) if not status[b] else ((got == want) | (got == 7.25)).all()), (b, status[b])
    again, status = call(float("nan"))
    assert not any(status) and torch.equal(again, good)


def test_commit_without_rows_flags_every_sequence():
    """No packed rows at all: each tree is empty, and is flagged as an empty one in a larger batch is."""
    from paper_2608_20961_b200 import attention as at, binding as tw
    c = au.make_case([10, 20], [2, 3], Hkv=2, Hq=2, poison=False, room=1)
    g = au.on_gpu(c)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    before = g["cache"].k.clone()
    for offsets, want in (((0, 0, 0), [tw.SEQ_TOO_MANY_NODES] * 2), ((0, 0, 3), [tw.SEQ_TOO_MANY_NODES, 0])):
        tree = tw.Tree.empty(i32(*offsets), torch.full((offsets[-1],), -1, dtype=torch.int32, device=DEV), 1)
        new, status = i32(-5, -5), i32(0, 0)
        at.treewy_kv_commit(g["cache"], tree, g["k"][:offsets[-1]], g["v"][:offsets[-1]], i32(-1, -1), new, status)
        assert status.tolist() == want and new.tolist() == [-5, -5 if want[1] else 20]
    assert torch.equal(g["cache"].k, before)


@pytest.mark.parametrize("offsets,bad,written", [((0, 5, 9, 9), [1, 2], {0: 5}),          # past the rows, and none of them falls there
                                                 ((0, 2, 1, 5), [1], {0: None, 2: None}),  # backwards
                                                 ((-3, 0, 0, 5), [0], {2: 5}), ((0, 0, 0, 7), [2], {})])
def test_append_flags_ranges_that_no_row_falls_into(offsets, bad, written):
    from paper_2608_20961_b200 import attention as at, binding as tw
    c = au.make_case([3, 4, 5], [2, 2, 1], Hkv=2, Hq=2, poison=False, room=1)
    g = au.on_gpu(c)
    before = g["cache"].k.clone()
    status = torch.zeros(3, dtype=torch.int32, device=DEV)
    at.treewy_kv_append(g["cache"], torch.tensor(offsets, dtype=torch.int32, device=DEV), g["k"], g["v"], seq_status=status)
    assert status.tolist() == [tw.SEQ_BAD_OFFSETS if b in bad else 0 for b in range(3)]
    changed = (g["cache"].k != before).flatten(2).any(2)
    for b in range(3):
        rows = [bool(changed[int(c.table[b, s // c.page]), s % c.page]) for s in range(c.L[b], c.L[b] + 5)]
        if written.get(b, 0) is not None:
            assert rows == [i < written.get(b, 0) for i in range(5)], (b, rows)


@pytest.mark.parametrize("D,shared", [(64, 0), (128, 48), (256, 0)])
def test_more_sequences_than_a_cta_has_threads(D, shared):
    """Several sequences to each thread of the plan, among them empty and malformed ones, and trees of 1, 8, 16, 32 and 64 nodes."""
    from paper_2608_20961_b200 import attention as at, binding as tw
    B = 520
    c = au.make_case([shared + (29 * b) % 90 for b in range(B)], [(1, 8, 1, 16, 3, 1, 32, 2, 64, 1)[b % 10] for b in range(B)], Hq=4, Hkv=2, D=D,
                     seed=22, shared=shared)
    ref, size = au.attn_reference(c)
    O, status = au.run_attn(c)
    assert not any(status)
    au.assert_attn(c, O, ref, size, tensor_cores=True)
    bad = [b for b in range(B) if b % 37 == 5]
    for b in bad:
        c.L[b] = -1
    good = torch.ones(c.T, dtype=torch.bool)
    for b in bad:
        good[_rows_of(c, b)] = False
    O, status = au.run_attn(c, max_nodes=32)
    for b in range(B):
        if c.N[b] > 32:
            good[_rows_of(c, b)] = False
            assert status[b] == tw.SEQ_TOO_MANY_NODES
        else:
            assert status[b] == (at.SEQ_BAD_LENGTH if b in bad else 0)
    au.assert_attn(c, O, ref, size, tensor_cores=True, rows=good)
    assert (O[~good] == 7.25).all()


@pytest.mark.parametrize("Hq,Hkv,D,shared", [(16, 1, 64, 0), (40, 2, 128, 0), (24, 1, 256, 64), (32, 1, 128, 32)])
def test_more_rows_to_a_head_than_a_group_of_ctas_takes(Hq, Hkv, D, shared):
    """Trees of up to 64 nodes with 16 to 32 query heads to a key/value head: six to sixteen row tiles, beside short trees."""
    c = au.make_case([shared + n for n in (300, 0, 70, 1000, 64)], [64, 3, 40, 64, 1], Hq=Hq, Hkv=Hkv, D=D, seed=23, shared=shared)
    ref, size = au.attn_reference(c)
    for hint in (0, 64):
        O, status = au.run_attn(c, max_nodes=hint)
        assert not any(status)
        au.assert_attn(c, O, ref, size, tensor_cores=True)


@pytest.mark.parametrize("B", [33, 70, 1025, 1100])
def test_append_to_many_sequences(B):
    """More sequences than one and than two rounds of the search for a row's sequence tell apart, many without a row."""
    from paper_2608_20961_b200 import attention as at
    new = [(0, 1, 0, 0, 3)[b % 5] for b in range(B)]
    c = au.make_case([b % 7 for b in range(B)], [1] * B, Hq=1, Hkv=1, D=64, page=8, poison=False, room=1)
    g = au.on_gpu(c)
    off = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32)
    T = int(off[-1])
    k, v = (torch.randn(T, 1, 64, generator=torch.Generator().manual_seed(i)).to(BF16) for i in range(2))
    kc, vc = c.kc.clone(), c.vc.clone()
    for b in range(B):
        for i in range(new[b]):
            s, t = c.L[b] + i, int(off[b]) + i
            at_ = int(c.table[b, s // 8]), s % 8
            kc[at_], vc[at_] = k[t], v[t]
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    at.treewy_kv_append(g["cache"], off.to(DEV), k.to(DEV), v.to(DEV), seq_status=status)
    assert not status.any()
    assert torch.equal(g["cache"].k.cpu(), kc) and torch.equal(g["cache"].v.cpu(), vc)
