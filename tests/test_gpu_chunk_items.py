"""treewy_attn_chunk on batches in which every CTA has a run of short items of all kinds: two row tiles and one, one key tile and several,
streams without a tile.  What the roles hand to each other between items is what these are about."""
import math

import numpy as np
import pytest
import torch

from tests import prompt_util as pu

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _batch(kind, D, seed):
    """L, N of many sequences; a row tile has 128 / 2 rows here."""
    r = np.random.default_rng(seed)
    B = 160
    if kind == "pairs and tails":            # two row tiles and then one of few rows, little before them
        N = r.choice([65, 128, 129, 130, 160, 191, 200], B)
        L = r.choice([0, 0, 1, 30, 63, 64, 200], B)
    elif kind == "one key tile":             # decoding of contexts within the first tile, prompts of a tile among them
        N = r.choice([1, 1, 1, 1, 2, 60, 64], B)
        L = np.where(N == 1, r.integers(0, 63, B), 0)
    else:                                    # everything
        N = r.choice([0, 1, 1, 2, 50, 64, 65, 100, 129, 150], B)
        L = r.choice([0, 5, 62, 63, 64, 65, 127, 130, 300, 500], B)
    window, sinks = (70, 3) if kind == "all, window" else (0, 0)
    return dict(L=L.tolist(), N=N.tolist(), Hq=16, Hkv=8, D=D, page=16, window=window, sinks=sinks, seed=seed)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kind", ["pairs and tails", "one key tile", "all", "all, window"])
def test_runs_of_short_items(kind, D):
    from paper_2608_20961_b200 import attention as at
    c = pu.make_case(poison=False, **_batch(kind, D, seed=41))
    ref, size = pu.chunk_reference_gpu(c)
    want, status = pu.run_chunk(c)
    assert not any(status)
    pu.assert_chunk(c, want, ref, size, tensor_cores=True)
    g, want = pu.on_gpu(c), want.cuda()
    ws, O, words = at.attn_chunk_workspace(g["cache"], c.T, c.Hq, c.window, c.sinks), torch.empty_like(want), torch.zeros(c.B, dtype=torch.int32, device="cuda")
    for _ in range(30):
        O.fill_(7.25)
        at.treewy_attn_chunk(g["cache"], g["offsets"], g["q"], c.scale, O, ws, c.window, c.sinks, words)
        assert torch.equal(O, want)
    assert not words.any()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("L", [70, 200])     # of one row tile: two key tiles, four
def test_infinity_that_some_rows_of_one_row_tile_see(D, L):
    """Infinity among the values alone, in the last key tile and in the first one that the window leaves: taken out of the tile, and in the outputs of
    exactly the rows that see it, whichever stream has the tile and however far ahead the other is."""
    n, window = 20, 50
    many = 40                                # sequences, all of them alike: many items to a CTA
    c = pu.make_case([L] * many, [n] * many, Hq=4, Hkv=2, D=D, page=16, window=window, seed=42, poison=False)
    want = torch.zeros(c.T, c.Hq, c.D)
    for b in range(many):
        early, late = L - window + 5, L + 8 + b % 8
        for x, h, col, y in ((late, 1, 7, math.inf), (late, 0, 9, -math.inf), (early, 0, 3, math.inf)):
            c.vc[int(c.table[b, x // c.page]), x % c.page, h, col] = y
            rows = [b * n + i for i in range(n) if x in c.seen(L + i)]
            want[rows, 2 * h:2 * h + 2, col] = y
    inf = ~torch.isfinite(want)
    for _ in range(10):
        O, status = pu.run_chunk(c)
        assert not any(status)
        assert torch.equal(O[inf].float(), want[inf]) and torch.isfinite(O[~inf]).all()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("L,N", [([0], [700]), ([3000], [1]), ([1000, 30], [40, 200])], ids=["prompt", "token", "pieces"])
@pytest.mark.parametrize("bits", [7, 12, 36, 300])
def test_large_values_stay_finite(D, L, N, bits):
    """Values of 2^120 and scores that grow by `bits` (in log2) along the sequence: outputs are weighted means of the values, and so finite; the sums
    that they are the quotients of must not leave fp32 on the way."""
    c = pu.make_case(L, N, Hq=4, Hkv=2, D=D, seed=43, poison=False)
    top = max(l + n for l, n in zip(L, N))
    c.vc = (c.vc.float() * 2.0 ** 120).to(BF16)                       # (randn: up to 5 of it, below 2^123)
    for b, (l, n) in enumerate(zip(L, N)):
        x = torch.arange(l + n)
        grows = (x / top * bits * math.log(2.0) / (4 * D)).to(BF16)
        c.kc[c.table[b, x // c.page].long(), x % c.page] = grows[:, None, None].expand(-1, 2, D)
    c.q, c.scale = torch.full_like(c.q, 4.0), 1.0
    ref, size = pu.chunk_reference(c)
    for generic in (False, True):
        O, status = pu.run_chunk(c, generic=generic)
        assert not any(status) and torch.isfinite(O).all()
        # (a score is D equal products of 4 and a bf16 number, exact in fp32; the factor to log2 is off by 2^-24, which moves keys of up to 30 below the
        # maximum by 2^-19 of their weights, and exp by 2 steps: within the bounds' part for fp32)
        pu.assert_chunk(c, O, ref, size, tensor_cores=not generic)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_small_values_keep_their_bits(D):
    """Values about 2^-116, outputs down to bf16's last numbers."""
    c = pu.make_case([0, 500], [300, 1], Hq=4, Hkv=2, D=D, seed=44, poison=False)
    c.vc = (c.vc.double() * 2.0 ** -116).to(BF16)
    ref, size = pu.chunk_reference(c)
    # beside the bounds that are relative: an output's last step is 2^-133, and a sum of products (one for 16 keys) is off by 2^-149 at most, of which
    # weights of 2^-14 and more make 2^-135
    size = size + (501 / 16 * 2.0 ** -135 + 2.0 ** -134) / 2.0 ** -8
    for generic in (False, True):
        O, status = pu.run_chunk(c, generic=generic)
        assert not any(status)
        pu.assert_chunk(c, O, ref, size, tensor_cores=not generic)
