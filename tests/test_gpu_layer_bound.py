"""An AttentionLayer's steps against attention in 64 bits of the very queries that the kernels take (rounded as the layer rounds them) over the very
cache: the kernels' bound alone, so that a window off by one, a sink that is missing or a row a token short shows."""
import numpy as np
import pytest
import torch

from tests import attn_util as au
from tests.test_gpu_prompt_paths import _int, _layer, _qkv, _reference

pytestmark = pytest.mark.gpu

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4), (64, 0), (1, 1)])
@pytest.mark.parametrize("normed", [False, True])
def test_a_layer_is_within_its_kernels_bound(dtype, window, sinks, normed):
    from paper_2608_20961_b200 import attention as at, binding as tw
    layer, pool = _layer(dtype, window, sinks, normed, seed=21)
    c, gen, B = layer.cache, torch.Generator().manual_seed(22), 3
    lens, status = [0] * B, torch.zeros(B, dtype=I32, device=DEV)
    case = type("C", (), dict(dtype=dtype))
    for N in ([200, 1, 0], [130, 300, 5], [1, 1, 1], [70, 0, 64], [1, 1, 1]):
        T, off = sum(N), _int(*np.concatenate([[0], np.cumsum(N)]).tolist())
        positions = torch.empty(T, dtype=I32, device=DEV)
        at.treewy_pages_reserve(pool, c.context_len, off, T, positions, seq_status=status)
        q, k, v = _qkv(layer, T, gen)
        rope, turned = at.Rope(layer.cos_sin, positions), torch.empty((T, layer.H_q, c.d_head), dtype=dtype, device=DEV)
        if normed:
            at.treewy_norm_rope(layer.q_norm, rope, q, turned)
        else:
            at.treewy_rope(rope, q, turned)
        if N == [1, 1, 1]:
            tree = tw.Tree.empty(off, torch.full((B,), -1, dtype=I32, device=DEV), 1, 1)
            O = layer.append_and_attend(tree, positions, q, k, v, status)
        else:
            O = layer.prefill(off, positions, q, k, v, status)
        assert not status.any()
        lo = 0
        for b, n in enumerate(N):
            if n:
                ref, size = _reference(layer, b, list(range(lens[b], lens[b] + n)), turned[lo:lo + n].to(F64))
                err = (O[lo:lo + n].to(F64) - ref).abs()
                assert (err <= au.attn_bound(case, ref, size, dtype == BF16)).all(), (N, b, float((err / size).max()))
            lo += n
        lens = [a + n for a, n in zip(lens, N)]
    assert c.context_len.tolist() == lens
