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
