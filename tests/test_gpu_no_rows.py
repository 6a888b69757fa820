"""A step without packed rows (T = 0) whose offsets claim some all the same: flagged, as a range that leaves the rows is among others, and no length
is advanced by rows that are nowhere."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, I32, DEV = torch.bfloat16, torch.int32, "cuda:0"


def _int(*x):
    return torch.tensor(x, dtype=I32, device=DEV)


def _cache(at, lens):
    kv = lambda: torch.zeros((8, 16, 2, 64), dtype=BF16, device=DEV)
    return at.KVCache(kv(), kv(), torch.arange(6, dtype=I32, device=DEV).view(3, 2), lens)


# range of none; one that claims five rows; one that runs backwards from them
OFFSETS, WANT = (0, 0, 5, 0), [0, 32, 32]


@pytest.mark.parametrize("generic", [False, True])
def test_calls_flag_ranges_without_rows(generic):
    from paper_2608_20961_b200 import attention as at
    rows = lambda h: torch.zeros((0, h, 64), dtype=BF16, device=DEV)
    cache, off, norm = _cache(at, _int(3, 4, 5)), _int(*OFFSETS), at.HeadNorm(torch.ones(64, device=DEV))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    for call in (lambda s: at.treewy_kv_append(cache, off, rows(2), rows(2), seq_status=s),
                 lambda s: at.treewy_kv_append_norm(cache, off, rows(2), rows(2), norm, seq_status=s),
                 lambda s: at.treewy_attn_chunk(cache, off, rows(4), 1.0, rows(4), ws, seq_status=s, generic=generic)):
        status = _int(0, 0, 0)
        call(status)
        assert status.tolist() == WANT
        call(None)
    status = _int(0, 0, 0)                              # lengths that do not fit count for the attention, as they do among others
    at.treewy_attn_chunk(_cache(at, _int(-1, 32, 33)), _int(0, 0, 0, 0), rows(4), 1.0, rows(4), ws, seq_status=status, generic=generic)
    assert status.tolist() == [128, 0, 128]


@pytest.mark.parametrize("window", [0, 8])
@pytest.mark.parametrize("normed", [False, True])
def test_a_layer_keeps_its_lengths(window, normed):
    from paper_2608_20961_b200 import attention as at
    norm = at.HeadNorm(torch.ones(64, device=DEV)) if normed else None
    layer = at.AttentionLayer(_cache(at, _int(3, 4, 5)), 4, torch.zeros(64, 64, device=DEV), window=window, q_norm=norm, k_norm=norm)
    rows = lambda h: torch.zeros((0, h, 64), dtype=BF16, device=DEV)
    status = _int(0, 0, 0)
    layer.prefill(_int(*OFFSETS), _int(), rows(4), rows(2), rows(2), status)
    assert status.tolist() == WANT and layer.cache.context_len.tolist() == [3, 4, 5]
    layer.prefill(_int(*OFFSETS), _int(), rows(4), rows(2), rows(2))          # (with the layer's own words)
    assert layer.cache.context_len.tolist() == [3, 4, 5]


def test_more_sequences_than_a_block():
    from paper_2608_20961_b200 import attention as at
    B = 1000
    off = torch.zeros(B + 1, dtype=I32, device=DEV)
    off[700:] = 3
    kv = torch.zeros((8, 16, 2, 64), dtype=BF16, device=DEV)
    cache = at.KVCache(kv, kv.clone(), torch.zeros((B, 1), dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV))
    rows, status = torch.zeros((0, 2, 64), dtype=BF16, device=DEV), torch.zeros(B, dtype=I32, device=DEV)
    at.treewy_kv_append(cache, off, rows, rows, seq_status=status)
    want = torch.zeros(B, dtype=torch.bool)
    want[699:] = True                                   # the one that claims rows, and empty ranges behind the last row
    assert torch.equal(status.cpu() == 32, want)
