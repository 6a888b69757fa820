"""Windows and sinks that 32 bits do not hold are refused, not cut."""
import pytest
import torch

BF16, I32 = torch.bfloat16, torch.int32


@pytest.mark.parametrize("bad", [dict(window=1 << 31), dict(window=1 << 32), dict(window=(1 << 32) + 8), dict(window=8, sinks=1 << 32)],
                         ids=str)
def test_windows_past_32_bits_are_refused(bad):
    from paper_2608_20961_b200 import attention as at, build
    build.build()
    kv, i32 = torch.zeros(4, 8, 2, 64, dtype=BF16), lambda *s: torch.zeros(s, dtype=I32)
    cache = at.KVCache(kv, kv.clone(), i32(2, 2), i32(2))
    q, ws = torch.zeros(0, 4, 64, dtype=BF16), torch.zeros(16, dtype=torch.uint8)
    for call in (lambda **kw: at.treewy_attn_chunk(cache, i32(3), q, 1.0, q.clone(), ws, **kw), lambda **kw: at.attn_chunk_workspace(cache, 5, 4, **kw),
                 lambda **kw: at.AttentionLayer(cache, 4, torch.zeros(16, 64), **kw)):
        with pytest.raises(ValueError):
            call(**bad)
    at.AttentionLayer(cache, 4, torch.zeros(16, 64), window=(1 << 31) - 1, sinks=(1 << 31) - 1)
