"""Pages of a prompt that two sequences share: the pool does not count who holds them, so they go back with the last sequence."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _int(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_a_shared_prompts_pages_go_back_with_the_last_sequence():
    from paper_2608_20961_b200 import attention as at
    page, prompt = 8, 24
    pool, status = at.PagePool.empty(3, 6, page, 12, DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    lens = _int(0, 0, 0)
    at.treewy_pages_reserve(pool, lens, _int(0, prompt, prompt, prompt), prompt, seq_status=status)
    pool.page_table[1:, :3] = pool.page_table[0, :3]                     # the others read the first one's prompt
    lens.fill_(prompt)
    at.treewy_pages_reserve(pool, lens, _int(0, 10, 11, 20), 20, seq_status=status)
    held = pool.page_table[0, :3].tolist()
    ends = _int(prompt + 16, prompt + 8, prompt + 16)
    at.treewy_pages_release(pool, _int(prompt, 1 << 30, prompt), ends, status)      # two sequences end: their own pages
    assert pool.page_table[0].tolist() == held + [-1] * 3 and pool.page_table[2].tolist() == held + [-1] * 3
    free = lambda: pool.free_pages[:int(pool.free_count)].tolist()
    assert not set(free()) & set(held) and len(set(free())) == len(free()) == 12 - 3 - 1
    pool.page_table[0], pool.page_table[2] = -1, -1                      # (the tables' rows are the caller's to empty)
    at.treewy_pages_release(pool, _int(0, 0, 0), ends, status)                      # the last one: with the prompt's
    assert sorted(free()) == list(range(12)) and not status.any() and (pool.page_table == -1).all()
