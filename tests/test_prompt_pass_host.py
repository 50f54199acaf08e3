"""PromptPass's checks of its page table (no GPU: only the buffers are made)."""
import pytest
import torch


def _make(lens, max_pages, rows=None):
    from paper_2609_36546_gb300 import PromptPass, ipd

    pool = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    return PromptPass(ipd.KVCache(pool, pool.clone()), torch.zeros(100, 64, 2), lens,
                      torch.zeros(len(lens) if rows is None else rows, max_pages, dtype=torch.int32), 4, device="cpu")


@pytest.mark.parametrize("lens,max_pages", [([17], 1), ([1, 33, 0], 2), ([16], 0), ([96, 97], 6)])
def test_refuses_a_page_table_narrower_than_a_prompt(lens, max_pages):
    with pytest.raises(ValueError):
        _make(lens, max_pages)


@pytest.mark.parametrize("lens,max_pages", [([16], 1), ([0, 0], 1), ([0], 0), ([], 0), ([1, 32, 0], 2), ([17], 5)])
def test_takes_a_page_table_that_holds_its_prompts(lens, max_pages):
    p = _make(lens, max_pages)
    assert p.cu.tolist() == [sum(lens[:i]) for i in range(len(lens) + 1)] and p.seq_len.tolist() == lens
    assert tuple(p.page_table.shape) == (len(lens), max_pages)
