"""Reading and clearing the device error words of all the library's parts (needs a GB300)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd
    ipd.device_error()
    return ipd


def _rope(lib):  # a position outside the table
    x = torch.zeros(2, 1, 128, dtype=torch.bfloat16, device="cuda")
    lib.rope(x, x, torch.tensor([0, 9], dtype=torch.int32, device="cuda"), torch.zeros(4, 64, 2, device="cuda"))


def _prompt(lib):  # offsets past the tensors
    x = torch.zeros(2, 1, 128, dtype=torch.bfloat16, device="cuda")
    lib.prompt_attn(x, x, x, torch.tensor([0, 3], dtype=torch.int32, device="cuda"), 4, torch.empty_like(x), 0.1)


def _trunc(lib):  # a min_p above 1
    lib.sample_trunc(torch.zeros(1, 9, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, device="cuda"),
                     torch.empty(1, dtype=torch.int32, device="cuda"), min_p=torch.full((1,), 2.0, device="cuda"))


def _kv(lib):  # a page outside the pool
    pool = torch.zeros(2, 1, 16, 128, dtype=torch.bfloat16, device="cuda")
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    new = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device="cuda")
    lib.kv_append(lib.KVCache(pool, pool.clone()), new, new, i(0, 1), i(1), i(5).view(1, 1))


PARTS = {"rope": (_rope, 7), "prompt": (_prompt, 6), "trunc": (_trunc, 8), "kv": (_kv, 1)}


@pytest.mark.parametrize("part", PARTS)
def test_each_part_is_read_once(lib, part):
    assert lib.device_error() == 0
    for _ in range(2):  # a word that was cleared takes the next error
        PARTS[part][0](lib)
        assert lib.device_error() == PARTS[part][1]
        assert lib.device_error() == 0


def test_one_read_clears_every_part(lib):
    for f, _ in PARTS.values():
        f(lib)
    assert lib.device_error() in {code for _, code in PARTS.values()}
    assert lib.device_error() == 0
