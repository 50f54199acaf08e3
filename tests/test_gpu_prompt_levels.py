"""Prompt attention over more sequences than a warp has lanes, of lengths that
need several query tiles, against plain attention in 64 bits (needs a GB300).
The tolerance is tests/test_gpu_prompt.py's, with its derivation."""
import pytest
import torch

from tests.test_gpu_prompt import _close, _make, _ref, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd
    ipd.device_error()
    return ipd


# a group of G heads has floor(128 / G) positions a tile, two tiles an item
@pytest.mark.parametrize("hq,hkv,R,longest", [(2, 2, 33, 900), (4, 2, 70, 500), (8, 1, 65, 160), (7, 1, 100, 200),
                                              (3, 3, 64, 600), (128, 1, 40, 9)])
def test_many_sequences_of_several_tiles(lib, hq, hkv, R, longest):
    g = torch.Generator().manual_seed(R)
    lens = torch.randint(0, longest + 1, (R,), generator=g).tolist()
    lens[R - 1] = longest           # the longest last, empty ones around it and in front
    lens[0] = lens[R - 2] = 0
    q, k, v = _make(lens, hq, hkv, seed=hq)
    out, lse = _run(lib, q, k, v, lens)
    _close(out, lse, *_ref(q, k, v, lens, 128 ** -0.5))
    assert lib.device_error() == 0


def test_a_sequence_alone_and_among_many(lib):
    """A sequence's bits do not depend on how many others the call has."""
    lens = [300, 7, 129, 0, 64] * 9
    q, k, v = _make(lens, 8, 4, seed=1)
    out, lse = _run(lib, q, k, v, lens)
    at = 0
    for n in lens[:10]:
        if n:
            s = slice(at, at + n)
            one, l1 = _run(lib, q[s].contiguous(), k[s].contiguous(), v[s].contiguous(), [n])
            assert torch.equal(one, out[s]) and torch.equal(l1, lse[:, s])
        at += n


def test_bad_offsets_among_many(lib):
    """One sequence out of 45 with offsets out of order or over the bound is
    left out; the others keep their bits."""
    lens = [200, 30, 131] * 15
    q, k, v = _make(lens, 4, 2, seed=2)
    want, _ = _run(lib, q, k, v, lens)
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
    bad = cu.clone()
    bad[19] = -1                   # 18 ends, and 19 begins, before the tensors
    for offsets, max_len, code, left_out in ((cu, 199, 2, [i for i in range(45) if lens[i] == 200]),
                                             (bad, 200, 6, [18, 19])):
        out = torch.full_like(q, 7.0)
        lib.prompt_attn(q, k, v, offsets.cuda(), max_len, out, 128 ** -0.5)
        assert lib.device_error() == code
        for i in range(45):
            s = slice(int(cu[i]), int(cu[i + 1]))
            if i not in left_out:
                assert torch.equal(out[s], want[s]), i
            else:
                assert (out[s] == 7.0).all(), i
    assert lib.device_error() == 0
