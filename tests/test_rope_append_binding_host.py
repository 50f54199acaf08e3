"""rope_append's checks of what it passes on as bare pointers: offsets, lengths,
page table and pools (no GPU; a call that is let through reaches a stand-in for
the library)."""
import ctypes

import pytest
import torch

BF, I32 = torch.bfloat16, torch.int32
N, HQ, HKV, R, PAGES, MAX_PAGES = 6, 4, 2, 3, 9, 5


@pytest.fixture()
def ipd(monkeypatch):
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd as m

    class Library:
        calls = []

        def ipd_rope_append(self, desc, stream):
            self.calls.append(m._RopeAppendDesc.from_buffer_copy(desc))
            return 0

    Library.calls = []
    monkeypatch.setattr(m, "_lib", Library())
    return m


def _args(**kw):
    a = dict(k_pages=torch.zeros(PAGES, HKV, 16, 128, dtype=BF), v_pages=torch.zeros(PAGES, HKV, 16, 128, dtype=BF),
             q=torch.zeros(N, HQ, 128, dtype=BF), k=torch.zeros(N, HKV, 128, dtype=BF),
             v=torch.zeros(N, HKV, 128, dtype=BF), cu=torch.tensor([0, 1, 4, 6], dtype=I32),
             length=torch.tensor([20, 30, 40], dtype=I32), ptab=torch.zeros(R, MAX_PAGES, dtype=I32))
    return a | kw


def _call(ipd, **kw):
    a = _args(**kw)
    cache = ipd.KVCache(a["k_pages"], a["v_pages"])
    ipd.rope_append(cache, a["q"], torch.empty(N, HQ, 128, dtype=BF), a["k"], a["v"], a["cu"], a["length"], a["ptab"],
                    torch.zeros(64, 64, 2))


WIDE = torch.zeros(R, MAX_PAGES + 3, dtype=I32)
POOL = torch.zeros(PAGES, HKV, 16, 128, dtype=BF)
REFUSED = {
    "offsets of 64 bits": dict(cu=torch.tensor([0, 1, 4, 6])),
    "offsets apart": dict(cu=torch.zeros(2 * R + 2, dtype=I32)[::2]),
    "offsets in two dimensions": dict(cu=torch.zeros(R + 1, 2, dtype=I32)),
    "no offsets": dict(cu=torch.zeros(0, dtype=I32)),
    "lengths of 64 bits": dict(length=torch.tensor([20, 30, 40])),
    "lengths apart": dict(length=torch.zeros(2 * R, dtype=I32)[::2]),
    "too few lengths": dict(length=torch.zeros(R - 1, dtype=I32)),
    "page table of 64 bits": dict(ptab=torch.zeros(R, MAX_PAGES, dtype=torch.int64)),
    "columns of a wider page table": dict(ptab=WIDE[:, :MAX_PAGES]),
    "transposed page table": dict(ptab=torch.zeros(MAX_PAGES, R, dtype=I32).T),
    "too few rows of a page table": dict(ptab=torch.zeros(R - 1, MAX_PAGES, dtype=I32)),
    "flat page table": dict(ptab=torch.zeros(R * MAX_PAGES, dtype=I32)),
    "pools of 32 bits": dict(k_pages=POOL.float(), v_pages=POOL.float()),
    "value pool of another type": dict(v_pages=POOL.half()),
    "transposed key pool": dict(k_pages=torch.zeros(PAGES, 16, HKV, 128, dtype=BF).transpose(1, 2)),
    "every other page of a value pool": dict(v_pages=torch.zeros(2 * PAGES, HKV, 16, 128, dtype=BF)[::2]),
}


@pytest.mark.parametrize("what", REFUSED)
def test_refused(ipd, what):
    with pytest.raises(ipd.IpdError):
        _call(ipd, **REFUSED[what])
    assert not ipd._lib.calls


def test_pool_replaced_by_a_smaller_one(ipd):
    a = _args()
    cache = ipd.KVCache(a["k_pages"], a["v_pages"])
    cache.v_pages = a["v_pages"][:2]
    with pytest.raises(ipd.IpdError):
        ipd.rope_append(cache, None, None, a["k"], a["v"], a["cu"], a["length"], a["ptab"], torch.zeros(64, 64, 2))


@pytest.mark.parametrize("kw", [{}, dict(ptab=WIDE[:1, :MAX_PAGES], cu=torch.tensor([0, 6], dtype=I32)),
                                dict(ptab=torch.zeros(R + 2, MAX_PAGES, dtype=I32), length=torch.zeros(R + 4, dtype=I32)),
                                dict(ptab=torch.zeros(R + 2, MAX_PAGES, dtype=I32)[1:])],
                         ids=["plain", "one row of a wider table", "more rows than requests", "later rows"])
def test_passed_on(ipd, kw):
    """What is laid out as the call reads it is taken, longer buffers included."""
    _call(ipd, **kw)
    d, = ipd._lib.calls
    a = _args(**kw)
    assert (d.num_reqs, d.max_pages, d.total_new) == (a["cu"].numel() - 1, MAX_PAGES, N)
    assert d.num_pages == PAGES and ctypes.sizeof(d) == ctypes.sizeof(ipd._RopeAppendDesc)
