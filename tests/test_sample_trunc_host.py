"""Truncated sampling on the host: refusals before any launch (no GPU)."""
import pytest
import torch


@pytest.fixture(scope="module")
def ipd():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd as m
    return m


def test_sample_trunc_refusals(ipd):
    L, bad = ipd.lib(), ipd.STATUS_CODES

    def call(logits=16, stride=100, n=2, vocab=100, u=16, tokens=16):
        return L.ipd_sample_trunc(logits, stride, n, vocab, u, None, None, None, None, tokens, None,
                                  None, None)

    assert call(n=0) == 0
    for kw in (dict(n=-1), dict(vocab=0), dict(stride=-1), dict(logits=None), dict(u=None),
               dict(tokens=None), dict(logits=17)):
        assert call(**kw) == bad["IPD_ERR_INVALID_ARG"], kw
    assert call(vocab=ipd.TRUNC_MAX_VOCAB + 1) == bad["IPD_ERR_UNSUPPORTED"]
    assert call(n=0, vocab=ipd.TRUNC_MAX_VOCAB) == 0


def test_binding_refuses_wrong_tensors(ipd):
    l, f, i = torch.zeros(3, 10, dtype=torch.bfloat16), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    for args, kw in (((l.float(), f, i), {}), ((l, f.double(), i), {}), ((l, f[:2], i), {}),
                     ((l, f, i.long()), {}), ((l[:, ::2], f, i), {}), ((l, f, i), dict(top_k=f)),
                     ((l, f, i), dict(top_p=i)), ((l, f, i), dict(logp=f[:1])),
                     ((l, f, i), dict(n_kept=torch.zeros(6, dtype=torch.int32)[::2]))):
        with pytest.raises(ipd.IpdError):
            ipd.sample_trunc(*args, **kw)
