"""The 8-bit cache, its attention and the drafts' verification on the host:
refusals before any launch, C layouts, and the reference's own rounding (no GPU)."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests import kv8_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ipd():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd as m
    return m


def test_reference_rounding_matches_torch():
    """Every e4m3 value, the midpoints between neighbours and values beside them."""
    v = ref.VALUES
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    x = np.concatenate([x, -x])
    got = torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.encode(x.astype(np.float32)), got)
    codes = np.arange(256, dtype=np.uint8)
    want = torch.tensor(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.decode(codes), want, equal_nan=True)
    assert ref.least_byte(448.0) == 127 and ref.least_byte(448.1) == 128 and ref.least_byte(0.0) == ref.LEAST


def _cache(ipd, **kw):
    c = ipd._KV8Cache(16, 16, 16, 16, 10, 16, 4, 128)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def test_append_refusals(ipd):
    L, bad = ipd.lib(), ipd.STATUS_CODES

    def call(n=1, cache=None, **kw):
        a = ipd._Kv8AppendDesc(cache or _cache(ipd), 16, 16, 512, 512, 16, 16, 16, 2, 2, 3)
        for k, v in kw.items():
            setattr(a, k, v)
        return L.ipd_kv8_append(ctypes.byref(a), n, None)

    assert call(total_new=0) == 0 and L.ipd_kv8_append(None, 0, None) == 0
    assert L.ipd_kv8_append(None, 1, None) == bad["IPD_ERR_INVALID_ARG"]
    assert call(n=-1) == call(n=9) == bad["IPD_ERR_INVALID_ARG"]
    for kw in (dict(num_reqs=-1), dict(num_reqs=0), dict(total_new=-1), dict(max_pages=0), dict(k_new=None),
               dict(v_new=None), dict(cu_new=None), dict(seq_len=None), dict(page_table=None), dict(k_stride=504),
               dict(v_stride=0), dict(k_stride=516), dict(v_new=24), dict(cache=_cache(ipd, num_pages=-1)),
               dict(cache=_cache(ipd, num_kv_heads=0)), dict(cache=_cache(ipd, k_pages=None)),
               dict(cache=_cache(ipd, v_pages=8)), dict(cache=_cache(ipd, k_scale=None)),
               dict(cache=_cache(ipd, v_scale=None))):
        assert call(**kw) == bad["IPD_ERR_INVALID_ARG"], kw
    for kw in (dict(page_size=32), dict(head_dim=64), dict(num_kv_heads=65)):
        assert call(cache=_cache(ipd, **kw)) == bad["IPD_ERR_UNSUPPORTED"], kw


def test_attn8_refusals(ipd):
    L, bad = ipd.lib(), ipd.STATUS_CODES

    def call(cache=None, scale=0.1, ws=256, nbytes=1 << 30, n=1, **kw):
        c = cache or _cache(ipd)
        b = ipd._Attn8Batch(ctypes.pointer(c), 32, 2, 16, 16, 16, 16, 7, 8, 4, 100, 16)
        for k, v in kw.items():
            setattr(b, k, v)
        arr = (ipd._Attn8Batch * 9)(*([b] * 9))
        size = L.ipd_attn8_workspace_size(arr, n, None, 0)
        return L.ipd_verify_attn8(arr, n, None, 0, scale, ws, nbytes, None), size

    for kw in (dict(num_q_heads=30), dict(num_q_heads=0), dict(num_reqs=-1), dict(total_q=-1), dict(max_q_len=0),
               dict(max_seq_len=3), dict(max_pages=6), dict(q=None), dict(out=None), dict(cu_q=None), dict(seq_len=None),
               dict(page_table=None), dict(q=8), dict(out=24), dict(cache=_cache(ipd, num_pages=0)),
               dict(cache=_cache(ipd, k_pages=None)), dict(cache=_cache(ipd, v_scale=None)), dict(n=9)):
        st, size = call(**kw)
        assert st == bad["IPD_ERR_INVALID_ARG"] and size == 0, kw
    for kw in (dict(cache=_cache(ipd, page_size=32)), dict(cache=_cache(ipd, head_dim=64)),
               dict(cache=_cache(ipd, num_kv_heads=65)), dict(cache=_cache(ipd, num_pages=1 << 25)),
               dict(num_q_heads=4 * 129), dict(max_pages=1 << 27, max_seq_len=(1 << 30) + 1),
               dict(num_q_heads=4 * 128, max_pages=1 << 20, max_q_len=1 << 23, max_seq_len=1 << 23)):
        st, size = call(**kw)
        assert st == bad["IPD_ERR_UNSUPPORTED"] and size == 0, kw
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=scale)[0] == bad["IPD_ERR_INVALID_ARG"]
    assert call()[1] > 0
    assert call(ws=None)[0] == call(nbytes=16)[0] == call(ws=272)[0] == bad["IPD_ERR_WORKSPACE"]
    assert call(num_reqs=0)[0] == call(total_q=0, q=None)[0] == 0 and L.ipd_verify_attn8(None, 0, None, 0, 0.1, None, 0, None) == 0


def test_draft_refusals(ipd):
    L, bad = ipd.lib(), ipd.STATUS_CODES

    def call(ws=256, nbytes=1 << 20, **kw):
        a = ipd._DraftArgs(*([16] * 3), 1000, 1000, 1000, *([16] * 10), 2, 5, 1000)
        for k, v in kw.items():
            setattr(a, k, v)
        return L.ipd_verify_draft(ctypes.byref(a), ws, nbytes, None)

    assert call(num_reqs=0) == 0
    assert L.ipd_verify_draft(None, 256, 1 << 20, None) == bad["IPD_ERR_INVALID_ARG"]
    for kw in (dict(num_reqs=-1), dict(total=-1), dict(vocab=0), dict(logits_target=None), dict(logits_draft=None),
               dict(tokens=None), dict(cu_draft=None), dict(u_accept=None), dict(u_next=None), dict(n_accept=None),
               dict(next_token=None), dict(logits_target=17), dict(logits_bonus=3), dict(target_stride=-1),
               dict(draft_stride=-8), dict(bonus_stride=-1)):
        assert call(**kw) == bad["IPD_ERR_INVALID_ARG"], kw
    assert call(vocab=ipd.TRUNC_MAX_VOCAB + 1) == bad["IPD_ERR_UNSUPPORTED"]
    assert call(ws=None) == call(nbytes=100) == call(ws=264) == bad["IPD_ERR_WORKSPACE"]
    assert 0 < L.ipd_verify_draft_workspace_size(2, 5, 1000) <= 4096
    assert L.ipd_verify_draft_workspace_size(2, -1, 1000) == 0


def test_binding_refuses_wrong_tensors(ipd):
    bf, i32, e4 = torch.bfloat16, torch.int32, torch.float8_e4m3fn
    pages = lambda *s: torch.zeros(*s, dtype=torch.uint8).view(e4)
    sc = torch.full((3, 2), 127, dtype=torch.uint8)
    for args in ((pages(3, 2, 16, 128), pages(3, 2, 16, 128), sc, sc[:2]),
                 (pages(3, 2, 16, 128), pages(2, 2, 16, 128), sc, sc),
                 (pages(3, 2, 16, 128).view(torch.uint8), pages(3, 2, 16, 128), sc, sc),
                 (pages(3, 2, 16, 128), pages(3, 2, 16, 128), sc.float(), sc),
                 (pages(3, 2, 128, 16).transpose(2, 3), pages(3, 2, 16, 128), sc, sc)):
        with pytest.raises(ipd.IpdError):
            ipd.KVCache8(*args)
    cache = ipd.KVCache8.empty(3, 2, device="cpu")
    assert cache.num_kv_heads == 2 and ipd.KVCache8(cache.k_pages, cache.v_pages,
                                                    sc.view(torch.float8_e8m0fnu), sc).num_kv_heads == 2
    k, cu, ln, tab = torch.zeros(3, 2, 128, dtype=bf), torch.tensor([0, 3], dtype=i32), torch.tensor([3], dtype=i32), \
        torch.zeros(1, 2, dtype=i32)
    for args in ((k.float(), k, cu, ln, tab), (k[:, :1], k, cu, ln, tab), (k, k[:2], cu, ln, tab),
                 (k, k, cu.long(), ln, tab), (k, k, cu, ln.long(), tab), (k, k, cu, ln, tab[0]),
                 (k, k, torch.zeros(3, dtype=i32), ln, tab), (k, k, cu, ln, torch.zeros(2, 2, dtype=i32).T[:1]),
                 (k.transpose(1, 2).contiguous().transpose(1, 2), k, cu, ln, tab)):
        with pytest.raises(ipd.IpdError):
            ipd.kv8_append(cache, *args)
    q = torch.zeros(3, 4, 128, dtype=bf)
    for args in ((q.float(), cu, ln, tab, q), (q, cu, ln, tab, q[:2]), (q, cu.long(), ln, tab, q), (q, cu, ln, tab[:0], q),
                 (q[:, :, :64], cu, ln, tab, q[:, :, :64]), (q, cu[:1], ln, tab, q)):
        with pytest.raises(ipd.IpdError):
            ipd.AttnBatch8(cache, *args, 3, 3)
    lg, n1, f3, f1 = torch.zeros(3, 50, dtype=bf), torch.zeros(1, dtype=i32), torch.zeros(3), torch.zeros(1)
    ws = torch.zeros(256, dtype=torch.uint8)
    good = [lg, lg, torch.zeros(3, dtype=i32), cu, f3, f1, n1, n1, ws]
    for at, t in ((0, lg.float()), (1, lg[:, :49]), (1, lg[:2]), (2, torch.zeros(3, dtype=torch.int64)), (4, f1), (5, f3),
                  (6, f1), (7, torch.zeros(2, dtype=i32)), (0, torch.zeros(50, 3, dtype=bf).T)):
        with pytest.raises(ipd.IpdError):
            ipd.verify_draft(*[t if j == at else g for j, g in enumerate(good)])
    for kw in (dict(logits_bonus=lg), dict(inv_temp_target=f3), dict(logp_draft=f1)):
        with pytest.raises(ipd.IpdError):
            ipd.verify_draft(*good, **kw)


@pytest.mark.skipif(not shutil.which("gcc"), reason="needs a C compiler")
def test_struct_layouts(ipd, tmp_path):
    src, want = "#include <stdio.h>\n#include <stddef.h>\n#include \"ipd.h\"\nint main(void) {\n", []
    for name, cls in (("ipd_kv8_cache", ipd._KV8Cache), ("ipd_kv8_append_desc", ipd._Kv8AppendDesc),
                      ("ipd_attn8_batch", ipd._Attn8Batch), ("ipd_draft_args", ipd._DraftArgs)):
        src += f'printf("%zu ", sizeof({name}));\n'
        src += "".join(f'printf("%zu ", offsetof({name}, {f}));\n' for f, _ in cls._fields_)
        want += [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    c, exe = str(tmp_path / "l.c"), str(tmp_path / "l")
    open(c, "w").write(src + "return 0; }\n")
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), c, "-o", exe])
    assert [int(x) for x in subprocess.check_output([exe]).split()] == want
