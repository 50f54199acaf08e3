"""Rotary entry points on the host: refusals before any launch, and the C
layout of the binding's structs (no GPU)."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ipd():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd as m
    return m


def _args(ipd, **kw):
    a = ipd._RopeArgs(16, 16, 1024, 1024, 16, 16, ipd.DTYPE_BF16, 4, 8, 128, 100, 128, 0, 0)
    for n, v in kw.items():
        setattr(a, n, v)
    return ctypes.byref(a)


def _desc(ipd, **kw):
    d = ipd._RopeAppendDesc(16, 16, 16, 16, 16, 1024, 512, 512, 1024, 512, 16, 16, 10, 16, 16, 16,
                            16, 8, 4, 16, 128, 8, 2, 3, 100, 128, 0)
    for n, v in kw.items():
        setattr(d, n, v)
    return ctypes.byref(d)


def test_rope_refusals(ipd):
    L, bad = ipd.lib(), ipd.STATUS_CODES
    call = lambda **kw: L.ipd_rope(_args(ipd, **kw), None)
    assert call(n_tokens=0) == 0
    assert L.ipd_rope(None, None) == bad["IPD_ERR_INVALID_ARG"]
    for kw in (dict(n_tokens=-1), dict(n_heads=0), dict(dtype=2), dict(rot_dim=127),
               dict(rot_dim=0), dict(rot_dim=130), dict(layout=2), dict(max_pos=0),
               dict(x=None), dict(y=None), dict(pos=None), dict(table=None), dict(table=24),
               dict(x_stride=1023), dict(y_stride=0), dict(x=17), dict(head_dim=1)):
        assert call(**kw) == bad["IPD_ERR_INVALID_ARG"], kw
    assert call(head_dim=258, rot_dim=64) == bad["IPD_ERR_UNSUPPORTED"]


def test_rope_append_refusals(ipd):
    L, bad = ipd.lib(), ipd.STATUS_CODES
    call = lambda **kw: L.ipd_rope_append(_desc(ipd, **kw), None)
    assert call(total_new=0) == 0
    assert L.ipd_rope_append(None, None) == bad["IPD_ERR_INVALID_ARG"]
    for kw in (dict(num_reqs=-1), dict(num_reqs=0), dict(total_new=-1), dict(num_pages=-1),
               dict(num_kv_heads=0), dict(num_q_heads=-1), dict(max_pages=0), dict(q=None),
               dict(q_out=None), dict(k=None), dict(v=None), dict(k_pages=None), dict(v_pages=None),
               dict(cu_new=None), dict(seq_len=None), dict(page_table=None), dict(table=None),
               dict(rot_dim=126 + 5), dict(rot_dim=130), dict(layout=-1), dict(max_pos=0),
               dict(q=24), dict(v_pages=8), dict(k_out=8), dict(q_stride=1016), dict(q_stride=1028),
               dict(k_stride=511), dict(k_out_stride=500), dict(q_out_stride=8)):
        assert call(**kw) == bad["IPD_ERR_INVALID_ARG"], kw
    assert call(page_size=32) == bad["IPD_ERR_UNSUPPORTED"]
    assert call(head_dim=64) == bad["IPD_ERR_UNSUPPORTED"]


def test_rope_table_refusals(ipd):
    L, bad = ipd.lib(), ipd.STATUS_CODES

    def call(table=16, max_pos=10, rot=128, kind=0, base=1e6, factor=2.0, length=100.0, fast=32.0,
             slow=1.0):
        s = ipd._RopeScaling(kind, base, factor, length, fast, slow)
        return L.ipd_rope_table(table, max_pos, rot, ctypes.byref(s), None)

    for kw in (dict(table=None), dict(table=8), dict(max_pos=0), dict(rot=0), dict(rot=127),
               dict(kind=4), dict(kind=-1), dict(base=1.0), dict(base=float("nan")),
               dict(base=float("inf")), dict(kind=1, factor=0.5), dict(kind=1, factor=float("nan")),
               dict(kind=2, rot=2), dict(kind=3, length=0.0), dict(kind=3, slow=0.0),
               dict(kind=3, fast=0.5), dict(kind=3, length=float("inf"))):
        assert call(**kw) == bad["IPD_ERR_INVALID_ARG"], kw
    assert call(rot=258) == bad["IPD_ERR_UNSUPPORTED"]
    assert L.ipd_rope_table(16, 10, 128, None, None) == bad["IPD_ERR_INVALID_ARG"]


def test_binding_refuses_wrong_tensors(ipd):
    t = torch.zeros(10, 64, 2)
    x = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32)
    for args in ((x, x[:2], pos, t), (x, x.clone(), pos.long(), t), (x, x.clone(), pos[:2], t),
                 (x, x.float(), pos, t), (x.half(), x.half(), pos, t), (x, x.clone(), pos, t[:, ::2]),
                 (x.transpose(0, 1), x.transpose(0, 1), torch.zeros(4, dtype=torch.int32), t),
                 (x, x.clone(), pos, t.double())):
        with pytest.raises(ipd.IpdError):
            ipd.rope(*args)
    with pytest.raises(ipd.IpdError):
        ipd.rope_table(t, scaling="other")


@pytest.mark.skipif(not shutil.which("gcc"), reason="needs a C compiler")
def test_struct_layouts(ipd, tmp_path):
    """The binding's structs have the header's layout (plain C compile)."""
    pairs = [("ipd_rope_scaling", ipd._RopeScaling), ("ipd_rope_args", ipd._RopeArgs),
             ("ipd_rope_append_desc", ipd._RopeAppendDesc)]
    src = "#include <stdio.h>\n#include <stddef.h>\n#include \"ipd.h\"\nint main(void) {\n"
    want = []
    for name, cls in pairs:
        src += f'printf("%zu ", sizeof({name}));\n'
        want.append(ctypes.sizeof(cls))
        for f, _ in cls._fields_:
            src += f'printf("%zu ", offsetof({name}, {f}));\n'
            want.append(getattr(cls, f).offset)
    c, exe = str(tmp_path / "l.c"), str(tmp_path / "l")
    open(c, "w").write(src + "return 0; }\n")
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), c, "-o", exe])
    assert [int(x) for x in subprocess.check_output([exe]).split()] == want
