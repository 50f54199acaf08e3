"""Prompt attention on the host: refusals before any launch, and the C layout
of the binding's struct (no GPU)."""
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


def test_prompt_attn_refusals(ipd):
    L, bad = ipd.lib(), ipd.STATUS_CODES

    def call(**kw):
        a = ipd._PromptArgs(16, 16, 16, 16, 16, 16, 1024, 512, 512, 1024, 8, 4, 128, 2, 10, 6, 0.1)
        for n, v in kw.items():
            setattr(a, n, v)
        return L.ipd_prompt_attn(ctypes.byref(a), None)

    for kw in (dict(total=0), dict(num_seqs=0), dict(max_len=0)):
        assert call(**kw) == 0, kw  # nothing to do
    assert L.ipd_prompt_attn(None, None) == bad["IPD_ERR_INVALID_ARG"]
    for kw in (dict(num_seqs=-1), dict(total=-1), dict(max_len=-1), dict(num_kv_heads=0),
               dict(num_q_heads=0), dict(num_q_heads=6), dict(softmax_scale=0.0),
               dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")),
               dict(softmax_scale=float("inf")), dict(q=None), dict(k=None), dict(v=None),
               dict(out=None), dict(cu_seq=None), dict(q_stride=1016), dict(k_stride=504),
               dict(v_stride=0), dict(out_stride=-1024), dict(q=24), dict(out=8), dict(k=2),
               dict(q_stride=1028), dict(v_stride=516)):
        assert call(**kw) == bad["IPD_ERR_INVALID_ARG"], kw
    assert call(head_dim=64) == bad["IPD_ERR_UNSUPPORTED"]
    assert call(num_q_heads=129, num_kv_heads=1) == bad["IPD_ERR_UNSUPPORTED"]
    assert call(q_stride=1 << 39) == bad["IPD_ERR_UNSUPPORTED"]


def test_binding_refuses_wrong_tensors(ipd):
    bf = torch.bfloat16
    q, k, cu = torch.zeros(6, 8, 128, dtype=bf), torch.zeros(6, 4, 128, dtype=bf), torch.zeros(2, dtype=torch.int32)
    for args, lse in (((q, k, k[:5], cu, 6, q, 0.1), None), ((q, k[:5], k[:5], cu, 6, q, 0.1), None),
                      ((q, k, k, cu.long(), 6, q, 0.1), None), ((q.float(), k, k, cu, 6, q.float(), 0.1), None),
                      ((q, k, k, cu, 6, q[:, :4], 0.1), None),
                      ((q.transpose(1, 2).contiguous().transpose(1, 2), k, k, cu, 6, q, 0.1), None),
                      ((q, k, k, cu, 6, q, 0.1), torch.zeros(6, 8)), ((q, k, k, cu, 6, q, 0.1), torch.zeros(8, 6, dtype=bf))):
        with pytest.raises(ipd.IpdError):
            ipd.prompt_attn(*args, lse=lse)


@pytest.mark.skipif(not shutil.which("gcc"), reason="needs a C compiler")
def test_struct_layout(ipd, tmp_path):
    cls = ipd._PromptArgs
    src = "#include <stdio.h>\n#include <stddef.h>\n#include \"ipd.h\"\nint main(void) {\n"
    src += 'printf("%zu ", sizeof(ipd_prompt_args));\n'
    src += "".join(f'printf("%zu ", offsetof(ipd_prompt_args, {f}));\n' for f, _ in cls._fields_)
    c, exe = str(tmp_path / "l.c"), str(tmp_path / "l")
    open(c, "w").write(src + "return 0; }\n")
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), c, "-o", exe])
    want = [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    assert [int(x) for x in subprocess.check_output([exe]).split()] == want
