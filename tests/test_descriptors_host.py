"""The bytes that the rotary and prompt calls hand to the library, read back by
the fields' names (no GPU: a stand-in takes the calls)."""
import pytest
import torch

BF, I32 = torch.bfloat16, torch.int32


@pytest.fixture()
def ipd(monkeypatch):
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd as m

    class Library:
        def __init__(self):
            self.desc = None

        def __getattr__(self, name):
            kind = {"ipd_rope": m._RopeArgs, "ipd_rope_append": m._RopeAppendDesc, "ipd_prompt_attn": m._PromptArgs}[name]

            def call(desc, stream):
                assert stream == 77
                self.desc = kind.from_buffer_copy(desc)
                return 0
            return call

    monkeypatch.setattr(m, "_lib", Library())
    return m


def _fields(s):
    return {name: getattr(s, name) for name, _ in s._fields_}


def _rows(n, heads, wide, dtype=BF):
    return torch.zeros(n, wide, 128, dtype=dtype)[:, :heads]


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope(ipd, dtype, inverse):
    x, y, pos, table = _rows(3, 5, 6, dtype), _rows(3, 5, 9, dtype), torch.zeros(3, dtype=I32), torch.zeros(40, 31, 2)
    ipd.rope(x, y, pos, table, layout=1, inverse=inverse, stream=77)
    assert _fields(ipd._lib.desc) == dict(
        x=x.data_ptr(), y=y.data_ptr(), x_stride=6 * 128, y_stride=9 * 128, pos=pos.data_ptr(), table=table.data_ptr(),
        dtype=ipd.DTYPE_BF16 if dtype is BF else ipd.DTYPE_F32, n_tokens=3, n_heads=5, head_dim=128, max_pos=40,
        rot_dim=62, layout=1, inverse=int(inverse))


@pytest.mark.parametrize("with_q,with_k_out", [(True, True), (True, False), (False, True)])
def test_rope_append(ipd, with_q, with_k_out):
    n, hq, hkv, R = 7, 6, 3, 4
    q, qo, k, v, ko = _rows(n, hq, 7), _rows(n, hq, 8), _rows(n, hkv, 9), _rows(n, hkv, 10), _rows(n, hkv, 11)
    cache = ipd.KVCache(*(torch.zeros(13, hkv, 16, 128, dtype=BF) for _ in range(2)))
    cu, length, ptab, table = torch.zeros(R + 1, dtype=I32), torch.zeros(R, dtype=I32), torch.zeros(R, 21, dtype=I32), \
        torch.zeros(50, 32, 2)
    ipd.rope_append(cache, q if with_q else None, qo if with_q else None, k, v, cu, length, ptab, table, layout=1,
                    k_out=ko if with_k_out else None, stream=77)
    none = lambda on, value, off: value if on else off  # noqa: E731
    assert _fields(ipd._lib.desc) == dict(
        q=none(with_q, q.data_ptr(), None), q_out=none(with_q, qo.data_ptr(), None), k=k.data_ptr(), v=v.data_ptr(),
        k_out=none(with_k_out, ko.data_ptr(), None), q_stride=none(with_q, 7 * 128, 0), k_stride=9 * 128,
        v_stride=10 * 128, q_out_stride=none(with_q, 8 * 128, 0), k_out_stride=none(with_k_out, 11 * 128, 0),
        k_pages=cache.k_pages.data_ptr(), v_pages=cache.v_pages.data_ptr(), num_pages=13, cu_new=cu.data_ptr(),
        seq_len=length.data_ptr(), page_table=ptab.data_ptr(), table=table.data_ptr(),
        num_q_heads=none(with_q, hq, 0), num_kv_heads=hkv, page_size=16, head_dim=128, max_pages=21, num_reqs=R,
        total_new=n, max_pos=50, rot_dim=64, layout=1)


@pytest.mark.parametrize("with_lse", [True, False])
def test_prompt_attn(ipd, with_lse):
    n, hq, hkv = 5, 6, 2
    q, k, v, out = _rows(n, hq, 7), _rows(n, hkv, 8), _rows(n, hkv, 9), _rows(n, hq, 10)
    cu, lse = torch.zeros(4, dtype=I32), torch.zeros(hq, n)
    ipd.prompt_attn(q, k, v, cu, 17, out, 0.25, lse=lse if with_lse else None, stream=77)
    assert _fields(ipd._lib.desc) == dict(
        q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr() if with_lse else None,
        cu_seq=cu.data_ptr(), q_stride=7 * 128, k_stride=8 * 128, v_stride=9 * 128, out_stride=10 * 128, num_q_heads=hq,
        num_kv_heads=hkv, head_dim=128, num_seqs=3, total=n, max_len=17, softmax_scale=0.25)
