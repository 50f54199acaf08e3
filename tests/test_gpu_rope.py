"""Rotary positions on the GPU against numpy in 64 bits (needs a GB300).

Tolerance.  An output is y = fl(a c) -+ fl(b s) in fp32 (or fused), rounded
once to its type.  Three fp32 roundings are at most 3 * 2^-24 (|a c| + |b s|)
<= d = 2^-22 (|a c| + |b s|).  Rounding to bf16 is monotone, so a bf16 output
lies between the roundings of ref - d and ref + d.
"""
import math

import numpy as np
import pytest
import torch

import oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd
    ipd.device_error()
    return ipd


def _freqs(rot, kind="none", base=1e6, factor=1.0, length=32768.0, fast=32.0, slow=1.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if kind == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if kind == "linear":
        return f / factor, 1.0
    if kind != "yarn":
        return f, 1.0
    at = lambda beta: rot * math.log(length / (beta * 2 * math.pi)) / (2 * math.log(base))
    lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), rot - 1)
    ramp = np.clip((i - lo) / max(hi - lo, 1e-3), 0, 1)
    return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1


@pytest.mark.parametrize("rot,max_pos,kw", [
    (128, 40000, {}), (2, 7, {}), (50, 300, {}), (256, 1000, dict(kind="linear", factor=4.0)),
    (64, 131072, dict(kind="ntk", factor=8.0)), (128, 70000, dict(kind="yarn", factor=4.0)),
    (96, 5000, dict(kind="yarn", factor=1.0, length=4096.0, base=1e4))])
def test_table(lib, rot, max_pos, kw):
    """Each entry is the 64-bit cos / sin rounded once: half an fp32 ulp of the
    magnitude, and 1e-9 for the last bit of the frequency at the longest angle."""
    t = torch.empty(max_pos, rot // 2, 2, device="cuda")
    lib.rope_table(t, base=kw.get("base", 1e6), scaling=kw.get("kind", "none"),
                   factor=kw.get("factor", 1.0), trained_len=kw.get("length", 32768.0))
    f, mag = _freqs(rot, **kw)
    a = np.arange(max_pos, dtype=np.float64)[:, None] * f
    ref = np.stack([np.cos(a), np.sin(a)], -1) * mag
    err = np.abs(t.cpu().numpy().astype(np.float64) - ref)
    assert (err <= 2.0 ** -24 * np.abs(ref) + 1e-9).all()


def _ref(x, pos, table, layout, inverse):
    """(rotated, sum of the magnitudes of its two terms) in 64 bits."""
    h = table.shape[1]
    c, s = table[pos, :, 0][:, None], table[pos, :, 1][:, None] * (-1 if inverse else 1)
    y, mag = x.copy(), np.zeros_like(x)
    ia, ib = (np.arange(h), np.arange(h) + h) if layout == 0 else (2 * np.arange(h), 2 * np.arange(h) + 1)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    mag[..., ia], mag[..., ib] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return y, mag


def _within(got, ref, mag, bf16):
    d = 2.0 ** -22 * mag
    lo, hi = ref - d, ref + d
    if bf16:
        # one rounding from 64 bits, to nearest even
        lo, hi = (O.bf16_to_f64(O.f64_to_bf16(v)) for v in (lo, hi))
    return ((lo <= got) & (got <= hi)).all()


def _np(t):
    return t.detach().cpu().double().numpy()


def _table(max_pos, rot, device="cuda"):
    f, _ = _freqs(rot, base=1e4)
    a = np.arange(max_pos)[:, None] * f
    return torch.from_numpy(np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)).to(device)


CASES = [(1, 1, 128, 128), (5, 3, 128, 64), (37, 7, 128, 96), (64, 2, 64, 64), (9, 4, 256, 256),
         (11, 5, 128, 50), (3, 2, 80, 32), (2, 1, 7, 4), (300, 40, 128, 128), (4, 1, 128, 2),
         (6, 3, 96, 96)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("n,heads,D,rot", CASES)
def test_rope(lib, n, heads, D, rot, layout, dtype):
    g = torch.Generator(device="cuda").manual_seed(n * 131 + rot)
    x = torch.randn(n, heads, D, generator=g, device="cuda").to(dtype)
    table = _table(500, rot)
    pos = torch.randint(0, 500, (n,), generator=g, device="cuda").to(torch.int32)
    pos[0], pos[-1] = 0, 499
    for inverse in (False, True):
        ref, mag = _ref(_np(x), pos.cpu().numpy(), _np(table), layout, inverse)
        out = torch.full_like(x, 7.0)
        lib.rope(x, out, pos, table, layout=layout, inverse=inverse)
        assert _within(_np(out), ref, mag, dtype == torch.bfloat16)
        # what is not rotated is the same bits
        assert torch.equal(out[..., rot:], x[..., rot:])
        here = x.clone()
        lib.rope(here, here, pos, table, layout=layout, inverse=inverse)
        assert torch.equal(here, out)
    assert lib.device_error() == 0


@pytest.mark.parametrize("offset,stride", [(0, 640), (8, 648), (3, 601), (1, 512)])
def test_rope_strided_views(lib, offset, stride):
    """Rows inside a wider buffer, aligned or not: the same values as of a
    contiguous copy, and nothing beside them written."""
    n, heads, D, rot = 21, 4, 128, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    buf = torch.randn(offset + n * stride + 16, generator=g, device="cuda").to(torch.bfloat16)
    x = buf.as_strided((n, heads, D), (stride, D, 1), offset)
    table, pos = _table(64, rot), torch.arange(n, dtype=torch.int32, device="cuda")
    want = torch.empty(n, heads, D, dtype=torch.bfloat16, device="cuda")
    lib.rope(x.contiguous(), want, pos, table)
    dst = torch.full_like(buf, 9.0)
    out = dst.as_strided((n, heads, D), (stride, D, 1), offset)
    lib.rope(x, out, pos, table)
    assert torch.equal(out, want)
    out.fill_(9.0)
    assert (dst == 9.0).all()


def test_rope_gradient(lib):
    """The transposed rotation is the gradient: against the formula's inner
    product and against central differences (the rotation is linear, so they
    are exact up to fp32 rounding: 2^-22 of the sum of magnitudes each)."""
    n, heads, D, rot = 13, 3, 128, 96
    g = torch.Generator(device="cuda").manual_seed(5)
    x, d, gy = (torch.randn(n, heads, D, generator=g, device="cuda") for _ in range(3))
    table, pos = _table(64, rot), torch.arange(n, dtype=torch.int32, device="cuda") * 4
    for layout in (0, 1):
        f = lambda t: (lambda o: (lib.rope(t, o, pos, table, layout=layout), o)[1])(torch.empty_like(t))
        gx = torch.empty_like(gy)
        lib.rope(gy, gx, pos, table, layout=layout, inverse=True)
        lhs, rhs = (_np(f(d)) * _np(gy)).sum(), (_np(d) * _np(gx)).sum()
        size = (np.abs(_np(d)) + 1).sum() * (np.abs(_np(gy)).max())
        assert abs(lhs - rhs) <= 2.0 ** -22 * size
        diff = (_np(f(x + d)) - _np(f(x - d))) / 2
        # x +- d are rounded to fp32 themselves: 2^-24 of their size, twice
        assert np.abs((diff * _np(gy)).sum() - rhs) <= 2.0 ** -20 * size * 4


def test_rope_bad_positions(lib):
    """A position outside the table is recorded and its row left alone."""
    x = torch.randn(4, 2, 128, device="cuda").to(torch.bfloat16)
    table = _table(10, 128)
    pos = torch.tensor([3, 10, -1, 9], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 5.0)
    lib.rope(x, out, pos, table)
    assert lib.device_error() == 7
    assert (out[1:3] == 5.0).all() and not (out[0] == 5.0).all() and not (out[3] == 5.0).all()
    want = torch.empty_like(x)
    lib.rope(x, want, pos.clamp(0, 9), table)
    assert torch.equal(out[[0, 3]], want[[0, 3]])
    assert lib.device_error() == 0


def test_rope_special_values(lib):
    """An infinity or NaN stays in its own pair; the rest of the row is exact."""
    x = torch.ones(2, 1, 128, device="cuda", dtype=torch.bfloat16)
    x[0, 0, 3], x[1, 0, 100] = float("inf"), float("nan")
    table, pos = _table(10, 64), torch.tensor([4, 5], dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    lib.rope(x, out, pos, table)
    bad = ~torch.isfinite(out.float())
    assert set(map(tuple, bad.nonzero().tolist())) == {(0, 0, 3), (0, 0, 35), (1, 0, 100)}


def _append_case(seed, hq, hkv, old, new, spare=3):
    g = torch.Generator().manual_seed(seed)
    R, length = len(new), [a + b for a, b in zip(old, new)]
    pages = [(x + 15) // 16 for x in length]
    num = sum(pages) + spare
    perm = torch.randperm(num, generator=g).to(torch.int32)
    table = torch.full((R, max(1, max(pages))), -1, dtype=torch.int32)
    at = 0
    for r, p in enumerate(pages):
        table[r, :p] = perm[at:at + p]
        at += p
    n = sum(new)
    rn = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    cu = torch.tensor([0] + new).cumsum(0).to(torch.int32).cuda()
    return (rn(n, hq + 2 * hkv, 128), rn(num, hkv, 16, 128), rn(num, hkv, 16, 128), cu,
            torch.tensor(length, dtype=torch.int32).cuda(), table.cuda())


APPENDS = [
    (32, 4, [100, 7, 0, 31, 64], [8, 8, 8, 1, 16], 128),
    (16, 8, [1000, 15, 16, 300], [1, 1, 1, 1], 128),
    (7, 1, [3, 50, 0], [0, 17, 33], 64),
    (10, 2, [0], [1], 50),
    (8, 8, [5] * 70, [3, 0] * 35, 96),
    (0, 4, [0, 40], [129, 5], 32),
]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("hq,hkv,old,new,rot", APPENDS)
def test_append_is_rope_then_kv_append(lib, hq, hkv, old, new, rot, layout):
    """The fused call gives the bits of rope followed by kv_append: whole pools,
    queries and keys, from strided views."""
    qkv, kp, vp, cu, length, ptab = _append_case(len(new) + rot, hq, hkv, old, new)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    n = qkv.shape[0]
    pos = torch.cat([torch.arange(o, o + m) for o, m in zip(old, new)]).to(torch.int32).cuda()
    table = _table(max(o + m for o, m in zip(old, new)) + 1, rot)
    kr = torch.empty(n, hkv, 128, dtype=torch.bfloat16, device="cuda")
    lib.rope(k, kr, pos, table, layout=layout)
    want = lib.KVCache(kp.clone(), vp.clone())
    lib.kv_append(want, kr, v.contiguous(), cu, length, ptab)
    got = lib.KVCache(kp.clone(), vp.clone())
    qo = torch.empty(n, hq, 128, dtype=torch.bfloat16, device="cuda") if hq else None
    ko = torch.empty_like(kr)
    lib.rope_append(got, q if hq else None, qo, k, v, cu, length, ptab, table, layout=layout, k_out=ko)
    assert torch.equal(got.k_pages.view(torch.int16), want.k_pages.view(torch.int16))
    assert torch.equal(got.v_pages.view(torch.int16), want.v_pages.view(torch.int16))
    assert torch.equal(ko, kr)
    if hq:
        qr = torch.empty_like(qo)
        lib.rope(q, qr, pos, table, layout=layout)
        assert torch.equal(qo, qr)
        # in place over the projection's output
        lib.rope_append(got, q, q, k, v, cu, length, ptab, table, layout=layout, k_out=k)
        assert torch.equal(q, qr) and torch.equal(k, kr)
    assert lib.device_error() == 0


def test_append_bad_rows(lib):
    """Bad offsets, lengths, pages and positions are recorded; only their rows
    are left out."""
    hq, hkv, old, new = 4, 2, [20, 3, 30, 0], [5, 4, 3, 2]
    qkv, kp, vp, cu, length, ptab = _append_case(11, hq, hkv, old, new)
    q, k, v = qkv[:, :hq].contiguous(), qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]

    def run(cu=cu, length=length, ptab=ptab, max_pos=40):
        c = lib.KVCache(kp.clone(), vp.clone())
        qo = torch.full_like(q, 3.0)
        lib.rope_append(c, q, qo, k, v, cu, length, ptab, _table(40, 128)[:max_pos].contiguous())
        return c, qo, lib.device_error()

    good, qgood, err = run()
    assert err == 0
    rows = lambda r: slice(int(cu[r]), int(cu[r + 1]))

    def only(r, c, qo):
        keep = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
        keep[rows(r)] = False
        assert torch.equal(qo[keep], qgood[keep]) and (qo[rows(r)] == 3.0).all()
        page = ptab[r, (int(length[r]) - 1) // 16]
        assert torch.equal(c.k_pages[page], kp[page]) and torch.equal(c.v_pages[page], vp[page])

    bad = ptab.clone()
    bad[0, 1] = kp.shape[0]
    c, qo, err = run(ptab=bad)
    assert err == 1
    only(0, c, qo)
    bad[0, 1] = -1
    assert run(ptab=bad)[2] == 1
    short = length.clone()
    short[1] = 2  # shorter than its four new rows
    c, qo, err = run(length=short)
    assert err == 2 and (qo[rows(1)][:2] == 3.0).all()
    c, qo, err = run(max_pos=30)  # request 2's positions are 30 .. 32
    assert err == 7
    only(2, c, qo)
    late = cu.clone()
    late[0] = 2  # the first two rows belong to no request
    c, qo, err = run(cu=late, length=torch.tensor([23, 7, 33, 2], dtype=torch.int32).cuda())
    assert err == 6 and (qo[:2] == 3.0).all() and not (qo[2] == 3.0).all()


def test_append_on_a_side_stream(lib):
    """The call runs on the stream it is given, after what that stream holds."""
    qkv, kp, vp, cu, length, ptab = _append_case(4, 16, 8, [0, 9], [2000, 100])
    q, k, v = qkv[:, :16], qkv[:, 16:24], qkv[:, 24:]
    table = _table(2001, 128)
    want = torch.empty(2100, 16, 128, dtype=torch.bfloat16, device="cuda")
    lib.rope_append(lib.KVCache(kp.clone(), vp.clone()), q, want, k, v, cu, length, ptab, table)
    qo, late = torch.empty_like(want), torch.zeros_like(qkv)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late.copy_(qkv)
    lib.rope_append(lib.KVCache(kp.clone(), vp.clone()), late[:, :16], qo, late[:, 16:24], late[:, 24:],
                    cu, length, ptab, table, stream=side)
    side.synchronize()
    assert torch.equal(qo, want)
