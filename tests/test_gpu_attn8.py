"""Attention over the 8-bit cache on the GPU against plain attention in 64 bits
over the values its bytes stand for (needs a GB300).

Tolerance, with a = sum_j w_j |v_j| the weighted mean magnitude of what an output
averages: the weights enter the product with V as two e4m3 terms, off by at most
2^-9 of themselves and 2^-18 of the row's largest weight times scale, which over
all keys is c = 2^-18 max_j (w_j 2^ev_j) sum_j |entry_j|; the output is rounded to
bf16, 2^-8 (|o| + 2^-9 a).  q is exact to 2^-18 of its row's largest entry: a score
of 128 terms is off by at most 128 2^-18 |q|max |k|max scale, below 2^-9 at the
magnitudes here (4, 4 and 1 / 11.3 for most, checked for each case), and so is a
weight, relative to itself; fp32 scores and sums stay far below.  Together
2^-8 |o| + (2^-9 + 2^-9 + 2^-10) a + c.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

D = 128
E4 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd
    ipd.device_error()
    return ipd


class Case:
    def __init__(self, hq, hkv, q_len, length, seed=0, spread=2, spare=4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
        ri = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda")
        self.hq, self.hkv, self.q_len, self.length = hq, hkv, q_len, length
        pages = [(x + 15) // 16 for x in length]
        n = sum(pages) + spare
        perm, at = torch.randperm(n, generator=g, device="cuda").to(torch.int32), 0
        self.table = torch.full((len(length), max(1, max(pages))), -1, dtype=torch.int32, device="cuda")
        for r, x in enumerate(pages):
            self.table[r, :x] = perm[at:at + x]
            at += x
        self.unused = perm[at:].long()
        self.kp, self.vp = ((rn(n, hkv, 16, D) * 100).clamp(-448, 448).to(E4) for _ in "kv")
        self.ks, self.vs = ((120 + ri(-spread, spread + 1, n, hkv)).to(torch.uint8) for _ in "kv")
        self.ks.clamp_(max=120)
        self.q = rn(sum(q_len), hq, D).to(torch.bfloat16)
        self.n = n

    def batch(self, lib, out=None):
        cu = torch.tensor([0] + self.q_len).cumsum(0).to(torch.int32).cuda()
        self.out = torch.full_like(self.q, 7.0) if out is None else out
        cache = lib.KVCache8(self.kp, self.vp, self.ks, self.vs)
        return lib.AttnBatch8(cache, self.q, cu, torch.tensor(self.length, dtype=torch.int32, device="cuda"), self.table,
                              self.out, max(1, max(self.q_len)), max(1, max(self.length)))

    def wide(self, r, h):
        page = self.table[r, :(self.length[r] + 15) // 16].long()
        one = lambda p, s: (p.view(torch.uint8)[page, h].view(E4).double(), torch.exp2(s[page, h].double() - 127)[:, None, None])
        (k, fk), (v, fv) = one(self.kp, self.ks), one(self.vp, self.vs)
        n = self.length[r]
        return (k * fk).view(-1, D)[:n], v.view(-1, D)[:n], fv.expand(-1, 16, 1).reshape(-1)[:n]

    def ref(self, scale):
        """(output, tolerance) in 64 bits; only visible keys enter a sum."""
        out = torch.zeros(self.q.shape, dtype=torch.float64, device="cuda")
        tol, G, row = torch.zeros_like(out), self.hq // self.hkv, 0
        for r, n in enumerate(self.q_len):
            for h in range(self.hkv):
                k, v, fv = self.wide(r, h) if n else (None,) * 3
                for i in range(n):
                    m = self.length[r] - n + i + 1
                    q = self.q[row + i, h * G:(h + 1) * G].double()
                    w = torch.softmax(q @ k[:m].T * scale, -1) * fv[:m]
                    x = v[:m]
                    if torch.isfinite(x).all():
                        o, a, s = w @ x, w @ x.abs(), x.abs().sum(0)
                    else:
                        o = (w[:, :, None] * x).sum(1)
                        a, s = ((w[:, :, None] * x.abs()).sum(1).nan_to_num(), x.abs().nan_to_num().sum(0))
                    c = 2.0 ** -18 * w.amax(-1, keepdim=True) * s
                    out[row + i, h * G:(h + 1) * G] = o
                    tol[row + i, h * G:(h + 1) * G] = 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -10) * a + c
            row += n
        return out, tol


def _run(lib, *cases, scale=D ** -0.5, decode=0):
    bs = [c.batch(lib) for c in cases]
    v, d = bs[:len(bs) - decode], bs[len(bs) - decode:]
    ws = torch.full((max(256, lib.attn8_workspace_size(v, d)),), 0xff, dtype=torch.uint8, device="cuda")
    lib.verify_attn8(v, d, scale, ws)
    return ws


def _check(c, scale=D ** -0.5):
    want, tol = c.ref(scale)
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(c.out))
    err = (c.out.double() - want).abs()
    assert bool((err <= tol)[fine].all()), float((err / tol)[fine].max())
    return float((err / tol.clamp_min(1e-30))[fine].max()) if fine.any() else 0.0


@pytest.mark.parametrize("hq,hkv,q_len,length", [
    (16, 8, [1], [1]), (16, 8, [1], [77]), (32, 4, [1], [1000]), (16, 8, [1, 1, 1, 1, 1], [15, 16, 17, 128, 129]),
    (16, 8, [1, 0, 1], [127, 5, 2049]),
    (32, 4, [16, 5, 1, 0, 8], [16, 300, 129, 0, 1024]),         # spans up to 128 rows; a whole prompt as a span
    (32, 4, [8, 9, 2], [500, 501, 640]), (10, 2, [9, 3, 0, 1], [9, 1500, 77, 31]), (7, 1, [3, 1], [200, 7]),
    (12, 4, [5, 11], [640, 127]), (8, 8, [1, 16], [33, 400]), (128, 1, [1, 2], [300, 130]), (100, 1, [3], [257]),
    (64, 1, [1, 1], [4000, 20]), (1, 1, [40], [1025]), (64, 64, [2], [90]), (2, 1, [100, 17], [100, 300])])
def test_attn8(lib, hq, hkv, q_len, length):
    c = Case(hq, hkv, q_len, length, seed=hq + len(length))
    _run(lib, c)
    _check(c)
    assert lib.device_error() == 0


@pytest.mark.parametrize("hq,hkv,q,length", [(32, 4, 1, 30011), (16, 8, 1, 9000), (32, 4, 13, 20000), (4, 2, 3, 70001)])
def test_long_contexts_are_split(lib, hq, hkv, q, length):
    c = Case(hq, hkv, [q], [length], seed=q)
    _run(lib, c)
    _check(c)


def test_many_requests(lib):
    """More requests than CTAs, lengths 1 to 400, spans 0 to 6."""
    g = torch.Generator().manual_seed(1)
    length = torch.randint(1, 401, (400,), generator=g).tolist()
    q_len = [min(int(x), n) for x, n in zip(torch.randint(0, 7, (400,), generator=g), length)]
    c = Case(8, 2, q_len, length, seed=2)
    _run(lib, c)
    _check(c)


@pytest.mark.parametrize("hq,hkv,q_hi,n,lo,hi", [(16, 8, 1, 60, 1500, 5000), (32, 4, 16, 50, 200, 4000), (8, 8, 9, 40, 100, 3000),
                                                 (12, 2, 14, 90, 1, 2600), (16, 8, 1, 500, 100, 900)])
def test_many_long_requests(lib, hq, hkv, q_hi, n, lo, hi):
    """Several tasks a CTA of more tiles than any ring holds, of every number of
    warpgroups; the same bytes again and again."""
    g = torch.Generator().manual_seed(hq)
    length = torch.randint(lo, hi + 1, (n,), generator=g).tolist()
    q_len = [min(int(x), m) for x, m in zip(torch.randint(0 if q_hi > 1 else 1, q_hi + 1, (n,), generator=g), length)]
    c = Case(hq, hkv, q_len, length, seed=n)
    _run(lib, c)
    _check(c)
    first = c.out.clone()
    for _ in range(5):
        _run(lib, c)
        assert torch.equal(c.out, first)
    assert lib.device_error() == 0


@pytest.mark.parametrize("hq,hkv,q_lo,q_hi,n,hi", [(32, 4, 4, 7, 300, 3000), (32, 4, 1, 16, 300, 1500), (32, 4, 3, 12, 200, 150),
                                                   (64, 8, 1, 5, 100, 700)])
def test_tasks_of_different_widths_side_by_side(lib, hq, hkv, q_lo, q_hi, n, hi):
    """Tasks of one, two and four warpgroups in turn in every CTA, warpgroups that wait for
    their tiles among them."""
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        length = torch.randint(q_hi, hi + 1, (n,), generator=g).tolist()
        q_len = torch.randint(q_lo, q_hi + 1, (n,), generator=g).tolist()
        c = Case(hq, hkv, q_len, length, seed=seed)
        _run(lib, c)
        if seed == 0:
            _check(c)
        first = c.out.clone()
        for _ in range(10):
            _run(lib, c)
        assert torch.equal(c.out, first)
        assert lib.device_error() == 0


def test_several_batches_in_one_call(lib):
    """Spans over two caches and decode tokens over both, and a batch without
    queries: the same bytes as one call each."""
    cs = [Case(32, 4, [8, 3], [300, 4000], seed=1), Case(16, 8, [2, 16], [900, 31], seed=2), Case(4, 4, [0], [20], seed=3),
          Case(16, 8, [1, 1, 1], [100, 2, 3000], seed=4), Case(32, 4, [1], [777], seed=5)]
    _run(lib, *cs, decode=2)
    for c in cs:
        _check(c)


def test_scores_that_grow_and_fall(lib):
    """Keys that grow along the sequence by powers of two (the running maximum moves
    far, tile after tile) and that fall; and large queries."""
    for sign in (1, -1):
        for q_len, length in (([1, 1], [3000, 513]), ([16, 9], [2000, 700])):
            c = Case(32, 4, q_len, length, seed=7)
            for r in range(2):
                n = (length[r] + 15) // 16
                step = torch.arange(n, device="cuda") * 6 // n
                c.ks[c.table[r, :n].long()] = ((118 + sign * step) if sign > 0 else (124 - step)).to(torch.uint8)[:, None]
            # q is exact to 2^-18: scores of up to 2^7 larger keys need smaller queries
            c.q.mul_(2.0 ** -4)
            _run(lib, c)
            _check(c)


def test_values_of_very_different_scale(lib):
    """Pages whose V scales lie 60 binades apart, dominated by either kind; zero
    pages with the least scale."""
    for far in (30, -30):
        c = Case(16, 8, [1, 4], [900, 2000], seed=3, spread=0)
        for r in range(2):
            page = c.table[r, ::3][c.table[r, ::3] >= 0].long()
            c.vs[page] = torch.tensor(120 + far, dtype=torch.uint8, device="cuda")
            c.vs[c.table[r, 0].long()] = 60
            zero = c.table[r, 1].long()
            c.vs[zero] = 87
            c.vp.view(torch.uint8)[zero] = 0
        _run(lib, c)
        _check(c)
        # weights that fall steeply: the pages of the larger scale have next to no weight
        c.ks[c.table[:, ::3][c.table[:, ::3] >= 0].long()] = 90
        c.q.mul_(4.0)
        _run(lib, c)
        _check(c)


def test_equal_keys_and_one_row_of_weight(lib):
    """All keys equal (the output is the mean of V), and one key far above the rest."""
    c = Case(32, 4, [2], [5000], seed=5)
    c.kp.view(torch.uint8)[:] = 0x30
    c.ks.fill_(115)
    _run(lib, c)
    _check(c)
    c.kp.view(torch.uint8)[c.table[0, 3].long(), :, 5] = (torch.sign(c.q[0, ::8].float()) * 100).to(E4).view(torch.uint8)
    _run(lib, c)
    _check(c)


def test_hidden_bytes_reach_nothing(lib):
    """NaN in every slot that no row sees: behind a sequence's end, in unused pages,
    in scales of unused pages; and NaN in a span's own keys reaches the rows that see
    them, no other."""
    c = Case(32, 4, [1, 6, 3, 16], [77, 300, 16, 250], seed=6)
    want, tol = c.ref(D ** -0.5)
    for r, n in enumerate(c.length):
        if n % 16:
            page = c.table[r, n // 16].long()
            c.kp.view(torch.uint8)[page, :, n % 16:] = 0x7f
            c.vp.view(torch.uint8)[page, :, n % 16:] = 0xff
    for p, s in ((c.kp, c.ks), (c.vp, c.vs)):
        p.view(torch.uint8)[c.unused] = 0x7f
        s[c.unused] = 255
    _run(lib, c)
    assert bool(((c.out.double() - want).abs() <= tol).all())
    # the span's 4th key of request 1: V in some dims, K of its 5th in one head
    at = lambda r, pos: (c.table[r, pos // 16].long(), pos % 16)
    page, slot = at(1, 294 + 3)
    c.vp.view(torch.uint8)[page, 2, slot, 3:40] = 0x7f
    page, slot = at(1, 294 + 4)
    c.kp.view(torch.uint8)[page, 1, slot, 7] = 0xff
    page, slot = at(3, 234 + 15)
    c.vp.view(torch.uint8)[page, :, slot, 100] = 0x7f
    want, tol = c.ref(D ** -0.5)
    _run(lib, c)
    nan = torch.isnan(want)
    assert int(nan.sum()) == 3 * 8 * 37 + 2 * 8 * 128 + 32
    _check(c)


def test_hidden_nan_in_tasks_side_by_side(lib):
    """NaN in V of spans' own keys, in some of many short requests of every width: tasks of one, two
    and four warpgroups note them while others end."""
    g = torch.Generator().manual_seed(2)
    n = 150
    q_len = torch.randint(1, 17, (n,), generator=g).tolist()
    length = [q + int(x) for q, x in zip(q_len, torch.randint(0, 300, (n,), generator=g))]
    c = Case(32, 4, q_len, length, seed=12)
    for r in torch.randperm(n, generator=g)[:90].tolist():
        pos = length[r] - 1 - int(torch.randint(0, q_len[r], (1,), generator=g))
        page, head, dim = int(c.table[r, pos // 16]), int(torch.randint(0, 4, (1,), generator=g)), int(torch.randint(0, 128, (1,), generator=g))
        c.vp.view(torch.uint8)[page, head, pos % 16, dim] = 0x7f
    _run(lib, c)
    _check(c)
    first = c.out.nan_to_num(nan=77.0).clone()
    for _ in range(20):
        _run(lib, c)
        assert torch.equal(c.out.nan_to_num(nan=77.0), first)
    assert lib.device_error() == 0


def test_rows_do_not_reach_each_other(lib):
    """A NaN and an infinite query, and one 2^40 times as large, beside ordinary ones."""
    c = Case(32, 4, [3, 1], [300, 900], seed=8)
    want, tol = c.ref(D ** -0.5)
    c.q[1, 5, 3] = float("nan")
    c.q[2, 9, 100] = float("inf")
    c.q[0, 20] *= 2.0 ** 40
    _run(lib, c)
    keep = torch.ones(4, 32, dtype=torch.bool, device="cuda")
    keep[1, 5] = keep[2, 9] = keep[0, 20] = False
    assert bool(((c.out.double() - want).abs() <= tol)[keep].all())
    assert bool(torch.isnan(c.out[1, 5]).all())
    # the large query's weight lies on its best key alone
    k, v, fv = c.wide(0, 2)
    m = 300 - 3 + 1
    best = (c.q[0, 20].double() @ k[:m].T).argmax()
    assert bool(((c.out[0, 20].double() - v[best] * fv[best]).abs() <= 2.0 ** -7 * v[best].abs() * fv[best] + 1e-9).all())


def test_nan_scales_and_zero_queries(lib):
    c = Case(16, 8, [1, 1, 2], [100, 200, 300], seed=9)
    c.q[1].zero_()  # equal weights
    c.ks[c.table[0, 2].long(), 3] = 255
    c.vs[c.table[2, 1].long(), 6] = 255
    _run(lib, c)
    keep = torch.ones(4, 16, dtype=torch.bool, device="cuda")
    keep[0, 6:8] = keep[2:, 12:14] = False
    want, tol = c.ref(D ** -0.5)
    assert bool(((c.out.double() - want).abs() <= tol)[keep].all())
    assert bool(torch.isnan(c.out[~keep]).all())


def test_bad_pages_lengths_and_offsets(lib):
    """A page outside the pool leaves its keys out (all of them: zeros); a request
    with a bad length or offsets is not written; the others are as they were."""
    c = Case(16, 8, [1, 2, 1, 3], [100, 200, 33, 300], seed=10)
    want, tol = c.ref(D ** -0.5)
    for what, code in (("page", 1), ("all pages", 1), ("length", 2), ("short", 2), ("offsets", 6)):
        b = c.batch(lib)
        q, cu, ln, table, out = b._keep
        table, other = table.clone(), slice(1, 3)
        if what == "page":
            table[1, 3] = c.n + 9
        elif what == "all pages":
            table[1] = -1
        elif what == "length":
            ln[1] = 301
        elif what == "short":
            ln[1] = 1
        else:
            cu[2] = 9  # past the tensor for request 1, out of order for request 2
            other = slice(1, 4)
        cache = lib.KVCache8(c.kp, c.vp, c.ks, c.vs)
        b = lib.AttnBatch8(cache, q, cu, ln, table, out, 3, 300)
        ws = torch.empty(lib.attn8_workspace_size([b]), dtype=torch.uint8, device="cuda")
        lib.verify_attn8([b], [], D ** -0.5, ws)
        assert lib.device_error() == code, what
        rest = torch.ones(7, dtype=torch.bool, device="cuda")
        rest[other] = False
        assert bool(((out.double() - want).abs() <= tol)[rest].all()), what
        if what == "all pages":
            assert bool((out[1:3] == 0).all())
        elif what == "page":
            keys = torch.ones(200, dtype=torch.bool, device="cuda")
            keys[48:64] = False
            k, v, fv = c.wide(1, 5)
            w = torch.softmax(c.q[1, 10].double() @ k[:199][keys[:199]].T * D ** -0.5, -1)
            o = w @ (v * fv[:, None])[:199][keys[:199]]
            assert bool(((out[1, 10].double() - o).abs() < 0.02).all())
        else:
            assert bool((out[other] == 7.0).all()), what


def test_rows_behind_the_last_request_stay(lib):
    c = Case(16, 8, [1, 2], [50, 60], seed=11)
    c.q = torch.cat([c.q, c.q])
    b = c.batch(lib)
    ws = torch.empty(lib.attn8_workspace_size([b]), dtype=torch.uint8, device="cuda")
    lib.verify_attn8([b], [], D ** -0.5, ws)
    assert bool((c.out[3:] == 7.0).all()) and not bool((c.out[:3] == 7.0).all(-1).any())


def test_captured_twice_over_one_workspace(lib):
    """Two captured calls that share a workspace, replayed in turn with new contents,
    and a call on another stream: bytes as those of a plain call, time after time."""
    c1, c2 = Case(32, 4, [4, 1], [900, 3000], seed=12), Case(16, 8, [1, 1], [5000, 40], seed=13)
    b1, b2 = c1.batch(lib), c2.batch(lib)
    ws = torch.empty(max(lib.attn8_workspace_size([b]) for b in (b1, b2)), dtype=torch.uint8, device="cuda")
    for b in (b1, b2):
        lib.verify_attn8([b], [], D ** -0.5, ws)
    plain = [b.out.clone() for b in (b1, b2)]
    graphs = []
    for b in (b1, b2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            lib.verify_attn8([b], [], D ** -0.5, ws)
        graphs.append(g)
    for _ in range(3):
        for b in (b1, b2):
            b.out.fill_(7.0)
        ws.fill_(0xff)
        for g in graphs:
            g.replay()
        assert all(torch.equal(b.out, p) for b, p in zip((b1, b2), plain))
    c1.q.copy_(torch.randn_like(c1.q.float()))
    graphs[0].replay()
    _check(c1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b2.out.fill_(7.0)
    torch.cuda.synchronize()
    lib.verify_attn8([b2], [], D ** -0.5, ws, stream=s)
    s.synchronize()
    assert torch.equal(b2.out, plain[1])


def test_pools_past_32_bits(lib):
    """Pages at the end of a pool of more than 2^32 bytes a tensor."""
    n, hkv = (1 << 18) + 64, 8
    cache = lib.KVCache8.empty(n, hkv)
    c = Case(16, 8, [2], [700], seed=14)
    pages = c.table[0].long()
    high = torch.arange(n - 60, n - 60 + len(pages), device="cuda")
    for a, b in ((cache.k_pages, c.kp), (cache.v_pages, c.vp)):
        a.view(torch.uint8)[high] = b.view(torch.uint8)[pages]
    cache.k_scale[high], cache.v_scale[high] = c.ks[pages], c.vs[pages]
    b = c.batch(lib)
    q, cu, ln, _, out = b._keep
    b = lib.AttnBatch8(cache, q, cu, ln, high.to(torch.int32)[None].contiguous(), out, 2, 700)
    ws = torch.empty(lib.attn8_workspace_size([b]), dtype=torch.uint8, device="cuda")
    lib.verify_attn8([b], [], D ** -0.5, ws)
    _check(c)


def _rows_ref(c, r, h, keep=None, scale=D ** -0.5, ends=False, block=None):
    """(output, tolerance) of request r's rows over KV head h in 64 bits, over the keys in `keep`:
    the tolerance is the weights' and the output's rounding alone, relative to what an
    output averages: 2^-8 |o| + (2^-8 + 2^-10) a, a = sum_j w_j |v_j|.  With `ends` also what the
    weights' two terms end at: half of e4m3's least value over the second's factor, 2^-10 / 32, beside
    a largest weight of 2^4 or more: 2^-19 of the row's largest weight times scale, per entry.  With
    `block` that of the keys in this block of 128 alone, which may be missing whole: sum w_j |v_j|."""
    G, n, L = c.hq // c.hkv, c.q_len[r], c.length[r]
    row, page = sum(c.q_len[:r]), c.table[r, :(L + 15) // 16].long().clamp(0, c.n - 1)
    one = lambda p, s: (p.view(torch.uint8)[page, h].view(E4).double() *
                        torch.exp2(s[page, h].double() - 127)[:, None, None]).view(-1, D)[:L]
    k, v = one(c.kp, c.ks), one(c.vp, c.vs)
    fv = torch.exp2(c.vs[page, h].double() - 127)[:, None].expand(-1, 16).reshape(-1)[:L]
    keep = torch.ones(L, dtype=torch.bool, device="cuda") if keep is None else keep
    out, tol = [], []
    for i in range(n):
        m = keep.clone()
        m[L - n + i + 1:] = False
        w = torch.softmax(c.q[row + i, h * G:(h + 1) * G].double() @ k[m].T * scale, -1)
        o, a = w @ v[m], w @ v[m].abs()
        c0 = 2.0 ** -19 * (w * fv[m]).amax(-1, keepdim=True) * (v[m] / fv[m][:, None]).abs().sum(0) if ends else 0.0
        if block is not None:
            c0 = c0 + w[:, 128 * block:128 * block + 128] @ v[m][128 * block:128 * block + 128].abs()
        out.append(o), tol.append(2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -10) * a + c0)
    return torch.stack(out), torch.stack(tol)


def _check_rows(c, r, h, keep=None, scale=D ** -0.5, ends=False, block=None):
    row, G = sum(c.q_len[:r]), c.hq // c.hkv
    got = c.out[row:row + c.q_len[r], h * G:(h + 1) * G].double()
    want, tol = _rows_ref(c, r, h, keep, scale, ends, block)
    assert bool(torch.isfinite(got).all())
    err = (got - want).abs() / tol
    assert float(err.max()) <= 1, (r, h, float(err.max()))


def _along(c, score, noise=0.02):
    """Keys and queries along one direction: every score is near `score` nats (a number or one
    a key of request 0 ...)."""
    g = torch.Generator(device="cuda").manual_seed(99)
    u = torch.sign(torch.randn(D, generator=g, device="cuda"))
    c.ks.fill_(120)
    c.q = (u * 0.75 + noise * torch.randn(c.q.shape, generator=g, device="cuda")).to(torch.bfloat16)
    unit = 0.75 * D ** 0.5 * 2.0 ** -7  # nats a unit of the entries
    for r, L in enumerate(c.length):
        page = c.table[r, :(L + 15) // 16].long()
        s = score[r] if isinstance(score, (list, tuple)) else torch.full((L,), float(score), device="cuda")
        s = torch.cat([s, s.new_zeros(16 * len(page) - L)])
        k = (u * (s / unit)[:, None]).clamp(-448, 448).to(E4).view(torch.uint8).view(len(page), 1, 16, D)
        c.kp.view(torch.uint8)[page] = k.expand(-1, c.hkv, -1, -1).contiguous()


@pytest.mark.parametrize("hq,hkv,q_len,length", [(16, 8, [1, 1], [400, 1000]), (32, 4, [3, 16], [300, 700]), (16, 8, [1], [128 * 300 + 40])])
@pytest.mark.parametrize("score", [-8, -20, -28])
def test_a_first_tile_that_is_not_there(lib, hq, hkv, q_len, length, score):
    """All pages of a part's first tile outside the pool (of every other tile, so that this
    holds for many parts of a request that is cut): the rest's softmax, however small the scores."""
    c = Case(hq, hkv, q_len, length, seed=21, spread=0)
    _along(c, score)
    b = c.batch(lib)
    q, cu, ln, table, out = b._keep
    gone, keep = table.clone(), []
    for r, L in enumerate(length):
        m = torch.ones(L, dtype=torch.bool, device="cuda")
        for t in range(0, (L + 127) // 128, 2):
            gone[r, 8 * t:8 * t + 8] = c.n + 5
            m[128 * t:128 * t + 128] = False
        keep.append(m)
    b = lib.AttnBatch8(b.cache, q, cu, ln, gone, out, max(q_len), max(length))
    ws = torch.empty(lib.attn8_workspace_size([b]), dtype=torch.uint8, device="cuda")
    lib.verify_attn8([b], [], D ** -0.5, ws)
    assert lib.device_error() == 1
    for r in range(len(length)):
        for h in (0, hkv - 1):
            _check_rows(c, r, h, keep[r])


@pytest.mark.parametrize("nats", [6, 10, 12, 13, 14, 20, 25])
@pytest.mark.parametrize("hq,hkv,q_len,length,at", [(16, 8, [1], [33000], 0), (32, 4, [2], [40000], 0), (32, 4, [16], [35011], 7000),
                                                    (16, 8, [1, 3], [50000, 40000], 5)])
def test_one_key_far_above_many(lib, hq, hkv, q_len, length, at, nats):
    """A key `nats` above all others whose values are zero: the output is the others' mean.  (The 127
    keys of its own tile, below 2^-8 of all, may be lost beside it.)"""
    c = Case(hq, hkv, q_len, length, seed=22, spread=0)
    g = torch.Generator(device="cuda").manual_seed(nats)
    # (the others between 12 and 13 nats below zero, the one above)
    low = [-12.5 + torch.rand(L, generator=g, device="cuda") for L in length]
    for s in low:
        s[at] = nats - 12.0
    _along(c, low, noise=0.0)
    c.vp = c.vp.float().abs().to(E4)
    for r in range(len(length)):
        c.vp.view(torch.uint8)[c.table[r, at // 16].long(), :, at % 16] = 0
    _run(lib, c)
    for r in range(len(length)):
        _check_rows(c, r, hkv // 2)
    assert lib.device_error() == 0


@pytest.mark.parametrize("far", [8, 14, 18, 24, 40])
@pytest.mark.parametrize("hq,hkv,q_len,length,at", [(16, 8, [1], [33000], 0), (32, 4, [4], [40000], 33), (16, 8, [2, 1], [35000, 50000], 60)])
def test_a_page_of_far_larger_values(lib, hq, hkv, q_len, length, at, far):
    """A page whose V scale is 2^far larger, zero in most dims: keys of other pages still count there
    (but for the 112 of its own tile, below 2^-8 of all)."""
    c = Case(hq, hkv, q_len, length, seed=23, spread=0)
    c.vp = c.vp.float().abs().to(E4)
    for r in range(len(length)):
        page = c.table[r, at].long()
        c.vs[page] = 120 + far
        c.vp.view(torch.uint8)[page, :, :, 5:] = 0
    _run(lib, c)
    for r in range(len(length)):
        _check_rows(c, r, 0)


@pytest.mark.parametrize("hq,hkv,q_len,length", [(16, 8, [1], [20000]), (32, 4, [16], [9000])])
def test_scores_that_swing(lib, hq, hkv, q_len, length):
    """Levels that rise and fall by up to 30 nats from tile to tile, values of the highest ones
    zero: references move in both directions, and the same bytes come out each time."""
    c = Case(hq, hkv, q_len, length, seed=24, spread=0)
    c.vp = c.vp.float().abs().to(E4)
    L = length[0]
    tile = torch.arange(L, device="cuda") // 128
    g = torch.Generator(device="cuda").manual_seed(5)
    level = torch.tensor([0.0, -25.0, -12.0, -28.0, -5.0, -20.0], device="cuda")[tile % 6]
    s = level + torch.rand(L, generator=g, device="cuda")
    _along(c, [s], noise=0.0)
    flat = c.vp.view(torch.uint8)[c.table[0, :(L + 15) // 16].long()].clone()
    high = torch.nn.functional.pad(level > -19, (0, flat.shape[0] * 16 - L)).view(-1, 16)
    flat.permute(0, 2, 1, 3)[high] = 0
    c.vp.view(torch.uint8)[c.table[0, :(L + 15) // 16].long()] = flat
    _run(lib, c)
    for h in (0, hkv - 1):
        _check_rows(c, 0, h, ends=True)
    first = c.out.clone()
    _run(lib, c)
    assert torch.equal(c.out, first)


@pytest.mark.parametrize("scale", [254, 200, 1])
@pytest.mark.parametrize("hq,hkv,q_len,length", [(16, 8, [40], [90]), (32, 4, [30], [300]), (4, 4, [100, 20], [260, 40])])
def test_a_hidden_page_s_scale(lib, hq, hkv, q_len, length, scale):
    """A page of the span whose V scale lies at an end of the range: rows that do not see it
    keep their bits, at scales 2^20 apart among the pages that they see."""
    c = Case(hq, hkv, q_len, length, seed=25, spread=0)
    for r, L in enumerate(length):
        c.vs[c.table[r, 1:(L + 15) // 16:3].long()] = 100
    _run(lib, c)
    first = c.out.clone()
    for r in range(len(length)):
        for h in (0, hkv - 1):
            _check_rows(c, r, h)
    row = 0
    keep = torch.zeros(sum(q_len), dtype=torch.bool, device="cuda")
    for r, (n, L) in enumerate(zip(q_len, length)):
        last = (L - 1) // 16 - 1
        c.vs[c.table[r, last:(L + 15) // 16].long()] = scale
        see = torch.arange(n, device="cuda") + L - n
        keep[row:row + n] = see < 16 * last
        row += n
    assert 0 < int(keep.sum()) < len(keep)
    _run(lib, c)
    assert torch.equal(c.out[keep], first[keep])


@pytest.mark.parametrize("byte", [30, 127, 215])
def test_scales_far_from_one_behind_absent_pages(lib, byte):
    """V scales 2^97 below and 2^88 above 1, the first tiles' pages outside the pool: exponents count
    from those of the first pages that there are."""
    c = Case(16, 8, [1, 2], [300, 1000], seed=26, spread=1)
    c.vs = (c.vs.int() - 120 + byte).to(torch.uint8)
    b = c.batch(lib)
    q, cu, ln, table, out = b._keep
    gone = table.clone()
    gone[:, :16] = c.n + 1
    b = lib.AttnBatch8(b.cache, q, cu, ln, gone, out, 2, 1000)
    ws = torch.empty(lib.attn8_workspace_size([b]), dtype=torch.uint8, device="cuda")
    lib.verify_attn8([b], [], D ** -0.5, ws)
    assert lib.device_error() == 1
    for r, L in enumerate(c.length):
        keep = torch.ones(L, dtype=torch.bool, device="cuda")
        keep[:256] = False
        _check_rows(c, r, 3, keep)


@pytest.mark.parametrize("hq,hkv,q_len,length", [(16, 8, [1], [33000]), (32, 4, [8, 3], [9000, 2000])])
@pytest.mark.parametrize("nats", [35, 44, 70, 110])
def test_one_key_out_of_reach(lib, hq, hkv, q_len, length, nats):
    """A key so far above the others that references reach their floor, 64 binades below their highest
    (44 nats), and past it: the others' part is right as far as it counts, and nothing overflows."""
    c = Case(hq, hkv, q_len, length, seed=27, spread=0)
    low = [torch.full((L,), -nats / 8 - 0.05, device="cuda") for L in length]
    for s in low:
        s[3], s[-200:] = nats / 8, nats / 16
    _along(c, low, noise=0.0)
    c.q.mul_(4.0)  # (scores four times as large: `nats` from the lowest to the highest)
    c.vp = c.vp.float().abs().to(E4)
    _run(lib, c)
    for r in range(len(length)):
        _check_rows(c, r, hkv - 1, ends=True)
    for r in range(len(length)):  # without the keys between, and the highest one's values
        c.kp.view(torch.uint8)[c.table[r, (length[r] - 200) // 16 - 1:(length[r] + 15) // 16].long()] = \
            c.kp.view(torch.uint8)[c.table[r, 5:6].long()]
        c.vp.view(torch.uint8)[c.table[r, 0].long(), :, 3] = 0
    _run(lib, c)
    for r in range(len(length)):
        _check_rows(c, r, hkv - 1, ends=nats > 44, block=0)
