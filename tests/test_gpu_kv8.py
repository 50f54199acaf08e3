"""Append to the 8-bit cache on the GPU: every byte of the pools against the
definition in 64 bits (needs a GB300)."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref

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


class Case:
    """A cache with random contents, a page table, and new rows of random sizes."""

    def __init__(self, hkv, old, new, seed=0, spread=3, spare=3):
        g = np.random.default_rng(seed)
        self.length = [a + b for a, b in zip(old, new)]
        pages = [(x + 15) // 16 for x in self.length]
        n = sum(pages) + spare
        perm, at = g.permutation(n), 0
        self.table = np.full((len(new), max(1, max(pages))), -1, dtype=np.int32)
        for r, x in enumerate(pages):
            self.table[r, :x] = perm[at:at + x]
            at += x
        raw = lambda: np.where(g.random((n, hkv, 16, 128)) < 0.5, 0, 0x80).astype(np.uint8) | \
            g.integers(0, 127, (n, hkv, 16, 128), dtype=np.uint8)
        self.pages = {t: raw() for t in "kv"}
        self.scale = {t: g.integers(113, 122, (n, hkv), dtype=np.uint8) for t in "kv"}
        total = sum(new)
        size = 2.0 ** g.integers(-spread, spread + 1, (total, hkv, 1)) if total else 1.0
        self.x = {t: torch.tensor(g.standard_normal((total, hkv, 128)) * size, dtype=torch.bfloat16) for t in "kv"}
        self.new, self.hkv, self.n = new, hkv, n

    def want(self):
        """(pages, scales) after the append."""
        out = {}
        for t in "kv":
            pages, scale, row = self.pages[t].copy(), self.scale[t].copy(), 0
            x = self.x[t].float().numpy()
            for r, n in enumerate(self.new):
                pos = self.length[r] - n
                while pos < self.length[r]:
                    m = min(16 - pos % 16, self.length[r] - pos)
                    page = self.table[r, pos // 16]
                    ref.append(pages[page], scale[page], x[row:row + m], list(range(pos % 16, pos % 16 + m)))
                    row, pos = row + m, pos + m
            out[t] = (pages, scale)
        return out

    def args(self, lib, wide=0):
        """A device cache and kv8_append's other arguments; wide: k and v as views
        into rows with that many heads more."""
        dev = lambda a: torch.from_numpy(a.copy()).cuda()
        page = lambda t: dev(self.pages[t]).view(torch.float8_e4m3fn)
        cache = lib.KVCache8(page("k"), page("v"), dev(self.scale["k"]), dev(self.scale["v"]))
        cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        x = []
        for t in "kv":
            full = torch.full((sum(self.new), self.hkv + wide, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
            full[:, wide // 2:wide // 2 + self.hkv] = self.x[t].cuda()
            x.append(full[:, wide // 2:wide // 2 + self.hkv])
        return cache, x[0], x[1], dev(cu), dev(np.array(self.length, dtype=np.int32)), dev(self.table)


def _check(cache, want):
    for t in "kv":
        pages, scale = want[t]
        assert np.array_equal(getattr(cache, t + "_scale").cpu().numpy(), scale), t
        assert ref.same_bytes(getattr(cache, t + "_pages").view(torch.uint8).cpu().numpy(), pages), t


@pytest.mark.parametrize("hkv,old,new", [
    (8, [16, 15, 0, 255, 31], [1, 1, 1, 1, 1]),              # decode steps: a page's first row and its last
    (4, [0, 7, 8, 100, 200, 3], [16, 16, 9, 1, 13, 0]),      # spans, page crossings, an empty request
    (1, [0], [1]), (64, [5, 0], [12, 33]), (3, [0, 1, 15], [17, 31, 2]),
    (4, [0, 0, 40], [700, 1333, 250]), (2, [0] * 9, [300] * 9)])  # prompts: warps with groups of rows
def test_append_is_the_definition(lib, hkv, old, new):
    c = Case(hkv, old, new, seed=hkv + len(new))
    a = c.args(lib)
    lib.kv8_append(*a)
    _check(a[0], c.want())
    assert lib.device_error() == 0


def test_strided_rows(lib):
    c = Case(4, [5, 0, 30], [16, 40, 3], seed=5)
    a = c.args(lib, wide=6)
    lib.kv8_append(*a)
    _check(a[0], c.want())


@pytest.mark.parametrize("old,new", [([3, 0], [9, 20]), ([0, 14], [1, 1])])
def test_rows_out_of_the_usual_range(lib, old, new):
    """Zeros, subnormals, the largest bf16, infinities and NaN in rows, and held
    NaN; pages whose scale grows by up to 250 binades."""
    c = Case(2, old, new, seed=9)
    bits = torch.tensor([0x0000, 0x8000, 0x0001, 0x8001, 0x7f7f, 0xff7f, 0x7f80, 0xff80, 0x7fc0, 0x0080, 0x3f80, 0x43e0,
                         0x43e1, 0x2b80], dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    g = torch.Generator().manual_seed(1)
    for t in "kv":
        for h in range(2):
            rows = c.x[t].shape[0]
            pick = bits[torch.randint(0, len(bits), (rows, 128), generator=g)]
            some = torch.rand(rows, 1, generator=g) < (0.3 if h else 1.1)
            c.x[t][:, h] = torch.where(some, pick, c.x[t][:, h])
        c.x[t][0] = 0.0  # (a page may begin with zeros alone)
        c.pages[t][:, :, 1, 5] = 0x7f
        c.scale[t][:, 1] = 1
    a = c.args(lib)
    lib.kv8_append(*a)
    _check(a[0], c.want())


def test_scale_bytes_at_the_ends(lib):
    """A page that goes on with the largest byte, with NaN (255) and with one below
    the least."""
    c = Case(3, [4, 4, 4], [3, 3, 3], seed=2)
    for t in "kv":
        for r, b in enumerate((254, 255, 0)):
            c.scale[t][c.table[r, 0]] = b
    a = c.args(lib)
    lib.kv8_append(*a)
    _check(a[0], c.want())


def test_one_by_one_and_after_a_rollback(lib):
    """Forty tokens one at a time (every page's scale grows on its way), then a
    rollback by eleven and other rows over them."""
    c = Case(2, [0], [40], seed=3)
    cache, k, v, cu, length, table = c.args(lib)
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    pages = {t: (c.pages[t].copy(), c.scale[t].copy()) for t in "kv"}

    def put(pos, j):
        lib.kv8_append(cache, k[j:j + 1], v[j:j + 1], one, torch.tensor([pos + 1], dtype=torch.int32, device="cuda"), table)
        for t in "kv":
            page = c.table[0, pos // 16]
            ref.append(pages[t][0][page], pages[t][1][page], c.x[t][j:j + 1].float().numpy(), [pos % 16])

    for j in range(40):
        put(j, j)
    for j in range(29, 40):
        put(j, 39 - j)
    _check(cache, pages)


def test_many_in_one_launch(lib):
    cases = [Case(4, [9, 0], [16, 50], seed=6), Case(8, [3, 4, 5], [1, 1, 1], seed=7), Case(1, [0], [0], seed=8),
             Case(2, [16], [2000], seed=9)]
    args = [c.args(lib) for c in cases]
    lib.kv8_append_many(args)
    for c, a in zip(cases, args):
        _check(a[0], c.want())
    assert lib.device_error() == 0


def test_captured_and_replayed_on_another_stream(lib):
    c = Case(4, [9, 30], [7, 20], seed=11)
    a = c.args(lib)
    lib.kv8_append(*c.args(lib))  # (a first call outside the capture)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        lib.kv8_append(*a)
    graph.replay()
    torch.cuda.synchronize()
    _check(a[0], c.want())
    c2 = Case(4, [9, 30], [7, 20], seed=12)  # other rows and contents in the same buffers
    b = c2.args(lib)
    for x, y in ((a[0].k_pages, b[0].k_pages), (a[0].v_pages, b[0].v_pages), (a[0].k_scale, b[0].k_scale),
                 (a[0].v_scale, b[0].v_scale), (a[1], b[1]), (a[2], b[2]), (a[5], b[5])):
        x.copy_(y)
    graph.replay()
    torch.cuda.synchronize()
    _check(a[0], c2.want())


def test_faulty_rows_are_recorded_and_skipped(lib):
    """A page outside the pool, a position past the table, rows no offsets cover,
    offsets out of order: the other rows are appended, no scale counts the others'."""
    c = Case(4, [3, 20, 0], [5, 4, 2], seed=13)
    good = c.want()
    for what, code in (("page", 1), ("length", 2), ("offsets", 6), ("order", 6)):
        a = list(c.args(lib))
        want = {t: (good[t][0].copy(), good[t][1].copy()) for t in "kv"}
        page = c.table[1, 1]
        if what == "page":
            a[5][1, 1] = c.n + 5
        elif what == "length":
            a[4][1] = 16 * c.table.shape[1] + 4
        elif what == "offsets":
            a[3][3] = 9  # the last request's rows are not covered
            page = c.table[2, 0]
            a[4][2] = 0
        else:
            a[3][:] = torch.tensor([0, 5, 9, 7], dtype=torch.int32)  # rows past the last offset: none's
            page = c.table[2, 0]
        for t in "kv":
            want[t][0][page], want[t][1][page] = c.pages[t][page], c.scale[t][page]
        lib.kv8_append(*a)
        assert lib.device_error() == code, what
        if what == "order":  # offsets 0 5 9 7: rows 7 and 8 lie past the last, row 5 and 6 are request 1's
            continue
        _check(a[0], want)


def test_pools_past_32_bits(lib):
    """A pool of more than 2^32 bytes a tensor: a page at its very end."""
    n, hkv = (1 << 18) + 5, 8
    cache = lib.KVCache8.empty(n, hkv)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    x = torch.randn(3, hkv, 128, device="cuda").to(torch.bfloat16)
    lib.kv8_append(cache, x, -x, i32(0, 3), i32(3), i32(n - 1).view(1, 1))
    pages, scale = np.zeros((hkv, 16, 128), dtype=np.uint8), np.full(hkv, 127, dtype=np.uint8)
    ref.append(pages, scale, x.float().cpu().numpy(), [0, 1, 2])
    assert np.array_equal(cache.k_pages[n - 1].view(torch.uint8).cpu().numpy(), pages)
    assert np.array_equal(cache.k_scale[n - 1].cpu().numpy(), scale)
    assert int(cache.k_pages[:n - 1].view(torch.uint8).max()) == 0 and int(cache.k_scale[:n - 1].min()) == 127
