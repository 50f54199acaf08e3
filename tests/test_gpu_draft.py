"""Verification of drafted tokens on the GPU (needs a GB300): verdicts and tokens
equal to the definition's in whole numbers; log-probabilities ln 2 (x - log2 Z),
in fp32, to 2^-21 of themselves plus 2^-21: Z is off by 2^-24 of itself, its log2 by
2^-23 of a number no larger than the difference (x <= 0), the difference, the factor
and the product by 2^-24 each, x by one rounding that the definition has too:
2^-22.4 of the result and 2^-24 in all."""
import numpy as np
import pytest
import torch

from tests import draft_ref as ref

pytestmark = pytest.mark.gpu
NINF = float("-inf")


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
    def __init__(self, k, V, seed=0, noise=0.8, bonus=True, temps=True, sigma=2.0):
        g = torch.Generator().manual_seed(seed)
        T, R = sum(k), len(k)
        self.k, self.V = k, V
        base = torch.randn(T, V, generator=g) * sigma
        base.scatter_add_(1, torch.randint(0, V, (T, min(V, 8)), generator=g), torch.full((T, min(V, 8)), 6.0))
        self.target = base.to(torch.bfloat16)
        self.draft = (base + noise * torch.randn(T, V, generator=g)).to(torch.bfloat16)
        self.bonus = (torch.randn(R, V, generator=g) * sigma).to(torch.bfloat16) if bonus else None
        pick = lambda: torch.tensor([1.0, 1 / 0.7, 1 / 1.3])[torch.randint(0, 3, (R,), generator=g)] if temps else torch.ones(R)
        self.inv_p, self.inv_q = pick(), pick()
        per = torch.repeat_interleave(self.inv_q, torch.tensor(k, dtype=torch.int64))[:, None]
        self.tokens = torch.multinomial(torch.softmax(self.draft.float() * per, -1), 1, generator=g).squeeze(1).int() \
            if T else torch.zeros(0, dtype=torch.int32)
        self.u, self.u_next = torch.rand(T, generator=g), torch.rand(R, generator=g)
        self.temps = temps
        self.cu = torch.tensor([0] + k).cumsum(0).int()

    def run(self, lib, place=lambda t: t.cuda(), logp=True, stream=None):
        R, T = len(self.k), sum(self.k)
        dev = lambda t: None if t is None else t.cuda()
        self.n, self.nxt = (torch.full((R,), 77, dtype=torch.int32, device="cuda") for _ in "ab")
        self.lp, self.lq = (torch.full((T,), 77.0, device="cuda") for _ in "ab")
        ws = torch.full((max(256, lib.verify_draft_workspace_size(R, T, self.V)),), 0xff, dtype=torch.uint8, device="cuda")
        lib.verify_draft(place(self.target), place(self.draft), dev(self.tokens), dev(self.cu), dev(self.u), dev(self.u_next),
                         self.n, self.nxt, ws, logits_bonus=None if self.bonus is None else place(self.bonus),
                         inv_temp_target=dev(self.inv_p) if self.temps else None,
                         inv_temp_draft=dev(self.inv_q) if self.temps else None,
                         logp_target=self.lp if logp else None, logp_draft=self.lq if logp else None)
        return self

    def want(self):
        f = lambda t: None if t is None else t.float().numpy()
        return ref.verify(f(self.target), f(self.draft), f(self.bonus), self.tokens.tolist(), self.cu.tolist(),
                          self.u.tolist(), self.u_next.tolist(), self.inv_p.numpy(), self.inv_q.numpy())

    def check(self):
        verdict, logp = self.want()
        assert list(zip(self.n.tolist(), self.nxt.tolist())) == verdict
        got = torch.stack([self.lp, self.lq], 1).double().cpu().numpy()
        logp = np.array(logp, dtype=np.float64).reshape(-1, 2)
        assert np.array_equal(np.isfinite(got), np.isfinite(logp)) and np.array_equal(np.isnan(got), np.isnan(logp))
        ok = np.isfinite(logp)
        assert np.all(np.abs(got[ok] - logp[ok]) <= 2.0 ** -21 * np.abs(logp[ok]) + 2.0 ** -21)
        return verdict


@pytest.mark.parametrize("k,V", [([4], 1000), ([1], 8), ([0, 3, 1], 1001), ([2, 5, 0, 7], 4096), ([3], 50021), ([1, 1], 1),
                                 ([2], 7), ([16, 9], 2049), ([1], 151936), ([2, 2], 151933)])
@pytest.mark.parametrize("bonus", [True, False])
def test_verdicts_are_the_definition(lib, k, V, bonus):
    c = Case(k, V, seed=V + len(k), bonus=bonus).run(lib)
    c.check()
    assert lib.device_error() == 0


def test_many_requests_of_both_kinds(lib):
    """600 requests: both outcomes, every split of a row over CTAs."""
    g = torch.Generator().manual_seed(3)
    c = Case(torch.randint(0, 5, (600,), generator=g).tolist(), 515, seed=4, noise=1.0).run(lib)
    verdict = c.check()
    share = sum(n for n, _ in verdict) / sum(c.k)
    assert 0.2 < share < 0.95


@pytest.mark.parametrize("R,V", [(1500, 2), (160, 300), (200, 9001)])
def test_verdicts_at_their_border(lib, R, V):
    """For every request the largest uniform number that accepts its draft, and the next one,
    which rejects it: a weight (below 2^24 for most) that is off by one would move the border."""
    c = Case([1] * R, V, seed=R, noise=0.6, bonus=False)
    g = torch.Generator().manual_seed(V)
    if V == 2:
        c.target, c.draft = torch.zeros(R, 2, dtype=torch.bfloat16), torch.zeros(R, 2, dtype=torch.bfloat16)
        c.target[:, 1] = (-3 - 12 * torch.rand(R, generator=g)).to(torch.bfloat16)
        c.draft[:, 1] = (c.target[:, 1].float() + 0.7 * torch.rand(R, generator=g)).to(torch.bfloat16)
        c.tokens[:] = 1
    f = lambda t: t.float().numpy()
    below, above, used = [], [], []
    for r in range(R):
        (_, wp), (_, wq) = ref.weights(f(c.target[r]), c.inv_p[r].numpy()), ref.weights(f(c.draft[r]), c.inv_q[r].numpy())
        tok, zp, zq = int(c.tokens[r]), int(wp.sum()), int(wq.sum())
        ok = lambda u: float(u) * float(wq[tok]) * float(zp) < float(wp[tok]) * float(zq)
        u = np.float32(min(1.0, float(wp[tok]) * zq / max(1.0, float(wq[tok]) * zp)))
        up, down = np.float32(2), np.float32(0)
        for _ in range(4):
            u = np.nextafter(u, up)
        while u > 0 and not ok(u):
            u = np.nextafter(u, down)
        if 0 < u < 1 - 2.0 ** -20:
            below.append(float(u)), above.append(float(np.nextafter(u, up))), used.append(r)
    assert len(used) > R // 8
    for us, want in ((below, 1), (above, 0)):
        c.u[:] = 0.0
        c.u[used] = torch.tensor(us)
        c.run(lib)
        assert c.n[used].tolist() == [want] * len(used), (want, int((c.n[used] != want).sum()), len(used))


def test_equal_models_accept_everything(lib):
    c = Case([5, 3], 3001, seed=5, noise=0.0, temps=False)
    c.u[:] = torch.nextafter(torch.tensor(1.0), torch.tensor(0.0))
    assert [n for n, _ in c.run(lib).check()] == [5, 3]


def test_the_distribution_is_the_target_s(lib):
    """Small vocabulary, many independent requests of one draft each: the emitted
    first token (the draft, or the residual's) follows the target's softmax.  Chi
    square of 40,000 draws over 12 entries: below 40 but for one run in 30,000."""
    g = torch.Generator().manual_seed(6)
    R, V = 40000, 12
    p, q = torch.randn(V, generator=g) * 1.5, torch.randn(V, generator=g) * 1.5
    c = Case([1] * R, V, seed=7, bonus=False, temps=False)
    c.target, c.draft = (t.to(torch.bfloat16).expand(R, V).contiguous() for t in (p, q))
    c.tokens = torch.multinomial(torch.softmax(c.draft[0].float(), -1), R, replacement=True, generator=g).int()
    c.run(lib)
    first = torch.where(c.n == 1, c.tokens.cuda(), c.nxt)
    seen = torch.bincount(first.long(), minlength=V).double().cpu()
    want = torch.softmax(c.target[0].double(), -1) * R
    assert float(((seen - want) ** 2 / want).sum()) < 40


def test_uniform_numbers_at_the_ends(lib):
    c = Case([3, 3, 3, 3], 999, seed=8)
    c.u[:3], c.u[3:6], c.u[6:9] = 0.0, float("nan"), 0.99999994
    c.u_next[:] = torch.tensor([0.0, 0.99999994, float("nan"), 1.5])
    c.run(lib).check()


def test_unusual_rows(lib):
    """Rows with nothing left, with NaN, with +inf, masks of the type's lowest value,
    a draft token the draft model gives nothing, a token the target gives nothing."""
    c = Case([2, 2, 2, 2, 2, 2, 2, 2], 300, seed=9)
    low = torch.finfo(torch.bfloat16).min
    c.target[0] = NINF                                     # the target's row has no entry
    c.draft[2] = NINF                                      # the draft's row has none
    c.target[4, ::2], c.draft[4, 1::2] = float("nan"), float("nan")
    c.target[6, 17] = c.draft[6, 18] = float("inf")
    c.target[8, 5:], c.draft[8, 7:] = low, low
    c.draft[10, c.tokens[10]] = NINF
    c.target[12, c.tokens[12]] = NINF
    c.target[14:], c.draft[14:] = low, low
    c.target[13, :], c.draft[13, :] = -0.0, 0.0
    c.run(lib).check()
    c.bonus[:] = NINF
    c.u[:] = 0.0
    c.run(lib).check()


@pytest.mark.parametrize("R,V", [(90, 9001), (45, 60001), (90, 8193), (160, 8190)])
def test_long_rows_of_any_values(lib, R, V):
    """Rows that are read once, by a histogram of their values (whole ones, and pieces of split
    ones), and those that cannot be: values of both kinds of zero and near it (few, as many as a
    list holds, more), at both ends of what has a bin, masks, NaN, infinities, a temperature at
    which nothing is small."""
    c = Case([2] * R, V, seed=V)
    t, d = c.target, c.draft
    low, tiny = torch.finfo(torch.bfloat16).min, torch.finfo(torch.bfloat16).tiny
    cut = torch.tensor(2.0 ** -19).to(torch.bfloat16)
    t[0, ::3], t[0, 1::3], d[0, ::2] = 0.0, -0.0, -0.0
    t[2, :200], d[2, 40:90] = tiny, -tiny
    t[4, :256], d[4, :256] = cut / 2, -cut / 2            # a full list
    t[6, :257], d[6, 5000:5257] = cut / 2, cut / 4        # one more
    t[8, :], d[8, :] = tiny, 0.0
    t[10, ::5], d[10, 1::5] = cut, -cut                   # the smallest value with a bin
    t[12, 100], d[12, 101] = 4096.0, 4064.0               # the first without, the last with
    t[14, 100], d[14, 101] = -4096.0, -4064.0
    t[16, ::2], d[16, 1::2] = low, NINF
    t[18, ::2], d[18, ::7] = float("nan"), float("nan")
    t[20, V - 1] = d[20, 0] = float("inf")
    t[22, :], d[24, :] = NINF, NINF
    t[26, 1:], d[26, 1:] = low, low
    t[28, :], d[28, :] = -3000.0, -5000.0
    t[30, :], d[30, :] = 5000.0, 3000.0
    t[32, 3:], d[32, 3:] = NINF, NINF
    t[34, :], d[34, :] = 1.0, 1.0
    c.inv_p[18], c.inv_q[18] = 0.004, 0.004               # requests 18 to 20: -4096 has a weight
    c.inv_p[19], c.inv_q[20] = 0.01, 0.02
    t[38, ::2], d[40, ::2] = -4090.0, -9000.0
    c.inv_p[21], c.inv_q[21] = 50.0, 0.7
    c.run(lib).check()
    first = c.nxt.clone(), c.n.clone(), c.lp.clone()
    for x, y in zip(first, (lambda r: (r.nxt, r.n, r.lp))(c.run(lib))):
        assert torch.equal(x.nan_to_num(), y.nan_to_num())
    assert lib.device_error() == 0


def test_bad_tokens_settings_and_offsets(lib):
    c = Case([2, 3, 1, 2], 500, seed=10)
    c.tokens[0], c.tokens[3] = 500, -1
    c.run(lib).check()
    assert lib.device_error() == 3
    c = Case([2, 3, 1, 2], 500, seed=11)
    want, _ = c.want()
    for bad in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        c.inv_q[1] = bad
        c.run(lib)
        assert lib.device_error() == 8
        assert (int(c.n[1]), int(c.nxt[1])) == (0, -1) and bool(torch.isnan(c.lp[2:5]).all())
        assert [(int(c.n[r]), int(c.nxt[r])) for r in (0, 2, 3)] == [want[r] for r in (0, 2, 3)]
        assert lib.device_error() == 0
    c = Case([2, 3, 1, 2], 500, seed=11)
    for cu in ([0, 2, 5, 6, 9], [0, 2, 5, -1, 8], [-3, 2, 5, 6, 8]):
        c.cu = torch.tensor(cu).int()
        c.run(lib)
        assert lib.device_error() == 6, cu
        for r in range(4):
            if not (0 <= cu[r] <= cu[r + 1] <= 8):
                assert (int(c.n[r]), int(c.nxt[r])) == (0, -1)
            elif (cu[r], cu[r + 1]) == (int(Case([2, 3, 1, 2], 500, seed=11).cu[r]), int(Case([2, 3, 1, 2], 500, seed=11).cu[r + 1])):
                assert (int(c.n[r]), int(c.nxt[r])) == want[r], (cu, r)
    # positions that no offsets cover stay as they are
    c = Case([2, 3], 100, seed=12)
    c.cu = torch.tensor([1, 2, 4]).int()
    c.run(lib)
    assert float(c.lp[0]) == 77.0 and float(c.lq[4]) == 77.0 and float(c.lp[1]) != 77.0


@pytest.mark.parametrize("shift,extra", [(1, 0), (3, 5), (8, 3), (0, 1)])
def test_rows_of_any_alignment(lib, shift, extra):
    """Rows that begin inside a 16-byte vector, target and draft differently, beside
    entries that would change every sum."""
    c = Case([2, 3], 701, seed=13)

    def place(t):
        s = shift if t is c.target else 2 * shift + 1 if t is c.draft else 0
        wide = torch.full((t.shape[0], s + 701 + extra), 99.0, dtype=torch.bfloat16, device="cuda")
        wide[:, s:s + 701] = t.cuda()
        return wide[:, s:s + 701]

    c.run(lib, place).check()


def test_without_log_probabilities_and_captured(lib):
    c = Case([2, 4, 0], 2000, seed=14)
    c.run(lib, logp=False)
    want, _ = c.want()
    assert list(zip(c.n.tolist(), c.nxt.tolist())) == want
    args = [t.cuda() for t in (c.target, c.draft, c.tokens, c.cu, c.u, c.u_next)]
    n, nxt = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in "ab")
    ws = torch.empty(lib.verify_draft_workspace_size(3, 6, 2000), dtype=torch.uint8, device="cuda")
    bonus, ip, iq = c.bonus.cuda(), c.inv_p.cuda(), c.inv_q.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.verify_draft(*args, n, nxt, ws, logits_bonus=bonus, inv_temp_target=ip, inv_temp_draft=iq)
    for seed in (14, 15, 16):
        c = Case([2, 4, 0], 2000, seed=seed)
        for a, b in zip(args + [bonus, ip, iq], (c.target, c.draft, c.tokens, c.cu, c.u, c.u_next, c.bonus, c.inv_p, c.inv_q)):
            a.copy_(b)
        ws.fill_(0xff)
        graph.replay()
        assert list(zip(n.tolist(), nxt.tolist())) == c.want()[0]


def test_no_requests_and_no_drafts(lib):
    c = Case([0, 0], 123, seed=17).run(lib)
    c.check()
    Case([0, 0], 123, seed=18, bonus=False).run(lib).check()


@pytest.mark.parametrize("V", [700, 30011])
@pytest.mark.parametrize("cu", [[0, 2, 5, 8, 6], [4, 2, 5], [3, 8, 1, 3, 3], [6, 0, 1, 4, 2, 2], [0, 5, 3], [8, 8, 8, 2, 8]])
def test_offsets_out_of_order_leave_the_others(lib, V, cu):
    """Requests whose own offsets are in order get the results that each would get alone,
    wherever the offsets around them lie; 8 positions, and a workspace of old contents."""
    R = len(cu) - 1
    whole = Case([1] * 8, V, seed=19, bonus=False)
    for seed in range(4):
        c = Case([0] * R, V, seed=20 + seed)
        for x in ("target", "draft", "tokens", "u"):
            setattr(c, x, getattr(whole, x))
        c.u, c.cu, c.k = torch.rand(8, generator=torch.Generator().manual_seed(seed)), torch.tensor(cu).int(), [0] * (R - 1) + [8]
        c.run(lib)
        assert lib.device_error() == 6
        f = lambda t: t.float().numpy()
        for r in range(R):
            a, b = cu[r], cu[r + 1]
            if a > b:
                assert (int(c.n[r]), int(c.nxt[r])) == (0, -1)
                continue
            verdict, logp = ref.verify(f(c.target[a:b]), f(c.draft[a:b]), f(c.bonus[r:r + 1]), c.tokens[a:b].tolist(), [0, b - a],
                                       c.u[a:b].tolist(), [float(c.u_next[r])], c.inv_p[r:r + 1].numpy(), c.inv_q[r:r + 1].numpy())
            assert (int(c.n[r]), int(c.nxt[r])) == verdict[0], (cu, r, seed)
            got = torch.stack([c.lp, c.lq], 1)[a:b].double().cpu().numpy()
            logp = np.array(logp, dtype=np.float64).reshape(-1, 2)
            assert np.all(np.abs(got - logp) <= 2.0 ** -21 * np.abs(logp) + 2.0 ** -21)


@pytest.mark.parametrize("cu", [[0, 5, 3, 8], [2, 7, 1, 4, 8], [0, 8, 0, 8], [6, 0, 1, 4, 2, 6]])
def test_requests_that_share_positions(lib, cu):
    """Two requests of different temperatures with positions in common: each gets its own
    result or the one of a request whose offsets are at fault, not a mixture."""
    R, V, refused = len(cu) - 1, 900, 0
    for seed in range(12):
        whole = Case([1] * 8, V, seed=30 + seed, bonus=False, noise=1.5)
        c = Case([0] * R, V, seed=30 + seed)
        for x in ("target", "draft", "tokens", "u"):
            setattr(c, x, getattr(whole, x))
        c.inv_p, c.inv_q = torch.linspace(0.3, 2.5, R), torch.linspace(2.0, 0.4, R)
        c.cu, c.k = torch.tensor(cu).int(), [0] * (R - 1) + [8]
        c.run(lib)
        assert lib.device_error() == 6
        f = lambda t: t.float().numpy()
        for r in range(R):
            a, b = cu[r], cu[r + 1]
            got = (int(c.n[r]), int(c.nxt[r]))
            refused += a <= b and got == (0, -1)
            if a <= b and got != (0, -1):
                verdict, _ = ref.verify(f(c.target[a:b]), f(c.draft[a:b]), f(c.bonus[r:r + 1]), c.tokens[a:b].tolist(), [0, b - a],
                                        c.u[a:b].tolist(), [float(c.u_next[r])], c.inv_p[r:r + 1].numpy(), c.inv_q[r:r + 1].numpy())
                assert got == verdict[0], (cu, r, seed)
    assert refused >= 12
