"""Truncated sampling on the GPU (needs a GB300).

The draw is defined in whole numbers, so tokens and kept counts must be equal
to the definition's, evaluated here in numpy row by row (fp32 steps in fp32,
sums in int64).  The definition itself is held against a plain 64-bit softmax:
kept sets and probabilities up to its 2^-30 resolution.

logp tolerance: x carries two fp32 roundings of |x| <= 32 (2^-24 * 2 * 32), log2
of the fp32-rounded mass another 2^-24 and its own 2^-22 of |log2| <= 18, times
ln 2: below 1e-5.
"""
import numpy as np
import pytest
import torch

import oracle as O

pytestmark = pytest.mark.gpu

POW2 = np.array([0x3F800000, 0x3F317213, 0x3E75FCDB, 0x3D635D55, 0x3C1E760B, 0x3AAD4281],
                dtype=np.uint32).view(np.float32)


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd
    ipd.device_error()
    return ipd


def _weights(l, top, inv_t):
    """Whole-number weights of fp32 logits (the definition, step by step)."""
    f4 = np.float32
    with np.errstate(invalid="ignore", over="ignore"):
        c = f4(f4(1.4426950408889634) * f4(inv_t))
        x = np.where(l == top, f4(0), (l - top) * c).astype(f4)
    x = np.maximum(x, f4(-64))
    i = np.rint(x).astype(f4)
    f = (x - i).astype(f4)
    p = np.full_like(f, POW2[5])
    for k in (4, 3, 2, 1, 0):
        p = ((p * f).astype(f4) + POW2[k]).astype(f4)
    y = np.trunc(np.ldexp(p.astype(np.float64), i.astype(np.int64) + 31)).astype(np.int64)
    return (y + 1) >> 1, x


def _draw(l, u, inv_t=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logp, kept) of one fp32 row by the definition."""
    l = np.where(np.isnan(l), np.float32(-np.inf), l.astype(np.float32))
    top = l.max() if l.size else -np.inf
    if top == -np.inf:
        return -1, -np.inf, 0
    w, x = _weights(l, top, inv_t)
    order = np.argsort(-(l + np.float32(0)), kind="stable")
    w, x = w[order], x[order]
    if top_k > 0:
        w[top_k:] = 0
    w[w < np.ceil(np.float64(np.float32(min_p)) * 2.0 ** 30)] = 0
    m = int(w.sum())
    need = max(1, int(min(np.ceil(np.float64(np.float32(top_p)) * np.float64(m)), m)))
    w[np.cumsum(w) - w >= need] = 0
    s = int(w.sum())
    t = min(int(np.floor(np.float64(np.float32(u)) * np.float64(s))), s - 1) if u > 0 else 0
    at = int(np.searchsorted(np.cumsum(w), t, side="right"))
    logp = (float(x[at]) - np.log2(s / 2.0 ** 30)) * np.log(2.0)
    return int(order[at]), logp, int((w > 0).sum())


def _check(lib, logits, u, **settings):
    n, V = logits.shape
    dev = lambda a, t: torch.as_tensor(np.broadcast_to(a, (n,)).copy(), dtype=t).cuda()
    kw = {k: dev(v, torch.int32 if k == "top_k" else torch.float32) for k, v in settings.items()}
    tok = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    logp, kept = torch.full((n,), 9.0, device="cuda"), torch.full((n,), -9, dtype=torch.int32, device="cuda")
    lib.sample_trunc(logits, dev(u, torch.float32), tok, logp=logp, n_kept=kept,
                     inv_temperature=kw.get("inv_t"), top_k=kw.get("top_k"), top_p=kw.get("top_p"),
                     min_p=kw.get("min_p"))
    rows = logits.float().cpu().numpy()
    us = np.broadcast_to(np.float32(u), (n,))
    want = [_draw(rows[i], us[i], **{k: np.broadcast_to(v, (n,))[i] for k, v in settings.items()})
            for i in range(n)]
    assert tok.tolist() == [w[0] for w in want]
    assert kept.tolist() == [w[2] for w in want]
    lw = np.array([w[1] for w in want])
    got = logp.cpu().numpy().astype(np.float64)
    fin = np.isfinite(lw)
    assert (np.abs(got[fin] - lw[fin]) <= 1e-5 + 2.0 ** -22 * np.abs(lw[fin])).all()
    assert (got[~fin] == lw[~fin]).all()
    return tok


def _rows(n, V, seed, sigma=2.5, boost=0):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(n, V, generator=g) * sigma
    if boost:
        l.scatter_add_(1, torch.randint(0, V, (n, boost), generator=g), 8 + 2 * torch.randn(n, boost, generator=g))
    return l.to(torch.bfloat16).cuda()


SETTINGS = [{}, dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05),
            dict(top_k=20, top_p=0.8, min_p=0.01, inv_t=1 / 0.7), dict(top_k=1000, top_p=0.99, inv_t=0.5),
            dict(min_p=1.0), dict(top_p=0.0), dict(inv_t=3.0, min_p=1e-9), dict(inv_t=0.05)]


@pytest.mark.parametrize("n,V", [(1, 1), (2, 2), (3, 7), (9, 8), (5, 33), (40, 1001), (7, 4096),
                                 (3, 50021), (1, 151936), (20, 32000), (2, 262136)])
@pytest.mark.parametrize("settings", SETTINGS, ids=lambda s: "-".join(f"{k}{v:.3g}" for k, v in s.items()) or "plain")
def test_draws(lib, n, V, settings):
    rng = np.random.default_rng(V + n)
    _check(lib, _rows(n, V, V, boost=min(V, 12)), rng.random(n, dtype=np.float32), **settings)
    assert lib.device_error() == 0


@pytest.mark.parametrize("n,V", [(200, 4096), (64, 20011)])
def test_mixed_settings(lib, n, V):
    """Every row its own settings; more rows than one wave's clusters."""
    rng = np.random.default_rng(n)
    pick = lambda *v: rng.choice(np.array(v), n)
    _check(lib, _rows(n, V, n, boost=24), rng.random(n, dtype=np.float32),
           inv_t=pick(1.0, 1.25, 1 / 0.6, 0.8).astype(np.float32), top_k=pick(0, 1, 20, 50, 1000, V, V + 5, -3),
           top_p=pick(1.0, 0.95, 0.5, 0.1).astype(np.float32), min_p=pick(0.0, 0.05, 1e-4).astype(np.float32))


def test_ties(lib):
    """Equal logits: cuts and draws inside a run of ties go by the lower id."""
    n, V = 64, 3000
    g = torch.Generator().manual_seed(2)
    l = torch.randint(0, 3, (n, V), generator=g).float()
    l[:8] = 1.5                                  # one value only
    l[8:16] = torch.where(torch.rand(8, V, generator=g) < 0.5, 0.0, -0.0)  # signed zeros tie
    u = np.linspace(0, 1, n, endpoint=False, dtype=np.float32)
    rows = l.to(torch.bfloat16).cuda()
    for s in (dict(top_k=10), dict(top_k=700), dict(top_p=0.3), dict(top_k=1500, top_p=0.77), {}):
        _check(lib, rows, u, **s)


def test_special_rows(lib):
    """Rows of -inf, NaN, +inf, the type's lowest value, one entry, steep and
    flat ones."""
    V = 5000
    lo = torch.finfo(torch.bfloat16).min
    l = torch.randn(12, V, generator=torch.Generator().manual_seed(3)) * 2
    l[0] = float("-inf")
    l[1] = float("nan")
    l[2] = float("-inf")
    l[2, 4321] = -5.0
    l[3, ::7] = float("nan")
    l[4, [11, 999, 4000]] = float("inf")
    l[5] = lo
    l[6] = lo
    l[6, 17] = 0.0
    l[7] = float("-inf")
    l[7, 100:103] = lo
    l[8] = torch.arange(V).float() * 1e30
    l[9] = torch.linspace(-1e-38, 1e-38, V)      # subnormal differences
    l[10, 0:4990] = float("-inf")
    l[11] *= 1e-3
    rows = l.to(torch.bfloat16).cuda()
    for u in (0.0, 0.3, 0.999999):
        for s in ({}, dict(top_k=5, top_p=0.9), dict(top_k=4900), dict(min_p=0.3, inv_t=2.0)):
            tok = _check(lib, rows, u, **s)
            assert tok[:3].tolist() == [-1, -1, 4321]
    assert lib.device_error() == 0


def test_uniform_ends(lib):
    """u = 0 takes the first entry; the largest u below 1, 1 itself, and values
    outside [0, 1) stay inside the kept set."""
    rows = _rows(6, 2000, 5).contiguous()
    u = np.array([0.0, 1 - 2.0 ** -24, 1.0, 2.5, -1.0, np.nan], dtype=np.float32)
    tok = _check(lib, rows, u, top_k=3)
    top = torch.sort(rows.float().cpu(), dim=-1, descending=True, stable=True).indices
    assert tok[0] == top[0, 0] and tok[4] == top[4, 0] and tok[5] == top[5, 0]
    assert tok[1] == top[1, 2] and tok[2] == top[2, 2] and tok[3] == top[3, 2]


@pytest.mark.parametrize("offset,stride", [(0, 1001), (1, 1003), (5, 1016), (8, 1008), (7, 1000)])
def test_strided_and_unaligned_rows(lib, offset, stride):
    """Rows at any 2-byte alignment; entries beside a row are not read into it."""
    n, V = 9, 1000
    buf = torch.full((offset + n * stride + 8,), 50.0, dtype=torch.bfloat16, device="cuda")
    rows = buf.as_strided((n, V), (stride, 1), offset)
    rows.copy_(_rows(n, V, 6))
    _check(lib, rows, np.linspace(0, 0.99, n).astype(np.float32), top_p=0.9)


def test_bad_settings(lib):
    """A row with a setting that is not valid draws nothing and is recorded;
    its neighbours draw."""
    rows = _rows(8, 500, 7)
    nan, inf = float("nan"), float("inf")
    f = lambda *v: torch.tensor(v, device="cuda")
    tok = torch.full((8,), -9, dtype=torch.int32, device="cuda")
    lib.sample_trunc(rows, torch.rand(8, device="cuda"), tok,
                     inv_temperature=f(1.0, 0.0, -1.0, nan, inf, 1.0, 1.0, 1.0),
                     top_p=f(1.0, 1.0, 1.0, 1.0, 1.0, nan, 1.0, 1.0),
                     min_p=f(0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 1.5, 0.0))
    got = tok.tolist()
    assert got[1:7] == [-1] * 6 and got[0] >= 0 and got[7] >= 0
    assert lib.device_error() == 8
    assert lib.device_error() == 0


def test_distribution(lib):
    """Many draws of one row follow the truncated softmax: each token's share
    within 5 standard deviations, none outside the kept set."""
    n, V = 40000, 64
    row = (torch.randn(V, generator=torch.Generator().manual_seed(8)) * 1.5).to(torch.bfloat16)
    rows = row.cuda().expand(n, V)
    tok = torch.empty(n, dtype=torch.int32, device="cuda")
    full = lambda v, t=torch.float32: torch.full((n,), v, dtype=t, device="cuda")
    lib.sample_trunc(rows, torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda"),
                     tok, inv_temperature=full(1.25), top_k=full(30, torch.int32), top_p=full(0.9))
    p = torch.softmax(row.double() * 1.25, -1)
    v, idx = p.sort(descending=True, stable=True)
    v[30:] = 0
    v = v / v.sum()
    v = torch.where(v.cumsum(0) - v < 0.9, v, 0.0)
    p = torch.zeros_like(p).scatter(0, idx, v / v.sum())
    got = torch.bincount(tok.cpu().long(), minlength=V).double() / n
    assert bool((got[p == 0] == 0).all())
    assert bool(((got - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all())


def test_definition_against_softmax():
    """The whole-number weights are the softmax's ratios to 2^-31 of the largest
    plus the fit's 1.9e-7 relative (no GPU work; beside the tests that use it)."""
    l = np.linspace(-40, 3, 100001).astype(np.float32)
    w, x = _weights(l, l.max(), 1.0)
    # the exponent's own rounding: 2^-23 of |x| in base 2
    true = np.exp((l - l.max()).astype(np.float64))
    assert (np.abs(w / 2.0 ** 30 - true) <= 2.0 ** -31 + (1.9e-7 + 2.0 ** -23 * 64) * true).all()


def test_side_stream_and_repeat(lib):
    rows = _rows(30, 30000, 10, boost=20)
    u = torch.rand(30, device="cuda")
    a, b = (torch.empty(30, dtype=torch.int32, device="cuda") for _ in range(2))
    lib.sample_trunc(rows, u, a)
    side, late = torch.cuda.Stream(), torch.zeros_like(rows)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late.copy_(rows)
    lib.sample_trunc(late, u, b, stream=side)
    side.synchronize()
    assert torch.equal(a, b)
