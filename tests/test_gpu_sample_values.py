"""Draws of ipd_sample_trunc from rows whose values leave the usual range: near
0, beyond 2^16, infinite, all alike, at lengths that one CTA and several work on."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample_trunc import _check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2609_36546_gb300 import ipd
    return ipd


def _rows(V):
    g = torch.Generator().manual_seed(V)
    rn = lambda: torch.randn(V, generator=g)  # noqa: E731
    few = lambda n: torch.randperm(V, generator=g)[:n]  # noqa: E731
    rows = []
    rows.append(rn() * 1e-5)                      # most of it nearer to 0 than 2^-15
    rows.append(rn() * 0.02)                      # some of it
    r = torch.full((V,), -5.0)                    # zeros of both signs and tiny values above the rest
    r[few(200)] = 0.0
    r[few(100)] = -0.0
    r[few(20)] = 1e-20
    r[few(20)] = -1e-20
    r[few(9)] = 2.0 ** -16
    rows.append(r)
    rows.append(torch.zeros(V))
    rows.append(torch.full((V,), 2.5))
    rows.append(rn() * 2e4)                       # a maximum beyond 2^16
    r = rn()
    r[few(7)] = float("inf")
    rows.append(r)
    rows.append(-1e5 + 3e3 * rn())                # all below -2^16
    r = torch.full((V,), float("-inf"))           # the edge of the range, from both sides
    r[few(30)] = -65536.0
    r[few(30)] = -65280.0
    r[few(3)] = -65024.0
    rows.append(r)
    r = rn()
    r[V // 3:] = torch.finfo(torch.bfloat16).min  # forbidden
    r[few(V // 10)] = float("nan")
    rows.append(r)
    r = torch.full((V,), float("-inf"))           # one entry, at the end
    r[V - 1] = -3.0
    rows.append(r)
    rows.append(torch.full((V,), float("-inf")))
    return torch.stack(rows).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("V", [5003, 60001, 151936])
@pytest.mark.parametrize("settings", [{}, dict(top_k=7), dict(top_k=250, top_p=0.8), dict(top_p=0.5),
                                      dict(min_p=0.4, top_p=0.999), dict(inv_t=1e-4, top_p=0.7)],
                         ids=lambda s: "-".join(f"{k}{v:.3g}" for k, v in s.items()) or "plain")
def test_values(lib, V, settings):
    rows = _rows(V)
    for u in (0.0, 0.41, 0.9999):
        _check(lib, rows, u, **settings)
    # each row by itself: several CTAs where the row is long
    for i in (0, 2, 5, 6, 8):
        _check(lib, rows[i:i + 1], 0.73, **settings)


@pytest.mark.parametrize("start", range(8))
def test_rows_that_start_anywhere(lib, start):
    V = 50003
    g = torch.Generator().manual_seed(3)
    buf = (torch.randn(3, V + 24, generator=g) * 2).to(torch.bfloat16).cuda()
    buf[:, start + V:] = 30.0   # what lies around a row is not the row's
    buf[:, :start] = 30.0
    rows = buf[:, start:start + V]
    for s in ({}, dict(top_k=40), dict(top_p=0.9)):
        _check(lib, rows, np.float32([0.2, 0.6, 0.95]), **s)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("e", [12, 16, -15, -19, -24])
def test_neighbours_of_powers_of_two(lib, sign, e):
    # the bf16 values on both sides of a power of two, some of each, among -inf
    V = 5003
    g = torch.Generator().manual_seed(100 + e)
    row = torch.full((2, V), float("-inf"))
    row[1] = -300.0 if sign > 0 else -1e6
    for m in (1 - 2.0 ** -7, 1 - 2.0 ** -8, 1.0, 1 + 2.0 ** -7, 1 + 2.0 ** -6):
        row[:, torch.randperm(V, generator=g)[:20]] = sign * m * 2.0 ** e
    rows = row.to(torch.bfloat16).cuda()
    for u in (0.1, 0.5, 0.97):
        for s in ({}, dict(top_k=33), dict(top_p=0.6)):
            _check(lib, rows, u, inv_t=min(1.0, 2.0 ** (5 - e)), **s)


@pytest.mark.parametrize("V", [7, 1003, 50021])
def test_many_rows(lib, V):
    # more rows than two for each SM
    g = torch.Generator().manual_seed(V)
    n = 331
    rows = (torch.randn(n, V, generator=g) * 2).to(torch.bfloat16).cuda()
    rows[17] = float("-inf")
    rows[29] = 0.0
    rows[31] *= 1e4
    rng = np.random.default_rng(V)
    k = rng.integers(0, 60, n).astype(np.int32)
    p = rng.choice([1.0, 0.9, 0.4], n).astype(np.float32)
    _check(lib, rows, rng.random(n, dtype=np.float32), top_k=k, top_p=p)
