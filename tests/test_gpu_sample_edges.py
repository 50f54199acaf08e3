"""Draws of ipd_sample_trunc at the edges of its histogram (needs a GB300): values
around +-2^12 and 2^-19, between which a value has a bin of its own, and 0 to 257
entries nearer to 0 than 2^-19, of which it lists 256 (zeros count as one)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample_trunc import _check

pytestmark = pytest.mark.gpu

SETTINGS = [{}, dict(top_k=9), dict(top_k=300, top_p=0.7), dict(top_p=0.4), dict(min_p=0.2)]
ids = lambda s: "-".join(f"{k}{v:.3g}" for k, v in s.items()) or "plain"  # noqa: E731
NEAR = 0x3600  # bf16 bits of 2^-19


@pytest.fixture(scope="module")
def lib():
    from paper_2609_36546_gb300 import ipd
    return ipd


def _bits(values):
    """bf16 values from their bit patterns."""
    return torch.as_tensor(np.asarray(values, dtype=np.uint16).view(np.int16)).view(torch.bfloat16)


def _scatter(V, parts, rest, seed):
    """A row of `rest` with each part's values at places of their own."""
    g = torch.Generator().manual_seed(seed)
    row = torch.full((V,), rest, dtype=torch.bfloat16)
    at = torch.randperm(V, generator=g)
    for p in parts:
        row[at[:len(p)]] = p.to(torch.bfloat16)
        at = at[len(p):]
    return row


def _alone_and_together(lib, rows, settings, copies=1):
    """The rows in one call (more than two for each SM if copied), and each by
    itself, where a long row has several CTAs."""
    rows = rows.cuda()
    n = rows.shape[0] * copies
    u = np.linspace(0, 1, n, endpoint=False, dtype=np.float32)
    _check(lib, rows.repeat(copies, 1), u, **settings)
    for i in range(rows.shape[0]):
        _check(lib, rows[i:i + 1], 0.61, **settings)
    assert lib.device_error() == 0


@pytest.mark.parametrize("settings", SETTINGS, ids=ids)
@pytest.mark.parametrize("V", [5003, 151936])
def test_around_the_ends_of_the_range(lib, V, settings):
    few = lambda *v: torch.tensor([x for x in v for _ in range(11)])  # noqa: E731
    rows = [_scatter(V, [few(*v)], rest, i) for i, (v, rest) in enumerate((
        ((-4064.0, -4080.0, -4096.0, -4128.0), -5000.0),      # the lowest maximum in the range
        ((-4064.0, -4080.0, -4096.0), float("-inf")),
        ((-4080.0, -4096.0, -4128.0), float("-inf")),         # weights reach below it
        ((-4096.0, -4128.0), float("-inf")),                  # a maximum at its end
        ((4080.0, 4064.0, 4048.0), 4000.0),                   # the highest one in the range
        ((4080.0, -4080.0, -4096.0, 0.0), float("-inf")),
        ((4096.0, 4080.0, 4064.0), 4000.0),                   # and the first one past it
        ((4096.0, -4096.0), 4095.0)))]
    _alone_and_together(lib, torch.stack(rows), settings)


@pytest.mark.parametrize("settings", SETTINGS, ids=ids)
@pytest.mark.parametrize("V", [5003, 151936])
def test_around_the_smallest_bins(lib, V, settings):
    # the bit patterns on both sides of +-2^-19, and zeros of both signs
    b = [NEAR - 2, NEAR - 1, NEAR, NEAR + 1]
    part = _bits([s | x for s in (0, 0x8000) for x in b + [0] for _ in range(7)])
    rows = torch.stack([_scatter(V, [part], rest, i) for i, rest in enumerate((float("-inf"), -3.0, 1.5))])
    _alone_and_together(lib, rows, settings)


@pytest.mark.parametrize("V,copies", [(5003, 1), (5003, 60), (151936, 1)])
@pytest.mark.parametrize("settings", SETTINGS, ids=ids)
def test_the_list_of_values_near_zero(lib, V, copies, settings):
    rng = np.random.default_rng(V + copies)
    rows = []
    for i, n in enumerate((127, 254, 255, 256, 257, 256)):
        b = rng.choice(np.arange(1, NEAR), n, replace=False) | 0x8000 * rng.integers(0, 2, n)
        if i == 5:
            b[1::2] = b[::2]  # every value twice
        zeros = torch.tensor([0.0, -0.0] * 20) if i % 2 else torch.empty(0)
        rows.append(_scatter(V, [_bits(b), zeros], -4.0 if i < 3 else float("-inf"), n + i))
    # the list full with one value, with and without a zero beside it
    rows.append(_scatter(V, [_bits([5] * 256)], -2.0, 1))
    rows.append(_scatter(V, [_bits([0x8005] * 255), torch.zeros(1)], -2.0, 2))
    rows.append(_scatter(V, [_bits([0x8005] * 256), torch.zeros(1)], -2.0, 3))
    _alone_and_together(lib, torch.stack(rows), settings, copies)
