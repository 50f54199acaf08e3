"""Causal attention of packed prompts on the GPU against plain attention in 64
bits (needs a GB300).

Tolerance, with a = sum_j w_j |v_j| the weighted mean magnitude of what an
output averages: the weights are rounded to bf16 for the product with V, at
most 2^-8 of each term, 2^-8 a in all; the output is rounded to bf16, 2^-8
(|o| + 2^-8 a); the exponential (2^-22), fp32 scores (128 products: at most
2^-14 of a weight at these magnitudes) and fp32 sums stay far below 2^-10 a.
The log-sum carries the scores' error and the sum's: 1e-4 + 2^-22 |lse|.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd
    ipd.device_error()
    return ipd


def _cu(lens):
    return torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32).cuda()


def _make(lens, hq, hkv, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(lens)
    rn = lambda h: torch.randn(n, h, D, generator=g, device="cuda")
    return (rn(hq) * spread).to(torch.bfloat16), rn(hkv).to(torch.bfloat16), rn(hkv).to(torch.bfloat16)


def _ref(q, k, v, lens, scale):
    """(output, weighted mean |v|, lse) in 64 bits, sequence by sequence; only
    visible keys enter a sum."""
    hq, hkv = q.shape[1], k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(out)
    lse = torch.zeros(hq, q.shape[0], dtype=torch.float64, device="cuda")
    at = 0
    for n in lens:
        for h in range(hq):
            j = h * hkv // hq
            s = q[at:at + n, h].double() @ k[at:at + n, j].double().T * scale
            hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
            s = s.masked_fill(hidden, float("-inf"))
            w = torch.softmax(s, -1)
            vv = v[at:at + n, j].double()
            if torch.isfinite(vv).all():
                out[at:at + n, h], mag[at:at + n, h] = w @ vv, w @ vv.abs()
            else:
                for i in range(n):
                    out[at + i, h] = (w[i, :i + 1, None] * vv[:i + 1]).sum(0)
                    mag[at + i, h] = (w[i, :i + 1, None] * vv[:i + 1].abs()).sum(0)
            lse[h, at:at + n] = torch.logsumexp(s, -1)
        at += n
    return out, mag, lse


def _run(lib, q, k, v, lens, scale=D ** -0.5, max_len=None):
    out = torch.full_like(q, 7.0) if q.is_contiguous() else torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    lib.prompt_attn(q, k, v, _cu(lens), max(lens) if max_len is None else max_len, out, scale, lse=lse)
    return out, lse


def _close(out, lse, ref, mag, rlse):
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(out))
    assert torch.equal(torch.isnan(ref), torch.isnan(out))
    inf = torch.isinf(ref)
    assert torch.equal(out.double()[inf], ref[inf])
    err, tol = (out.double() - ref).abs(), 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -10) * mag
    assert bool((err <= tol)[fine].all()), float((err / tol)[fine].max())
    ok = torch.isfinite(rlse)
    assert torch.equal(lse.double()[~ok].nan_to_num(1e9), rlse[~ok].nan_to_num(1e9))
    assert bool(((lse.double() - rlse).abs() <= 1e-4 + 2.0 ** -22 * rlse.abs())[ok].all())


@pytest.mark.parametrize("hq,hkv,lens", [
    (16, 8, [29]), (16, 8, [1]), (32, 4, [1, 0, 2, 127, 128, 129, 0, 255, 256, 257]),
    (16, 8, [300, 64, 65, 1, 513]), (8, 8, [130, 700]), (7, 1, [200, 3, 37]), (10, 2, [77, 411]),
    (12, 4, [85, 84, 86]), (128, 1, [5, 130]), (100, 1, [140]), (64, 2, [33]), (32, 4, [1500, 900]),
    (1, 1, [1025]), (3, 1, [0, 42, 43, 126, 127])])
def test_prompt_attn(lib, hq, hkv, lens):
    q, k, v = _make(lens, hq, hkv, seed=len(lens) + hq)
    out, lse = _run(lib, q, k, v, lens)
    _close(out, lse, *_ref(q, k, v, lens, D ** -0.5))
    assert lib.device_error() == 0


def test_many_short_sequences(lib):
    """More sequences than lanes and than resident CTAs, lengths 0 .. 40."""
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 41, (333,), generator=g).tolist()
    q, k, v = _make(lens, 4, 2, seed=2)
    out, lse = _run(lib, q, k, v, lens)
    _close(out, lse, *_ref(q, k, v, lens, D ** -0.5))


def test_growing_scores_rescale(lib):
    """Scores that grow along the sequence (the running maximum moves by far
    more than the lazy threshold, tile after tile) and scores that fall."""
    lens = [700, 400]
    q, k, v = _make(lens, 8, 4, seed=3)
    pos = torch.cat([torch.arange(n) for n in lens]).cuda().float()
    for f in (1 + pos / 64, 12 / (1 + pos / 64)):
        kk = (k.float() * f[:, None, None]).to(torch.bfloat16)
        out, lse = _run(lib, q, kk, v, lens)
        ref, mag, rlse = _ref(q, kk, v, lens, D ** -0.5)
        # scores up to ~80 here: their fp32 sums carry up to 2^-20 of |q||k|, so
        # a weight up to 2^-12: within the 2^-10 a of the tolerance
        _close(out, lse, ref, mag, rlse)


def test_max_len_above_and_strided_views(lib):
    """q, k, v as views into one projection output, out into a wider buffer, and
    a generous length bound: the bits of the contiguous call."""
    lens, hq, hkv = [200, 31, 129], 16, 8
    n = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn(n, hq + 2 * hkv, D, generator=g, device="cuda").to(torch.bfloat16)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    want, wl = _run(lib, q.contiguous(), k.contiguous(), v.contiguous(), lens)
    wide = torch.full((n, hq + 3, D), 5.0, dtype=torch.bfloat16, device="cuda")
    lib.prompt_attn(q, k, v, _cu(lens), 10 ** 6, wide[:, 1:hq + 1], D ** -0.5)
    assert torch.equal(wide[:, 1:hq + 1], want)
    assert (wide[:, 0] == 5.0).all() and (wide[:, hq + 1:] == 5.0).all()


def test_broken_values_stay_where_they_are_seen(lib):
    """NaN and infinities in keys and values reach the rows that see them and
    no other: not earlier rows of the sequence, not the other sequences."""
    lens, hq, hkv = [150, 90, 300, 40], 8, 4
    q, k, v = _make(lens, hq, hkv, seed=5)
    clean, _ = _run(lib, q, k, v, lens)
    start = [0, 150, 240, 540]
    vb, kb = v.clone(), k.clone()
    vb[start[1] + 50, 1, 7] = float("nan")
    vb[start[2] + 0, 0, 0] = float("inf")
    vb[start[2] + 131, 2, 100] = float("-inf")
    vb[start[2] + 299, 3, :] = float("inf")
    vb[start[3] + 20, 0, 64] = float("inf")
    vb[start[3] + 30, 0, 64] = float("-inf")
    kb[start[0] + 149, 0, 3] = float("nan")
    kb[start[3] + 39, 2, :] = float("inf")
    out, lse = _run(lib, q, kb, vb, lens)
    ref, mag, rlse = _ref(q, kb, vb, lens, D ** -0.5)
    _close(out, lse, ref, mag.nan_to_num(0, 0, 0), rlse)
    # rows untouched by any of them keep their bits
    assert torch.equal(out[start[1]:start[1] + 50], clean[start[1]:start[1] + 50])
    assert torch.equal(out[:149], clean[:149])


def test_masks_of_minus_infinity(lib):
    """Keys whose scores are all -inf: rows that see only such keys are NaN with
    a log-sum of -inf, as the formula has it; later rows forget them."""
    lens = [140]
    q, k, v = _make(lens, 2, 1, seed=6)
    q[..., 0], k[..., 0] = 1.0, 0.0
    k[:130, :, 0] = float("-inf")
    out, lse = _run(lib, q, k, v, lens)
    assert torch.isnan(out[:130]).all() and (lse[:, :130] == float("-inf")).all()
    ref, mag, rlse = _ref(q, k, v, lens, D ** -0.5)
    _close(out, lse, ref, mag.nan_to_num(0), rlse)


def test_bad_offsets(lib):
    """Sequences out of order, past the tensors or longer than the bound are
    recorded and left out; the others are computed."""
    lens = [100, 50, 60]
    q, k, v = _make(lens, 4, 2, seed=7)
    want, _ = _run(lib, q, k, v, lens)
    for cu, max_len, code, good in (([0, 100, 90, 150], 100, 6, [0]), ([0, 100, 150, 211], 100, 6, [0, 1]),
                                    ([-1, 100, 150, 210], 101, 6, [1, 2]), ([0, 100, 150, 210], 99, 2, [1, 2])):
        out = torch.full_like(q, 7.0)
        lib.prompt_attn(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), max_len, out, D ** -0.5)
        assert lib.device_error() == code
        at = 0
        for r, n in enumerate(lens):
            if r in good:
                assert torch.equal(out[at:at + n], want[at:at + n]), (cu, r)
            at += n
        if code == 2:
            assert (out[:100] == 7.0).all()
    assert lib.device_error() == 0


def test_rows_outside_the_offsets(lib):
    """Rows before cu_seq[0] and after its end are not written."""
    q, k, v = _make([130], 4, 2, seed=8)
    out = torch.full_like(q, 7.0)
    lib.prompt_attn(q, k, v, torch.tensor([10, 10, 120], dtype=torch.int32, device="cuda"), 110, out, D ** -0.5)
    want, _ = _run(lib, q[10:120].contiguous(), k[10:120].contiguous(), v[10:120].contiguous(), [110])
    assert torch.equal(out[10:120], want)
    assert (out[:10] == 7.0).all() and (out[120:] == 7.0).all()
    empty = torch.empty(0, 4, D, dtype=torch.bfloat16, device="cuda")
    lib.prompt_attn(empty, empty[:, :2], empty[:, :2], _cu([0]), 0, empty, D ** -0.5)


def test_same_bits_every_run_and_on_a_side_stream(lib):
    lens = [800, 3, 250]
    q, k, v = _make(lens, 16, 8, seed=9)
    a, la = _run(lib, q, k, v, lens)
    b, lb = _run(lib, q, k, v, lens)
    assert torch.equal(a, b) and torch.equal(la, lb)
    side, late, cu = torch.cuda.Stream(), torch.zeros_like(q), _cu(lens)
    out = torch.empty_like(q)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late.copy_(q)
    lib.prompt_attn(late, k, v, cu, 800, out, D ** -0.5, stream=side)
    side.synchronize()
    assert torch.equal(out, a)


def test_last_row_is_decode_over_the_cache(lib):
    """The last query of each prompt is what the decode attention gives over a
    paged cache of the same keys (its weights are not rounded to bf16)."""
    lens, hq, hkv = [77, 300], 16, 8
    q, k, v = _make(lens, hq, hkv, seed=10)
    out, _ = _run(lib, q, k, v, lens)
    pages = [(n + 15) // 16 for n in lens]
    cache = lib.KVCache(*(torch.zeros(sum(pages), hkv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    ptab = torch.full((2, max(pages)), -1, dtype=torch.int32)
    ptab[0, :pages[0]] = torch.arange(pages[0])
    ptab[1, :pages[1]] = torch.arange(pages[0], sum(pages))
    ptab, length = ptab.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    lib.kv_append(cache, k, v, _cu(lens), length, ptab)
    last = torch.tensor([lens[0] - 1, sum(lens) - 1], device="cuda")
    b = lib.AttnBatch(cache, q[last].contiguous(), _cu([1, 1]), length, ptab, torch.empty_like(q[last]), 1, max(lens))
    ws = torch.empty(lib.attn_workspace_size([], [b]), dtype=torch.uint8, device="cuda")
    lib.decode_attn([b], 1 / math.sqrt(D), ws)
    _, mag, _ = _ref(q, k, v, lens, D ** -0.5)
    err = (b.out.double() - out[last].double()).abs()
    # both round the output (2^-8 each); the prompt's weights add 2^-8 mag
    assert bool((err <= 2.0 ** -7 * out[last].double().abs() + (2.0 ** -8 + 2.0 ** -10) * mag[last]).all())
