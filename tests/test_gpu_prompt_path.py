"""The path from prompts to a verified span (needs a GB300): the operators over
one cache agree with each other."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


def test_example_runs(lib):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import prompt_to_verify as ex
    finally:
        sys.path.pop(0)
    r = ex.main(requests=5, span=3, quiet=True)
    assert r["tokens"].min() >= 0 and torch.isfinite(r["logp"]).all()
    assert all(torch.isfinite(o).all() for o in r["outs"].values())
    n_emit = r["step"].score["n_emit"]
    assert bool(((n_emit >= 0) & (n_emit <= 3)).all())
    assert math.isfinite(float(r["step"].out8[0]))


@pytest.mark.parametrize("hq,hkv,layout", [(32, 4, 0), (16, 8, 1)])
def test_span_over_cache_is_prompt_of_both(lib, hq, hkv, layout):
    """A span verified over the cache that a prompt pass and an append filled
    gives what prompt attention gives for its rows when prompt and span are one
    prompt.  Both round the output to bf16 (2^-8 |o| each); the prompt's weights
    are rounded to bf16 as well, 2^-8 of the weighted mean |v|, and the verify
    attention's error is far below."""
    from paper_2609_36546_gb300 import PromptPass

    lens, span = [200, 37, 513], [5, 16, 1]
    g = torch.Generator(device="cuda").manual_seed(hq)
    R, whole = len(lens), [a + b for a, b in zip(lens, span)]
    qkv = torch.randn(sum(whole), hq + 2 * hkv, D, generator=g, device="cuda").to(torch.bfloat16)
    table = torch.empty(600, 48, 2, device="cuda")
    lib.rope_table(table, base=1e4, scaling="yarn", factor=2.0, trained_len=300.0)
    pages = [(n + 15) // 16 for n in whole]
    ptab = torch.full((R, max(pages)), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(pages):
        ptab[r, :n] = torch.arange(at, at + n, dtype=torch.int32).flip(0)
        at += n

    def cache():
        return lib.KVCache(*(torch.zeros(sum(pages), hkv, 16, D, dtype=torch.bfloat16, device="cuda")
                             for _ in range(2)))

    split = lambda t: (t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:])
    # all at once
    one = cache()
    both = PromptPass(one, table, whole, ptab, hq, layout=layout)
    want = both.run(*split(qkv))
    # prompt first, then the span behind it
    start = [0]
    for n in whole:
        start.append(start[-1] + n)
    head = torch.cat([torch.arange(s, s + n) for s, n in zip(start, lens)]).cuda()
    tail = torch.cat([torch.arange(s + n, s + n + k) for s, n, k in zip(start, lens, span)]).cuda()
    two = cache()
    PromptPass(two, table, lens, ptab, hq, layout=layout).run(*split(qkv[head].contiguous()))
    cu = torch.tensor([0] + span).cumsum(0).to(torch.int32).cuda()
    length = torch.tensor(whole, dtype=torch.int32).cuda()
    q, k, v = split(qkv[tail].contiguous())
    qr = torch.empty(len(tail), hq, D, dtype=torch.bfloat16, device="cuda")
    lib.rope_append(two, q, qr, k, v, cu, length, ptab.cuda(), table, layout=layout)
    assert torch.equal(one.k_pages, two.k_pages) and torch.equal(one.v_pages, two.v_pages)
    b = lib.AttnBatch(two, qr, cu, length, ptab.cuda(), torch.empty_like(qr), max(span), max(whole))
    ws = torch.empty(lib.attn_workspace_size([b], []), dtype=torch.uint8, device="cuda")
    lib.verify_attn([b], [], 1 / math.sqrt(D), ws)
    mag = PromptPass(cache(), table, whole, ptab, hq, layout=layout)
    av = qkv.clone()
    av[:, hq + hkv:] = av[:, hq + hkv:].abs()
    a = mag.run(*split(av))[tail].double()
    err = (b.out.double() - want[tail].double()).abs()
    assert bool((err <= 2.0 ** -7 * want[tail].double().abs() + (2.0 ** -8 + 2.0 ** -9) * a).all())
    assert lib.device_error() == 0


def test_prompt_pass_refuses(lib):
    from paper_2609_36546_gb300 import PromptPass

    c = lib.KVCache(*(torch.zeros(4, 8, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    table = torch.empty(50, 64, 2, device="cuda")
    for lens, rows in (([10, -1], 2), ([51], 1), ([10, 20], 3)):
        with pytest.raises(ValueError):
            PromptPass(c, table, lens, torch.zeros(rows, 4, dtype=torch.int32), 16)
    empty = PromptPass(c, table, [0, 0], torch.zeros(2, 1, dtype=torch.int32), 16)
    rows = lambda h: torch.empty(0, h, D, dtype=torch.bfloat16, device="cuda")
    assert empty.run(rows(16), rows(8), rows(8)).shape == (0, 16, D)
    assert empty.last.tolist() == [-1, -1]
