"""From prompts to a verified span, on one GPU.

    python examples/prompt_to_verify.py [--requests 8] [--span 4]

Both models read a batch of prompts into their own paged caches (rotary
positions, cache append, causal attention), the student draws the first token
of its span at the settings a serving user gives, its drafted span enters both
caches, and the teacher verifies it in one step.  The models' layers are not
part of this library: their projections and logits are random stand-ins here,
of the shapes of one attention layer and one LM head each.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_36546_gb300 import PromptPass, VerifyStep, ipd  # noqa: E402

TEACHER, STUDENT = (32, 4), (16, 8)  # query heads, KV heads; head_dim 128


def make_cache(hkv, pages, dev):
    shape = (pages, hkv, 16, 128)
    return ipd.KVCache(*(torch.zeros(shape, dtype=torch.bfloat16, device=dev) for _ in range(2)))


def main(requests=8, span=4, vocab=4096, max_prompt=700, seed=0, quiet=False):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    lens = torch.randint(1, max_prompt + 1, (requests,), generator=host).tolist()
    # pages for the prompt, the span and the draft's next token, in any order
    need = [(n + span + 1 + 15) // 16 for n in lens]
    perm = torch.randperm(sum(need), generator=host).to(torch.int32)
    ptab = torch.full((requests, max(need)), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        ptab[r, :n] = perm[at:at + n]
        at += n
    table = torch.empty(max_prompt + span + 1, 64, 2, device=dev)
    ipd.rope_table(table, base=1e6)
    rows = lambda n, heads: torch.randn(n, heads, 128, generator=g, device=dev).to(torch.bfloat16)

    caches, outs, spans = {}, {}, {}
    ctx = torch.tensor([n + span for n in lens], dtype=torch.int32)
    cu_span = torch.arange(requests + 1, dtype=torch.int32, device=dev) * span
    for name, (hq, hkv) in (("teacher", TEACHER), ("student", STUDENT)):
        caches[name] = make_cache(hkv, sum(need), dev)
        # the prompts: one projection's output holds q, k and v side by side
        qkv = rows(sum(lens), hq + 2 * hkv)
        p = PromptPass(caches[name], table, lens, ptab, hq, device=dev)
        outs[name] = p.run(qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:])
        # the drafted span's rows behind them
        qkv = rows(requests * span, hq + 2 * hkv)
        q = torch.empty(requests * span, hq, 128, dtype=torch.bfloat16, device=dev)
        ipd.rope_append(caches[name], qkv[:, :hq], q, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:],
                        cu_span, ctx.to(dev), ptab.to(dev), table)
        spans[name] = q

    # the student's draft: every position drawn at the user's settings
    logits_s = (torch.randn(requests * span, vocab, generator=g, device=dev) * 2.5).to(torch.bfloat16)
    logits_t = (logits_s.float() + 0.3 * torch.randn(logits_s.shape, generator=g, device=dev)).to(torch.bfloat16)
    n = requests * span
    u = torch.rand(n, generator=g, device=dev)
    full = lambda v, dt=torch.float32: torch.full((n,), v, dtype=dt, device=dev)
    tokens, logp = torch.empty(n, dtype=torch.int32, device=dev), torch.empty(n, device=dev)
    ipd.sample_trunc(logits_s, u, tokens, inv_temperature=full(1.25), top_k=full(50, torch.int32),
                     top_p=full(0.95), min_p=full(0.0), logp=logp)

    # one verify step over the caches just filled: the student proposed throughout
    none = lambda hq: torch.empty(0, hq, 128, dtype=torch.bfloat16, device=dev)
    step = VerifyStep(caches["teacher"].k_pages, caches["teacher"].v_pages,
                      caches["student"].k_pages, caches["student"].v_pages, ctx,
                      torch.full((requests,), span), torch.zeros(requests, dtype=torch.uint8),
                      ptab, ptab, spans["teacher"], none(STUDENT[0]),
                      spans["student"][span - 1::span].contiguous(), none(TEACHER[0]), tokens,
                      logits_s, logits_t, K=16)
    step.run()
    torch.cuda.synchronize()
    err = ipd.device_error()
    if err:
        raise RuntimeError(f"device error: {ipd.DEVERR[err]}")
    if not quiet:
        print(f"{requests} prompts of {min(lens)} to {max(lens)} tokens, spans of {span}")
        print("first drafted tokens", tokens.view(requests, span)[:, 0].tolist())
        print("emitted per request ", step.score["n_emit"].tolist())
        print("next driver         ", step.score["next_driver"].tolist())
        print("loss                ", float(step.out8[0]))
    return {"lens": lens, "outs": outs, "tokens": tokens, "logp": logp, "step": step,
            "caches": caches, "page_table": ptab, "spans": spans}


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--requests", type=int, default=8)
    a.add_argument("--span", type=int, default=4)
    a = a.parse_args()
    main(a.requests, a.span)
