"""Timed cases of the operators that take a prompt to its first proposed token.

Four operators, each in a plain form (elementary torch operations in 32 bits)
and, with ``own`` set, as a user calls them in this package:

  append   rotary positions of new queries and keys, and the write of the new
           K/V rows into the paged cache, in one call
  rotary   rotary positions alone, forward or transposed (its gradient)
  prompt   causal attention of packed prompts, grouped heads
  sample   one token per row from the softmax at a temperature, cut by top-k,
           min-p and top-p, from given uniform numbers
"""
import math
import random

import torch

own = False

PAGE = 16
D = 128
LN2 = math.log(2.0)


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one decode step of a batch: every request appends a single token
        {"name": "append decode", "op": "append", "seqs": 128, "new_lo": 1, "new_hi": 1, "old_lo": 16, "old_hi": 256,
         "hq": 16, "hkv": 8, "rot": 128, "layout": "half", "scaled": False, "k_out": False, "lens_seed": 1},
        # a verify step: spans of 1 to 16 drafted tokens into the verifier's cache
        {"name": "append spans", "op": "append", "seqs": 64, "new_lo": 1, "new_hi": 16, "old_lo": 0, "old_hi": 200,
         "hq": 32, "hkv": 4, "rot": 128, "layout": "half", "scaled": True, "k_out": False, "lens_seed": 2},
        # a batch of new prompts, half of each head rotated in the interleaved layout
        {"name": "append prompts", "op": "append", "seqs": 12, "new_lo": 200, "new_hi": 2000, "old_lo": 0, "old_hi": 0,
         "hq": 32, "hkv": 4, "rot": 64, "layout": "interleaved", "scaled": True, "k_out": True, "lens_seed": 3},
        # a few rows at scattered positions, as a re-scored span has them
        {"name": "rotary rows", "op": "rotary", "n": 37, "heads": 32, "rot": 128, "layout": "half",
         "dtype": "bf16", "inverse": False, "max_pos": 32768},
        # the gradient of rotated queries in a training batch, three quarters of each head rotated
        {"name": "rotary gradient", "op": "rotary", "n": 8191, "heads": 16, "rot": 96, "layout": "half",
         "dtype": "f32", "inverse": True, "max_pos": 8192},
        # one short question: the latency of a single small call
        {"name": "prompt one short", "op": "prompt", "seqs": 1, "len_lo": 29, "len_hi": 29, "hq": 16, "hkv": 8,
         "lens_seed": 5},
        # a ragged batch of prompts packed without padding, an empty slot among them
        {"name": "prompt ragged", "op": "prompt", "seqs": 24, "len_lo": 0, "len_hi": 900, "hq": 16, "hkv": 8,
         "lens_seed": 6},
        # one long context taken in whole, the larger model's heads
        {"name": "prompt one long", "op": "prompt", "seqs": 1, "len_lo": 8192, "len_hi": 8192, "hq": 32, "hkv": 4,
         "lens_seed": 7},
        # the next token of a single request
        {"name": "sample one", "op": "sample", "n": 1, "vocab": 151936, "cut": "top-p", "logits": "boost"},
        # a batch in which every request brings its own settings
        {"name": "sample mixed", "op": "sample", "n": 64, "vocab": 151936, "cut": "mixed", "logits": "boost"},
        # an odd vocabulary, nothing cut, flat logits with forbidden entries
        {"name": "sample uncut odd", "op": "sample", "n": 33, "vocab": 50021, "cut": "none", "logits": "normal"},
        # the first tokens of a whole rollout batch
        {"name": "sample rollout", "op": "sample", "n": 512, "vocab": 151936, "cut": "mixed", "logits": "boost"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["append", "rotary", "prompt", "sample"])
    hq, hkv = rng.choice([(32, 4), (16, 8), (16, 8), (8, 8), (12, 4), (7, 1), (10, 2)])
    if op == "append":
        kind = rng.choice(["decode", "span", "prompt"])
        if kind == "decode":
            seqs, new, old = _log_int(rng, 1, 128), (1, 1), (0, 256)
        elif kind == "span":
            seqs, new, old = _log_int(rng, 1, 64), (0, 16), (0, 200)
        else:
            seqs, new, old = _log_int(rng, 1, 12), (1, _log_int(rng, 20, 2000)), (0, 40)
        return {"op": op, "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "old_lo": old[0], "old_hi": old[1], "hq": hq, "hkv": hkv,
                "rot": rng.choice([128, 128, 64, 96, 32, 50]), "layout": rng.choice(["half", "interleaved"]),
                "scaled": rng.random() < 0.5, "k_out": kind == "prompt", "lens_seed": rng.randrange(1 << 30)}
    if op == "rotary":
        return {"op": op, "n": _log_int(rng, 1, 8191), "heads": rng.choice([1, 7, 8, 16]),
                "rot": rng.choice([128, 64, 96, 32, 50]), "layout": rng.choice(["half", "interleaved"]),
                "dtype": rng.choice(["bf16", "f32"]), "inverse": rng.random() < 0.5,
                "max_pos": rng.choice([8192, 32768])}
    if op == "prompt":
        seqs = _log_int(rng, 1, 40)
        hi = _log_int(rng, 17, max(18, min(8000, 16384 // seqs)))
        return {"op": op, "seqs": seqs, "len_lo": rng.choice([0, 1, hi // 2]), "len_hi": hi, "hq": hq, "hkv": hkv,
                "lens_seed": rng.randrange(1 << 30)}
    return {"op": op, "n": _log_int(rng, 1, 500), "vocab": rng.choice([151936, 50021, 32000, 4096, 1001]) - rng.choice([0, 0, 1, 3]),
            "cut": rng.choice(["none", "top-k", "top-p", "min-p", "mixed"]), "logits": rng.choice(["boost", "normal"])}


def _lens(case, key):
    lo, hi = case[key + "_lo"], case[key + "_hi"]
    rng = random.Random("%s %d" % (key, case["lens_seed"]))
    n = [rng.randint(lo, hi) for _ in range(case["seqs"])]
    if hi:
        n[0] = hi  # the range's upper end is always there
    return n


def _cu(n, device):
    return torch.tensor([0] + n, dtype=torch.int64).cumsum(0).to(torch.int32).to(device)


def _table(max_pos, rot, scaled, device):
    """cos and sin of position p times frequency i as [max_pos, rot / 2, 2] fp32; scaled: frequencies
    blended between interpolated and unchanged by their wavelength (Peng et al. 2023), with its magnitude."""
    i = torch.arange(rot // 2, dtype=torch.float64, device=device)
    freq, mag = 1e6 ** (-2.0 * i / rot), 1.0
    if scaled:
        factor, length, fast, slow = 4.0, 32768.0, 32.0, 1.0
        at = lambda turns: rot * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(1e6))  # noqa: E731
        lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), rot - 1)
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        freq = freq / factor * ramp + freq * (1 - ramp)
        mag = 0.1 * math.log(factor) + 1.0
    a = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None] * freq
    return (torch.stack([a.cos(), a.sin()], -1) * mag).float()


# ---------------------------------------------------------------- the inputs
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    st = {"case": case}
    if case["op"] == "append":
        new, old = _lens(case, "new"), _lens(case, "old")
        total, length = sum(new), [a + b for a, b in zip(new, old)]
        pages = [(x + PAGE - 1) // PAGE for x in length]
        n_pages = sum(pages) + 3
        perm = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        ptab = torch.full((case["seqs"], max(1, max(pages))), -1, dtype=torch.int32)
        host, at = perm.cpu(), 0
        for r, n in enumerate(pages):
            ptab[r, :n] = host[at:at + n]
            at += n
        hq, hkv = case["hq"], case["hkv"]
        # one projection's output holds q, k and v side by side
        qkv = rn(total, hq + 2 * hkv, D).to(torch.bfloat16)
        st |= {"q": qkv[:, :hq], "k": qkv[:, hq:hq + hkv], "v": qkv[:, hq + hkv:],
               "k_pages": rn(n_pages, hkv, PAGE, D).to(torch.bfloat16),
               "v_pages": rn(n_pages, hkv, PAGE, D).to(torch.bfloat16),
               "cu": _cu(new, dev), "length": torch.tensor(length, dtype=torch.int32, device=dev),
               "ptab": ptab.to(dev), "table": _table(max(length) + 1, case["rot"], case["scaled"], dev),
               "q_out": torch.empty(total, hq, D, dtype=torch.bfloat16, device=dev),
               "k_out": torch.empty(total, hkv, D, dtype=torch.bfloat16, device=dev) if case["k_out"] else None}
    elif case["op"] == "rotary":
        t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        x = rn(case["n"], case["heads"], D).to(t)
        pos = torch.randint(0, case["max_pos"], (case["n"],), generator=g, device=dev).to(torch.int32)
        st |= {"x": x, "out": torch.empty_like(x), "pos": pos,
               "table": _table(case["max_pos"], case["rot"], False, dev)}
    elif case["op"] == "prompt":
        n = _lens(case, "len")
        total, hq, hkv = sum(n), case["hq"], case["hkv"]
        st |= {"q": rn(total, hq, D).to(torch.bfloat16), "k": rn(total, hkv, D).to(torch.bfloat16),
               # v stays where the projection wrote it, beside k
               "v": rn(total, 2 * hkv, D).to(torch.bfloat16)[:, hkv:],
               "cu": _cu(n, dev), "n": n, "max_len": max(n),
               "out": torch.empty(total, hq, D, dtype=torch.bfloat16, device=dev),
               "lse": torch.empty(hq, total, dtype=torch.float32, device=dev)}
    else:
        n, V = case["n"], case["vocab"]
        logits = rn(n, V) * (2.5 if case["logits"] == "boost" else 1.5)
        if case["logits"] == "boost":  # a few likely tokens above the rest
            logits.scatter_add_(1, torch.randint(0, V, (n, 24), generator=g, device=dev), 8 + 2 * rn(n, 24))
        # entries no vocabulary item stands behind, and forbidden ones
        logits[:, V - V // 200:] = torch.finfo(torch.bfloat16).min
        logits[:, torch.randint(0, V, (V // 50,), generator=g, device=dev)] = float("-inf")
        if n > 8:
            logits[n // 2] = float("-inf")  # a row with nothing left
        pick = lambda vals: torch.tensor(vals, device=dev)[torch.randint(0, len(vals), (n,), generator=g, device=dev)]  # noqa: E731
        cut = case["cut"]
        full = lambda v, t: torch.full((n,), v, dtype=t, device=dev)  # noqa: E731
        mixed = cut == "mixed"
        st |= {"logits": logits.to(torch.bfloat16),
               "u": torch.rand(n, generator=g, device=dev),
               "inv_t": pick([1.0, 1.0, 1.0 / 0.6, 1.0 / 0.8, 1.0 / 1.2]).float(),
               "top_k": pick([0, 20, 50, 1000]).to(torch.int32) if mixed else full(50 if cut == "top-k" else 0, torch.int32),
               "top_p": pick([1.0, 0.95, 0.9, 0.5]).float() if mixed else full(0.95 if cut == "top-p" else 1.0, torch.float32),
               "min_p": pick([0.0, 0.05, 1e-3]).float() if mixed else full(0.05 if cut == "min-p" else 0.0, torch.float32),
               "tokens": torch.empty(n, dtype=torch.int32, device=dev),
               "logp": torch.empty(n, dtype=torch.float32, device=dev),
               "kept": torch.empty(n, dtype=torch.int32, device=dev)}
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    from paper_2609_36546_gb300 import ipd

    case = st["case"]
    if case["op"] == "append":
        cache = ipd.KVCache(st["k_pages"], st["v_pages"])
        ipd.rope_append(cache, st["q"], st["q_out"], st["k"], st["v"], st["cu"], st["length"], st["ptab"],
                        st["table"], layout=_layout(ipd, case), k_out=st["k_out"])
        return _append_outputs(st)
    if case["op"] == "rotary":
        ipd.rope(st["x"], st["out"], st["pos"], st["table"], layout=_layout(ipd, case), inverse=case["inverse"])
        return {"out": st["out"]}
    if case["op"] == "prompt":
        ipd.prompt_attn(st["q"], st["k"], st["v"], st["cu"], st["max_len"], st["out"], D ** -0.5, lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    ipd.sample_trunc(st["logits"], st["u"], st["tokens"], inv_temperature=st["inv_t"], top_k=st["top_k"],
                     top_p=st["top_p"], min_p=st["min_p"], logp=st["logp"], n_kept=st["kept"])
    return {"tokens": st["tokens"], "logp": st["logp"], "kept": st["kept"]}


def _layout(ipd, case):
    return ipd.ROPE_HALF if case["layout"] == "half" else ipd.ROPE_INTERLEAVED


def _append_outputs(st):
    out = {"q": st["q_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if st["k_out"] is not None:
        out["k"] = st["k_out"]
    return out


def _run_plain(st):
    case = st["case"]
    if case["op"] == "append":
        total = st["q"].shape[0]
        tok = torch.arange(total, device=st["q"].device)
        cu = st["cu"].long()
        req = torch.searchsorted(cu[1:], tok, right=True)
        pos = st["length"].long()[req] - cu[req + 1] + tok
        kr = _rotate(st["k"].float(), pos, st["table"], case["layout"], 1.0).to(torch.bfloat16)
        st["q_out"].copy_(_rotate(st["q"].float(), pos, st["table"], case["layout"], 1.0))
        page = st["ptab"][req, pos // PAGE].long()
        st["k_pages"][page, :, pos % PAGE] = kr
        st["v_pages"][page, :, pos % PAGE] = st["v"]
        if st["k_out"] is not None:
            st["k_out"].copy_(kr)
        return _append_outputs(st)
    if case["op"] == "rotary":
        y = _rotate(st["x"].float(), st["pos"].long(), st["table"], case["layout"], -1.0 if case["inverse"] else 1.0)
        st["out"].copy_(y)
        return {"out": st["out"]}
    if case["op"] == "prompt":
        at, G = 0, case["hq"] // case["hkv"]
        for n in st["n"]:  # one prompt at a time: the packed batch has no padding to share
            s = slice(at, at + n)
            q = st["q"][s].float().view(n, case["hkv"], G, D)
            s_ = torch.einsum("ihgd,jhd->hgij", q, st["k"][s].float()) * D ** -0.5
            s_.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=q.device).triu_(1), float("-inf"))
            if n:
                m = s_.amax(-1, keepdim=True)
                p = (s_ - m).exp_()
                z = p.sum(-1, keepdim=True)
                o = torch.einsum("hgij,jhd->ihgd", p.div_(z), st["v"][s].float())
                st["out"][s] = o.reshape(n, case["hq"], D).to(torch.bfloat16)
                st["lse"][:, s] = (m + z.log()).view(case["hq"], n)
            at += n
        return {"out": st["out"], "lse": st["lse"]}
    return _sample_plain(st)


def _rotate(x, pos, table, layout, sign):
    """The first rot entries of each head, as pairs turned by their position's angle; x [n, heads, D]."""
    h = table.shape[1]
    c, s = table[pos, :, 0].unsqueeze(1), sign * table[pos, :, 1].unsqueeze(1)
    y = x.clone()
    a, b = (slice(0, h), slice(h, 2 * h)) if layout == "half" else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


# 2^f on [-1/2, 1/2] by Horner's rule (a least-squares fit on Chebyshev nodes, constant term 1)
POW2 = (1.0, 0.6931468844413757, 0.24022237956523895, 0.05550893023610115, 0.009671698324382305, 0.0013218672247603536)


def _weights(x):
    """Whole-number weights round(2^30 2^x) of x <= 0: every fp32 product and sum rounded on its own."""
    x = x.clamp_min(-64.0)
    i = x.round()
    f = x - i
    p = torch.full_like(x, POW2[5])
    p = p * f + POW2[4]
    p = p * f + POW2[3]
    p = p * f + POW2[2]
    p = p * f + POW2[1]
    p = p * f + POW2[0]
    y = (p.view(torch.int32) + (i.to(torch.int32) << 23)).view(torch.float32)  # p 2^i, exact
    return ((y * 2.0 ** 31).to(torch.int64) + 1) >> 1


def _sample_plain(st):
    l = st["logits"].float()
    l = torch.where(l.isnan(), float("-inf"), l)
    c = (torch.tensor(1.0 / LN2, device=l.device) * st["inv_t"])[:, None]
    top = l.amax(-1, keepdim=True)
    v, idx = torch.sort(l, dim=-1, descending=True, stable=True)
    x = torch.where(v == top, 0.0, v - top) * c
    w = torch.where(v == float("-inf"), 0, _weights(x))
    rank = torch.arange(l.shape[1], device=l.device)
    k = st["top_k"].long()[:, None]
    w = torch.where((k > 0) & (rank >= k), 0, w)
    w = torch.where(w >= (st["min_p"].double() * 2.0 ** 30).ceil().long()[:, None], w, 0)
    cum = w.cumsum(-1)
    mass = cum[:, -1:]
    need = (st["top_p"].double()[:, None] * mass.double()).ceil().long()
    w = torch.where(cum - w < torch.minimum(need.clamp_min(1), mass), w, 0)
    cum = w.cumsum(-1)
    s = cum[:, -1:]
    t = (st["u"].double()[:, None] * s.double()).floor().long()
    at = (cum <= torch.minimum(t, s - 1)).sum(-1, keepdim=True).clamp_max(l.shape[1] - 1)
    none = s == 0
    logp = (x.gather(1, at) - (s.float() * 2.0 ** -30).log2()) * LN2
    return {"tokens": torch.where(none, -1, idx.gather(1, at)).to(torch.int32).squeeze(1),
            "logp": torch.where(none, float("-inf"), logp).squeeze(1),
            "kept": (w > 0).sum(-1).to(torch.int32)}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "append":
        total, hq, hkv = sum(_lens(case, "new")), case["hq"], case["hkv"]
        rows = total * (2 * hq + 4 * hkv + (hkv if case["k_out"] else 0))
        return {"bytes": rows * D * 2 + total * case["rot"] * 4, "flops": 3 * total * (hq + hkv) * case["rot"]}
    if case["op"] == "rotary":
        n, e = case["n"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * n * case["heads"] * D * e + n * (case["rot"] * 4 + 4),
                "flops": 3 * n * case["heads"] * case["rot"]}
    if case["op"] == "prompt":
        n, hq, hkv = _lens(case, "len"), case["hq"], case["hkv"]
        return {"bytes": sum(n) * (2 * hq + 2 * hkv) * D * 2 + sum(n) * hq * 4,
                "flops": sum(2 * D * hq * x * (x + 1) for x in n)}
    n, V = case["n"], case["vocab"]
    return {"bytes": n * V * 2 + n * 32, "flops": 4 * n * V}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "append":
        table, cu, length = st["table"].double().cpu(), st["cu"].tolist(), st["length"].tolist()
        pos = torch.tensor([length[r] - (cu[r + 1] - cu[r]) + i for r in range(case["seqs"])
                            for i in range(cu[r + 1] - cu[r])], dtype=torch.int64)
        req = torch.tensor([r for r in range(case["seqs"]) for _ in range(cu[r + 1] - cu[r])], dtype=torch.int64)
        q = _exact_rotate(st["q"].cpu(), pos, table, case["layout"], False)
        k = _exact_rotate(st["k"].cpu(), pos, table, case["layout"], False)
        kp, vp, ptab = st["k_pages"].double().cpu(), st["v_pages"].double().cpu(), st["ptab"].cpu().long()
        slot = ptab[req, torch.div(pos, PAGE, rounding_mode="floor")] * PAGE + pos % PAGE
        flat = lambda t: t.transpose(1, 2).reshape(-1, case["hkv"], D)  # noqa: E731
        back = lambda t: t.view(-1, PAGE, case["hkv"], D).transpose(1, 2).contiguous()  # noqa: E731
        kp, vp = back(flat(kp).index_copy(0, slot, k)), back(flat(vp).index_copy(0, slot, st["v"].double().cpu()))
        out = {"q": q, "k_pages": kp, "v_pages": vp}
        if st["k_out"] is not None:
            out["k"] = k
        return out
    if case["op"] == "rotary":
        return {"out": _exact_rotate(st["x"].cpu(), st["pos"].long().cpu(), st["table"].double().cpu(), case["layout"], case["inverse"])}
    if case["op"] == "prompt":
        G = case["hq"] // case["hkv"]
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
        cu = st["cu"].tolist()
        for a, b in zip(cu, cu[1:]):
            for h in range(case["hq"]):
                k, v = st["k"][a:b, h // G].double(), st["v"][a:b, h // G].double()
                for i in range(a, b, 2048):
                    j = min(i + 2048, b)
                    s = (st["q"][i:j, h].double() @ k[:j - a].T) / math.sqrt(D)
                    s += torch.full_like(s, float("-inf")).triu(i - a + 1)
                    lse[h, i:j] = torch.logsumexp(s, -1)
                    out[i:j, h] = torch.softmax(s, -1) @ v[:j - a]
        return {"out": out, "lse": lse}
    l = st["logits"].double()
    z = l * st["inv_t"].double()[:, None]
    ok = (l > float("-inf")).any(-1)
    p, idx = torch.where(ok[:, None], torch.softmax(z, -1), 0.0).sort(dim=-1, descending=True, stable=True)
    zs = z.gather(1, idx)
    k = st["top_k"][:, None]
    keep = (k <= 0) | (torch.arange(p.shape[1], device=p.device) < k)
    keep &= p >= st["min_p"].double()[:, None] * p[:, :1]
    p = p * keep
    p = p * (p.cumsum(-1) - p < st["top_p"].double()[:, None] * p.sum(-1, keepdim=True))
    s = p.sum(-1, keepdim=True)
    at = (p.cumsum(-1) <= st["u"].double()[:, None] * s).sum(-1, keepdim=True).clamp_max(p.shape[1] - 1)
    kept = torch.where(p > 0, zs, float("-inf"))
    logp = zs.gather(1, at).squeeze(1) - torch.logsumexp(kept, -1)
    return {"tokens": None, "logp": torch.where(ok, logp, float("-inf")), "kept": None}


def _exact_rotate(x, pos, table, layout, inverse):
    """Each pair as a complex number times cos + i sin (its conjugate for the transposed rotation)."""
    h = table.shape[1]
    x = x.double()
    turn = torch.view_as_complex(table[pos].contiguous())[:, None]
    turn = turn.conj() if inverse else turn
    pairs = torch.stack([x[..., :h], x[..., h:2 * h]], -1) if layout == "half" else x[..., :2 * h].reshape(*x.shape[:-1], h, 2)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y = torch.cat([y[..., 0], y[..., 1]], -1) if layout == "half" else y.reshape(*x.shape[:-1], 2 * h)
    return torch.cat([y, x[..., 2 * h:]], -1)
