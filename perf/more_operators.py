"""Timed cases of the operators of a verify step over a cache held in 8 bits.

Three operators, each in a plain form (elementary torch operations) and, with
``own`` set, as a user calls them in this package:

  append  new K/V rows into pages of e4m3 values with one power-of-two scale a
          page, KV head and tensor; a page's scale grows when new rows need it,
          and what the page holds already is brought to the new one
  attend  span-causal attention of a few queries a request (one: decode) over
          such a cache, grouped heads
  drafts  verification of drafted tokens against the target's probabilities:
          accepted while u q(x) < p(x), then one token from the normalised
          (p - q)+ of the first rejected position (from the target's row behind
          the drafts when none was), from given uniform numbers
"""
import math
import random

import torch

own = False

PAGE = 16
D = 128
LN2 = math.log(2.0)
LEAST = 87  # least scale byte: 2^(87 - 127)


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one decode step of a batch: every request appends a single token
        {"name": "append decode", "op": "append", "seqs": 128, "new_lo": 1, "new_hi": 1, "old_lo": 16, "old_hi": 256,
         "hkv": 8, "lens_seed": 1},
        # a verify step: spans of 1 to 16 drafted tokens into the verifier's cache
        {"name": "append spans", "op": "append", "seqs": 64, "new_lo": 1, "new_hi": 16, "old_lo": 0, "old_hi": 200,
         "hkv": 4, "lens_seed": 2},
        # a batch of new prompts
        {"name": "append prompts", "op": "append", "seqs": 12, "new_lo": 200, "new_hi": 2000, "old_lo": 0, "old_hi": 0,
         "hkv": 4, "lens_seed": 3},
        # the latency of one request's token early in its answer
        {"name": "attend one short", "op": "attend", "seqs": 1, "q_lo": 1, "q_hi": 1, "len_lo": 77, "len_hi": 77,
         "hq": 16, "hkv": 8, "lens_seed": 4},
        # one request's token at the end of a long context: the work has to be split along the keys
        {"name": "attend one long", "op": "attend", "seqs": 1, "q_lo": 1, "q_hi": 1, "len_lo": 100003, "len_hi": 100003,
         "hq": 32, "hkv": 4, "lens_seed": 5},
        # a decode step of a rollout batch with contexts of very different lengths
        {"name": "attend decode", "op": "attend", "seqs": 128, "q_lo": 1, "q_hi": 1, "len_lo": 256, "len_hi": 16384,
         "hq": 16, "hkv": 8, "lens_seed": 6},
        # the larger model verifies spans of up to 16 tokens: up to 128 rows share a KV head's keys
        {"name": "attend spans", "op": "attend", "seqs": 64, "q_lo": 1, "q_hi": 16, "len_lo": 256, "len_hi": 16384,
         "hq": 32, "hkv": 4, "lens_seed": 7},
        # short ragged spans with an odd group of heads, empty requests among them
        {"name": "attend odd", "op": "attend", "seqs": 24, "q_lo": 0, "q_hi": 9, "len_lo": 1, "len_hi": 1500,
         "hq": 10, "hkv": 2, "lens_seed": 8},
        # the drafts of a single request
        {"name": "drafts one", "op": "drafts", "seqs": 1, "k_lo": 4, "k_hi": 4, "vocab": 151936, "bonus": True,
         "noise": 0.8, "lens_seed": 9},
        # a serving batch with short drafts, settings of its own in every request
        {"name": "drafts batch", "op": "drafts", "seqs": 32, "k_lo": 0, "k_hi": 6, "vocab": 151936, "bonus": True,
         "noise": 0.8, "lens_seed": 10},
        # an odd vocabulary, no row behind the drafts, two models that agree less
        {"name": "drafts odd", "op": "drafts", "seqs": 33, "k_lo": 1, "k_hi": 5, "vocab": 50021, "bonus": False,
         "noise": 1.5, "lens_seed": 11},
        # the spans of a rollout batch
        {"name": "drafts rollout", "op": "drafts", "seqs": 64, "k_lo": 1, "k_hi": 16, "vocab": 151936, "bonus": False,
         "noise": 0.8, "lens_seed": 12},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["append", "attend", "attend", "drafts"])
    hq, hkv = rng.choice([(32, 4), (16, 8), (16, 8), (8, 8), (12, 4), (7, 1), (10, 2)])
    if op == "append":
        kind = rng.choice(["decode", "span", "prompt"])
        if kind == "decode":
            seqs, new, old = _log_int(rng, 1, 128), (1, 1), (0, 256)
        elif kind == "span":
            seqs, new, old = _log_int(rng, 1, 64), (0, 16), (0, 200)
        else:
            seqs, new, old = _log_int(rng, 1, 12), (1, _log_int(rng, 20, 1000)), (0, 40)
        return {"op": op, "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "old_lo": old[0], "old_hi": old[1],
                "hkv": hkv, "lens_seed": rng.randrange(1 << 30)}
    if op == "attend":
        seqs = _log_int(rng, 1, 128)
        hi = _log_int(rng, 30, max(31, min(100000, 400000 // seqs)))
        q = rng.choice([(1, 1), (1, 1), (1, 16), (0, rng.randint(2, 12))])
        if q != (1, 1):
            seqs, hi = max(1, seqs // 2), min(hi, 12000)
        return {"op": op, "seqs": seqs, "q_lo": q[0], "q_hi": q[1], "len_lo": rng.choice([1, max(1, hi // 4)]), "len_hi": hi,
                "hq": hq, "hkv": hkv, "lens_seed": rng.randrange(1 << 30)}
    lo, hi = rng.choice([(0, 4), (1, 8), (1, 12), (3, 3)])
    return {"op": op, "seqs": _log_int(rng, 1, 48), "k_lo": lo, "k_hi": hi,
            "vocab": rng.choice([151936, 50021, 32000, 4096, 1001]) - rng.choice([0, 0, 1, 3]), "bonus": rng.random() < 0.5,
            "noise": rng.choice([0.3, 0.8, 1.5]), "lens_seed": rng.randrange(1 << 30)}


def _whole(case, key, spread=False):
    """One whole number a request between the case's bounds (over their logarithm where spread)."""
    lo, hi = case[key + "_lo"], case[key + "_hi"]
    rng = random.Random("%s %d" % (key, case["lens_seed"]))
    n = [min(hi, max(lo, _log_int(rng, lo, hi) if spread else rng.randint(lo, hi))) for _ in range(case["seqs"])]
    n[0] = hi  # the range's upper end is always there
    return n


def _attend_lens(case):
    """(queries, cached tokens) a request; a request has no more queries than tokens."""
    n = _whole(case, "len", spread=True)
    return [min(a, b) for a, b in zip(_whole(case, "q"), n)], n


def _cu(n, device):
    return torch.tensor([0] + n, dtype=torch.int64).cumsum(0).to(torch.int32).to(device)


def _i32(v, device):
    return torch.tensor(v, dtype=torch.int32, device=device)


def _page_table(length, spare, g, device):
    """Pages of every request, drawn at random from a pool with a few more."""
    pages = [(x + PAGE - 1) // PAGE for x in length]
    n = sum(pages) + spare
    perm = torch.randperm(n, generator=g, device=device).to(torch.int32).cpu()
    table = torch.full((len(length), max(1, max(pages))), -1, dtype=torch.int32)
    at = 0
    for r, x in enumerate(pages):
        table[r, :x] = perm[at:at + x]
        at += x
    return table.to(device), n


# ---------------------------------------------------------------- the inputs
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    ri = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device=dev)  # noqa: E731
    st = {"case": case}
    e4m3 = torch.float8_e4m3fn
    if case["op"] in ("append", "attend"):
        hkv = case["hkv"]
        if case["op"] == "append":
            new, old = _whole(case, "new"), _whole(case, "old")
            length = [a + b for a, b in zip(new, old)]
        else:
            new, length = _attend_lens(case)
        table, pages = _page_table(length, 3, g, dev)
        # a page's largest entry lies in the upper half of what 8 bits hold; heads and pages differ in scale
        fill = lambda: (rn(pages, hkv, PAGE, D) * 90).clamp_(-448, 448).to(e4m3)  # noqa: E731
        head = ri(-1, 2, hkv)
        scale = lambda: (121 + head + ri(-2, 2, pages, hkv)).to(torch.uint8)  # noqa: E731
        st |= {"k_pages": fill(), "v_pages": fill(), "k_scale": scale(), "v_scale": scale(), "table": table,
               "cu": _cu(new, dev), "length": _i32(length, dev)}
        if case["op"] == "append":
            # K and V stay where a projection wrote them, side by side
            kv = (rn(sum(new), 2 * hkv, D) * torch.exp2(ri(-2, 3, sum(new), 1, 1).float())).to(torch.bfloat16)
            st |= {"k": kv[:, :hkv], "v": kv[:, hkv:]}
        else:
            q = rn(sum(new), case["hq"], D).to(torch.bfloat16)
            st |= {"q": q, "out": torch.empty_like(q), "q_len": new, "len": length}
        return st
    R, V, k = case["seqs"], case["vocab"], _whole(case, "k")
    T, B = sum(k), (R if case["bonus"] else 0)
    target = rn(T + B, V) * 2.0
    target.scatter_add_(1, ri(0, V, T + B, 24), 8 + 2 * rn(T + B, 24))  # a few likely tokens above the rest
    target[:, V - V // 200:] = torch.finfo(torch.bfloat16).min  # entries no vocabulary item stands behind
    target[:, ri(0, V, V // 50)] = float("-inf")                # and forbidden ones
    draft = (target[:T] + case["noise"] * rn(T, V)).to(torch.bfloat16)
    target = target.to(torch.bfloat16)
    pick = lambda vals: torch.tensor(vals, device=dev)[ri(0, len(vals), R)].float()  # noqa: E731
    inv_p, inv_q = pick([1.0, 1.0, 1.0 / 0.6, 1.0 / 0.8, 1.0 / 1.2]), pick([1.0, 1.0, 1.0 / 0.8])
    # the draft model's tokens, drawn from its own softmax
    per = torch.repeat_interleave(inv_q, torch.tensor(k, device=dev))[:, None]
    noise = -torch.log(-torch.log(torch.rand(T, V, generator=g, device=dev).clamp_(1e-12, 1 - 2.0 ** -24)))
    tokens = (draft.float() * per + noise).argmax(-1).to(torch.int32)
    return st | {"target": target[:T], "draft": draft, "bonus": target[T:] if B else None, "tokens": tokens,
                 "cu": _cu(k, dev), "k": k, "u": torch.rand(T, generator=g, device=dev),
                 "u_next": torch.rand(R, generator=g, device=dev), "inv_p": inv_p, "inv_q": inv_q,
                 "accepted": _i32([0] * R, dev), "next": _i32([0] * R, dev),
                 "logp_p": torch.empty(T, device=dev), "logp_q": torch.empty(T, device=dev)}


# ---------------------------------------------------------------- one pass
def run(st):
    return (_run_own if own else _run_plain)(st)


def _outputs(st):
    op = st["case"]["op"]
    if op == "append":
        return {n: st[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale")}
    if op == "attend":
        return {"out": st["out"]}
    return {n: st[n] for n in ("accepted", "next", "logp_p", "logp_q")}


def _run_own(st):
    from paper_2609_36546_gb300 import ipd

    op = st["case"]["op"]
    if op == "append":
        if "cache" not in st:
            st["cache"] = ipd.KVCache8(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
        ipd.kv8_append(st["cache"], st["k"], st["v"], st["cu"], st["length"], st["table"])
    elif op == "attend":
        if "batch" not in st:
            cache = ipd.KVCache8(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
            st["batch"] = [ipd.AttnBatch8(cache, st["q"], st["cu"], st["length"], st["table"], st["out"],
                                          max(1, max(st["q_len"])), max(st["len"]))]
            st["ws"] = torch.empty(max(256, ipd.attn8_workspace_size(st["batch"])), dtype=torch.uint8, device="cuda")
        ipd.verify_attn8(st["batch"], [], D ** -0.5, st["ws"])
    else:
        if "ws" not in st:
            st["ws"] = torch.empty(max(256, ipd.verify_draft_workspace_size(len(st["k"]), st["u"].numel(), st["case"]["vocab"])),
                                   dtype=torch.uint8, device="cuda")
        ipd.verify_draft(st["target"], st["draft"], st["tokens"], st["cu"], st["u"], st["u_next"], st["accepted"],
                         st["next"], st["ws"], logits_bonus=st["bonus"], inv_temp_target=st["inv_p"],
                         inv_temp_draft=st["inv_q"], logp_target=st["logp_p"], logp_draft=st["logp_q"])
    return _outputs(st)


def _run_plain(st):
    op = st["case"]["op"]
    if op == "append":
        n = st["k"].shape[0]
        tok = torch.arange(n, device=st["k"].device)
        cu = st["cu"].long()
        req = torch.searchsorted(cu[1:], tok, right=True)
        pos = st["length"].long()[req] - cu[req + 1] + tok
        page, slot = st["table"][req, pos // PAGE].long(), pos % PAGE
        lead = (slot == 0) | (tok == cu[req])  # the first new row of its page
        _append_plain(st["k_pages"], st["k_scale"], st["k"].float(), page, slot, lead)
        _append_plain(st["v_pages"], st["v_scale"], st["v"].float(), page, slot, lead)
    elif op == "attend":
        # padded groups of requests, as many as a gigabyte of keys in 32 bits holds
        order = sorted(range(len(st["len"])), key=lambda r: st["len"][r])
        while order:
            n = 1
            while n < len(order) and st["len"][order[-1]] * (n + 1) * st["case"]["hkv"] * D * 4 <= 1 << 30:
                n += 1
            _attend_plain(st, order[-n:])
            del order[-n:]
    else:
        _drafts_plain(st)
    return _outputs(st)


def _append_plain(pages, scale, x, page, slot, lead):
    amax = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)  # [n, heads]
    most = torch.zeros(scale.shape, device=x.device).index_reduce_(0, page, amax, "amax")
    # the least power of two that brings the largest entry to 448 = 7/8 2^9 or below
    frac, exp = torch.frexp(most)
    need = torch.where(most > 0, (exp - 9 + (frac > 0.875).int() + 127).clamp(LEAST, 254), LEAST)
    at, first = page[lead], slot[lead]  # a page once
    was = torch.where((first > 0)[:, None], scale[at].int(), LEAST)
    now = torch.maximum(need[at], was)
    held = pages[at].float() * torch.exp2((was - now).float())[..., None, None]
    stays = torch.arange(PAGE, device=x.device) < first[:, None]
    raw = pages.view(torch.uint8)
    raw[at] = torch.where(stays[:, None, :, None], held.to(pages.dtype).view(torch.uint8), raw[at])
    scale[at] = now.to(torch.uint8)
    y = x * torch.exp2(127.0 - scale[page].float())[..., None]
    raw[page, :, slot] = y.to(pages.dtype).view(torch.uint8)


def _attend_plain(st, reqs):
    dev, hkv = st["q"].device, st["case"]["hkv"]
    G = st["case"]["hq"] // hkv
    q_len, n = [st["q_len"][r] for r in reqs], [st["len"][r] for r in reqs]
    nq, np_ = max(q_len), (max(n) + PAGE - 1) // PAGE
    if nq == 0:
        return
    sel = torch.tensor(reqs, device=dev)
    ql, ln, first = torch.tensor(q_len, device=dev), torch.tensor(n, device=dev), st["cu"].long()[sel]
    page = st["table"][sel, :np_].clamp_min(0).long()

    def wide(pages, scale):
        x = pages.view(torch.uint8)[page].view(pages.dtype).float()
        x = x * torch.exp2(scale[page].float() - 127)[..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(len(reqs), hkv, np_ * PAGE, D)

    i = torch.arange(nq, device=dev)
    row = (first[:, None] + i).clamp_max(st["q"].shape[0] - 1)
    q = st["q"][row].float().view(len(reqs), nq, hkv, G, D).permute(0, 2, 3, 1, 4).reshape(len(reqs), hkv, G * nq, D)
    s = q @ wide(st["k_pages"], st["k_scale"]).transpose(-1, -2) * D ** -0.5
    key = torch.arange(np_ * PAGE, device=dev)
    seen = key <= ((ln - ql)[:, None] + i)[..., None]  # [request, query, key]
    s = s.view(len(reqs), hkv, G, nq, -1).masked_fill_(~seen[:, None, None], float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = (s - m).exp_()
    p = p.div_(p.sum(-1, keepdim=True)).view(len(reqs), hkv, G * nq, -1)
    v = wide(st["v_pages"], st["v_scale"]).masked_fill_((key >= ln[:, None])[:, None, :, None], 0.0)
    o = (p @ v).view(len(reqs), hkv, G, nq, D).permute(0, 3, 1, 2, 4).reshape(len(reqs), nq, hkv * G, D)
    live = i < ql[:, None]
    st["out"][row[live]] = o[live].to(torch.bfloat16)


# 2^f on [-1/2, 1/2] by Horner's rule (a least-squares fit on Chebyshev nodes, constant term 1)
POW2 = (1.0, 0.6931468844413757, 0.24022237956523895, 0.05550893023610115, 0.009671698324382305, 0.0013218672247603536)


def _weights(logits, inv_t):
    """(x, whole-number weights round(2^30 2^x)) of x = (l - max l) log2(e) / temperature: every fp32 product and sum
    rounded on its own, as the draws of this package define them."""
    l = logits.float()
    l = torch.where(l.isnan(), float("-inf"), l)
    top = l.amax(-1, keepdim=True)
    c = (torch.tensor(1.0 / LN2, device=l.device) * inv_t)[:, None]
    x = torch.where(l == top, 0.0, l - top) * c
    y = x.clamp_min(-64.0)
    i = y.round()
    f = y - i
    p = torch.full_like(y, POW2[5])
    p = p * f + POW2[4]
    p = p * f + POW2[3]
    p = p * f + POW2[2]
    p = p * f + POW2[1]
    p = p * f + POW2[0]
    y = (p.view(torch.int32) + (i.to(torch.int32) << 23)).view(torch.float32)  # p 2^i, exact
    w = ((y * 2.0 ** 31).to(torch.int64) + 1) >> 1
    return x, torch.where(l == float("-inf"), 0, w)


def _drafts_plain(st):
    dev, R, T = st["u"].device, len(st["k"]), st["u"].numel()
    cu = st["cu"].long()
    tok = torch.arange(T, device=dev)
    req = torch.searchsorted(cu[1:], tok, right=True)
    xp, wp = _weights(st["target"], st["inv_p"][req])
    xq, wq = _weights(st["draft"], st["inv_q"][req])
    zp, zq = wp.sum(-1), wq.sum(-1)
    at = st["tokens"].long()[:, None]
    for x, z, name in ((xp, zp, "logp_p"), (xq, zq, "logp_q")):
        logp = (x.gather(1, at).squeeze(1).double() - (z.double() * 2.0 ** -30).log2()) * LN2
        st[name].copy_(torch.where(z > 0, logp, float("-inf")))
    px, qx = wp.gather(1, at).squeeze(1).double(), wq.gather(1, at).squeeze(1).double()
    ok = st["u"].double() * qx * zp.double() < px * zq.double()
    k = cu[1:] - cu[:-1]
    n = k.scatter_reduce(0, req, torch.where(ok, k[req], tok - cu[req]), "amin")  # drafts before the first rejected one
    row = (cu[:-1] + n).clamp_max(max(T - 1, 0))
    full = n == k
    if T:
        p, q, zp, zq = wp[row], wq[row], zp[row], zq[row]
    else:
        p = q = torch.zeros(R, st["case"]["vocab"], dtype=torch.int64, device=dev)
        zp = zq = p[:, 0]
    # (p - q)+ in units of p's weights: q's times the ratio of the sums, whose 31 leading bits count
    frac, exp = torch.frexp(zp.double() / zq.double())
    m = (frac * 2.0 ** 31).to(torch.int64)[:, None]
    less = torch.where((zq > 0)[:, None], (q * m) >> (31 - exp).clamp(0, 62)[:, None].long(), 0)
    r = (p - less).clamp_min(0)
    r = torch.where(r.sum(-1, keepdim=True) > 0, r, p)
    if st["bonus"] is not None:
        r = torch.where(full[:, None], _weights(st["bonus"], st["inv_p"])[1], r)
    cum = r.cumsum(-1)
    s = cum[:, -1]
    t = torch.minimum((st["u_next"].double() * s.double()).floor().long(), s - 1)
    nxt = (cum <= t[:, None]).sum(-1).clamp_max(r.shape[1] - 1)
    none = (s == 0) | (full if st["bonus"] is None else torch.zeros_like(full))
    st["next"].copy_(torch.where(none, -1, nxt))
    st["accepted"].copy_(n)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "append":
        n, hkv = sum(_whole(case, "new")), case["hkv"]
        return {"bytes": n * hkv * 2 * D * 3, "flops": 3 * n * hkv * 2 * D}
    if case["op"] == "attend":
        q, n = _attend_lens(case)
        live = [(a, b) for a, b in zip(q, n) if a]
        kv = sum(b * 2 * D + (b + PAGE - 1) // PAGE * 2 for _, b in live) * case["hkv"]
        return {"bytes": kv + sum(q) * case["hq"] * D * 4,
                "flops": sum(4 * D * case["hq"] * (a * b - a * (a - 1) // 2) for a, b in live)}
    T, V = sum(_whole(case, "k")), case["vocab"]
    return {"bytes": 4 * T * V + 24 * T, "flops": 16 * T * V}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "append":
        new = _whole(case, "new")
        length, table = st["length"].tolist(), st["table"].tolist()
        rows = [(r, length[r] - new[r] + i) for r in range(len(new)) for i in range(new[r])]
        out = {}
        for t in ("k", "v"):
            x, pages, scale = st[t].double().cpu(), st[t + "_pages"].double().cpu(), st[t + "_scale"].long().cpu()
            groups = {}
            for j, (r, pos) in enumerate(rows):
                groups.setdefault(table[r][pos // PAGE], []).append((pos % PAGE, j))
            for page, what in groups.items():
                slots, js = [a for a, _ in what], [b for _, b in what]
                top = x[js].abs().amax(dim=(0, 2))
                e = torch.ceil(torch.log2(top / 448)).clamp_min(LEAST - 127).long() + 127
                if slots[0]:
                    e = torch.maximum(e, scale[page])
                    pages[page, :, :slots[0]] *= (2.0 ** (scale[page] - e).double())[:, None, None]
                pages[page, :, slots] = (x[js] / (2.0 ** (e - 127).double())[:, None]).transpose(0, 1)
                scale[page] = e
            out[t + "_pages"], out[t + "_scale"] = pages, None
        return out
    if case["op"] == "attend":
        G, cu = case["hq"] // case["hkv"], st["cu"].tolist()
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        for r, (a, n) in enumerate(zip(st["q_len"], st["len"])):
            if not a:
                continue
            page = st["table"][r, :(n + PAGE - 1) // PAGE].long()
            hidden = torch.ones(a, n, dtype=torch.bool, device="cuda").triu(n - a + 1)
            for h in range(case["hkv"]):
                k, v = ((st[t + "_pages"].view(torch.uint8)[page, h].view(torch.float8_e4m3fn).double()
                         * 2.0 ** (st[t + "_scale"][page, h].double() - 127)[:, None, None]).view(-1, D)[:n] for t in ("k", "v"))
                q = st["q"][cu[r]:cu[r] + a, h * G:(h + 1) * G].double()
                s = torch.einsum("igd,jd->gij", q, k) / math.sqrt(D)
                s = s.masked_fill(hidden, float("-inf"))
                out[cu[r]:cu[r] + a, h * G:(h + 1) * G] = torch.einsum("gij,jd->igd", torch.softmax(s, -1), v)
        return {"out": out}
    per = torch.tensor(st["k"], device="cuda")
    out = {"accepted": None, "next": None}
    for name, logits, inv in (("logp_p", st["target"], st["inv_p"]), ("logp_q", st["draft"], st["inv_q"])):
        z = logits.double() * torch.repeat_interleave(inv, per).double()[:, None]
        out[name] = torch.log_softmax(z, -1).gather(1, st["tokens"].long()[:, None]).squeeze(1)
    return out
