"""The 8-bit cache, the attention over it and the verification of drafts as a serving
loop uses them together (needs a GB300).

Two models read their prompts into 8-bit caches.  Every round the draft's tokens enter
both caches, one call attends the target's spans and the draft's last tokens, the target
verifies the drafted tokens, and the lengths move to what was kept: the rows of rejected
tokens are written over in the next round.  The caches' bytes are compared with the
append's definition, the attention with plain attention in 64 bits over those bytes, the
verdicts with their definition.

The attention's tolerance is its own tests' but for the scores, which are larger here: q is
off by 2^-17 of its row's largest entry at most, so a score of 128 terms by
128 2^-17 |q|max |k|max / 11.3, which is 0.0095 where |q|max |k|max is 110 (checked), and
a normalised weight by twice that of itself: 0.019 a beside the (2^-9 + 2^-10) a of the rest,
0.022 a together, within 5 (2^-8 + 2^-10) a = 0.024 a.
"""
import numpy as np
import pytest
import torch

from . import draft_ref, kv8_ref
from .test_gpu_attn8 import Case

pytestmark = pytest.mark.gpu

TARGET, DRAFT = (32, 4), (16, 8)


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_36546_gb300 import ipd
    ipd.device_error()
    return ipd


class Model:
    """One model's cache on the GPU and by its definition."""

    def __init__(self, lib, heads, pages, table):
        (self.hq, self.hkv), self.lib, self.table = heads, lib, table
        self.cache = lib.KVCache8.empty(pages, self.hkv)
        self.kv = [(np.zeros((pages, self.hkv, 16, 128), np.uint8), np.full((pages, self.hkv), 127, np.uint8)) for _ in "kv"]

    def note(self, k, v, lens, counts):
        """The append by its definition: `counts` rows that end at `lens`."""
        for (pages, scale), x in zip(self.kv, (k, v)):
            x, at = x.float().cpu().numpy(), 0
            for r, (end, n) in enumerate(zip(lens, counts)):
                pos = end - n
                while pos < end:
                    m = min(end, (pos // 16 + 1) * 16)
                    p = int(self.table[r, pos // 16])
                    kv8_ref.append(pages[p], scale[p], x[at:at + m - pos], np.arange(pos % 16, pos % 16 + m - pos))
                    at, pos = at + m - pos, m

    def same(self, lens):
        c = self.cache
        for (pages, scale), gp, gs in zip(self.kv, (c.k_pages, c.v_pages), (c.k_scale, c.v_scale)):
            gp, gs = gp.view(torch.uint8).cpu().numpy(), gs.cpu().numpy()
            for r, n in enumerate(lens):
                for i in range((n + 15) // 16):
                    p, m = int(self.table[r, i]), min(16, n - 16 * i)
                    assert np.array_equal(gs[p], scale[p])
                    assert kv8_ref.same_bytes(gp[p][:, :m], pages[p][:, :m])

    def case(self, lens, counts):
        """For the attention's reference: the cache's own bytes."""
        c = Case.__new__(Case)
        c.hq, c.hkv, c.q_len, c.length = self.hq, self.hkv, list(counts), list(lens)
        c.table, c.kp, c.vp, c.ks, c.vs = self.table, self.cache.k_pages, self.cache.v_pages, self.cache.k_scale, self.cache.v_scale
        return c


def test_prompts_then_rounds_of_drafts(lib):
    from paper_2609_36546_gb300 import PromptPass

    R, span, V, rounds = 7, 4, 3001, 4
    g = torch.Generator(device="cuda").manual_seed(3)
    host = torch.Generator().manual_seed(3)
    lens = [1, 15, 16, 17, 130, 333, 600]
    need = [(n + rounds * (span + 1) + 15) // 16 for n in lens]
    table = torch.full((R, max(need)), -1, dtype=torch.int32)
    perm, at = torch.randperm(sum(need), generator=host).to(torch.int32), 0
    for r, n in enumerate(need):
        table[r, :n] = perm[at:at + n]
        at += n
    table = table.cuda()
    rope = torch.empty(max(lens) + rounds * (span + 1), 64, 2, device="cuda")
    lib.rope_table(rope, base=1e6)
    rows = lambda n, h, s=1.0: (torch.randn(n, h, 128, generator=g, device="cuda") * s).to(torch.bfloat16)
    target, draft = models = [Model(lib, h, sum(need), table) for h in (TARGET, DRAFT)]

    top = {}
    for m in models:
        qkv = rows(sum(lens), m.hq + 2 * m.hkv)
        q, k, v = qkv[:, :m.hq], qkv[:, m.hq:m.hq + m.hkv], qkv[:, m.hq + m.hkv:]
        p = PromptPass(m.cache, rope, lens, table, m.hq)
        out = p.run(q, k, v).clone()
        m.note(p.k, v, lens, lens)
        top[m] = float(p.k.abs().max())
        m.same(lens)
        # the output is that of a pass over a bf16 cache
        pools = [torch.zeros(sum(need), m.hkv, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        assert torch.equal(out, PromptPass(lib.KVCache(*pools), rope, lens, table, m.hq).run(q, k, v))

    cu = torch.arange(R + 1, dtype=torch.int32, device="cuda") * span
    cu1 = torch.arange(R + 1, dtype=torch.int32, device="cuda")
    i32 = lambda *s: torch.full(s, -9, dtype=torch.int32, device="cuda")
    n_accept, next_token = i32(R), i32(R)
    logp = [torch.empty(R * span, device="cuda") for _ in "pq"]
    seen = set()
    for step in range(rounds):
        lens = [n + span for n in lens]
        seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        new = []
        for m in models:
            # (magnitudes that rise and fall, so that the pages' scales have to move)
            k, v = rows(R * span, m.hkv, 2.0 ** (step % 3)), rows(R * span, m.hkv, 2.0 ** step)
            pos = torch.cat([torch.arange(n - span, n, dtype=torch.int32) for n in lens]).cuda()
            lib.rope(k, k, pos, rope)
            new.append((m.cache, k, v, cu, seq, table))
            m.note(k, v, lens, [span] * R)
            top[m] = max(top[m], float(k.abs().max()))
        lib.kv8_append_many(new)
        qt, qd = rows(R * span, target.hq), rows(R, draft.hq)
        ot, od = torch.empty_like(qt), torch.empty_like(qd)
        spans = [lib.AttnBatch8(target.cache, qt, cu, seq, table, ot, span, max(lens))]
        lasts = [lib.AttnBatch8(draft.cache, qd, cu1, seq, table, od, 1, max(lens))]
        ws = torch.empty(lib.attn8_workspace_size(spans, lasts), dtype=torch.uint8, device="cuda")
        lib.verify_attn8(spans, lasts, 128 ** -0.5, ws)

        lq = (torch.randn(R * span, V, generator=g, device="cuda") * 2.5).to(torch.bfloat16)
        lp = (lq.float() + 0.5 * torch.randn(R * span, V, generator=g, device="cuda")).to(torch.bfloat16)
        bonus = (torch.randn(R, V, generator=g, device="cuda") * 2.5).to(torch.bfloat16)
        tokens = i32(R * span)
        lib.sample_trunc(lq, torch.rand(R * span, generator=g, device="cuda"), tokens)
        u, un = torch.rand(R * span, generator=g, device="cuda"), torch.rand(R, generator=g, device="cuda")
        wd = torch.empty(lib.verify_draft_workspace_size(R, R * span, V), dtype=torch.uint8, device="cuda")
        lib.verify_draft(lp, lq, tokens, cu, u, un, n_accept, next_token, wd, logits_bonus=bonus, logp_target=logp[0],
                         logp_draft=logp[1])
        assert lib.device_error() == 0

        for m, q, o, counts in ((target, qt, ot, [span] * R), (draft, qd, od, [1] * R)):
            m.same(lens)
            c = m.case(lens, counts)
            c.q = q
            want, tol = c.ref(128 ** -0.5)
            assert float(q.abs().max()) * top[m] <= 110
            assert bool(((o.double() - want).abs() <= 5 * tol).all())
        f = lambda t: t.float().cpu().numpy()
        want, want_logp = draft_ref.verify(f(lp), f(lq), f(bonus), tokens.cpu().numpy(), cu.cpu().numpy(), u.cpu().numpy(),
                                           un.cpu().numpy(), np.ones(R, np.float32), np.ones(R, np.float32))
        assert [tuple(x) for x in torch.stack((n_accept, next_token), 1).tolist()] == want
        kept = n_accept.tolist()
        seen.update(kept)
        lens = [n - span + k for n, k in zip(lens, kept)]
    assert len(seen) > 1  # requests that kept all and that did not


def test_a_round_as_a_graph(lib):
    """Append, attention and verification captured in one graph and replayed on another
    stream over new inputs give what the calls give."""
    R, span, V, L = 5, 3, 2000, 700
    g = torch.Generator(device="cuda").manual_seed(5)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
    hq, hkv = TARGET
    pages = R * ((L + 15) // 16)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(R, -1)
    cu = torch.arange(R + 1, dtype=torch.int32, device="cuda") * span
    full = torch.tensor([L, 16, 3, 333, 50], dtype=torch.int32, device="cuda")
    ctx = full - span
    ctx_cu = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), ctx.cumsum(0).to(torch.int32)])

    def fresh():
        c = lib.KVCache8.empty(pages, hkv)
        lib.kv8_append(c, hist_k, hist_v, ctx_cu, ctx, table)
        return c

    hist_k, hist_v = rn(int(ctx.sum()), hkv, 128), rn(int(ctx.sum()), hkv, 128)
    k, v, q = rn(R * span, hkv, 128), rn(R * span, hkv, 128), rn(R * span, hq, 128)
    lp, lq = rn(R * span, V), rn(R * span, V)
    tokens = torch.randint(0, V, (R * span,), generator=g, device="cuda", dtype=torch.int32)
    u, un = torch.rand(R * span, generator=g, device="cuda"), torch.rand(R, generator=g, device="cuda")

    def make(cache):
        out, na, nt = torch.zeros_like(q), torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
        b = [lib.AttnBatch8(cache, q, cu, full, table, out, span, L)]
        ws = torch.empty(lib.attn8_workspace_size(b), dtype=torch.uint8, device="cuda")
        wd = torch.empty(lib.verify_draft_workspace_size(R, R * span, V), dtype=torch.uint8, device="cuda")

        def run():
            lib.kv8_append(cache, k, v, cu, full, table)
            lib.verify_attn8(b, [], 128 ** -0.5, ws)
            lib.verify_draft(lp, lq, tokens, cu, u, un, na, nt, wd)
        return run, (out, na, nt, cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.k_scale, cache.v_scale)

    cache = fresh()
    run, res = make(cache)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for t in (k, v, q, lp, lq):
        t.copy_(rn(*t.shape))
    lib.kv8_append(cache, hist_k, hist_v, ctx_cu, ctx, table)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph.replay()
        graph.replay()  # (an append of the same rows again changes nothing)
    side.synchronize()
    plain, want = make(fresh())
    plain()
    torch.cuda.synchronize()
    n = (full + 15) // 16
    for a, b in zip(res[:3], want[:3]):
        assert torch.equal(a, b)
    for a, b in zip(res[3:], want[3:]):
        for r in range(R):
            p = table[r, :int(n[r])].long()
            last, rows = int(p[-1]), int(full[r]) - 16 * (int(n[r]) - 1)
            assert torch.equal(a[p[:-1]], b[p[:-1]])
            assert torch.equal(a[last][:, :rows], b[last][:, :rows]) if a.dim() == 4 else torch.equal(a[last], b[last])
    assert lib.device_error() == 0
