"""Verification of drafted tokens by its definition, in whole numbers (numpy)."""
import math

import numpy as np

F = np.float32
POW2 = [F(x) for x in np.array([0x3F800000, 0x3F317213, 0x3E75FCDB, 0x3D635D55, 0x3C1E760B, 0x3AAD4281],
                               dtype=np.uint32).view(np.float32)]
LOG2E = F(1.4426950408889634)


def weights(l, inv_t):
    """(x, w) of a row of logits (fp32 values of bf16)."""
    l = np.where(np.isnan(l), F(-np.inf), l.astype(F))
    top = l.max()
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.where(l == top, F(0), (l - top).astype(F)) * F(LOG2E * F(inv_t))
    y = np.maximum(x, F(-64)).astype(F)
    i = np.rint(y).astype(F)
    f = (y - i).astype(F)
    p = np.full_like(y, POW2[5])
    for c in POW2[4::-1]:
        p = (p * f).astype(F)
        p = (p + c).astype(F)
    w = np.ldexp(p.astype(np.float64), i.astype(np.int64) + 31).astype(np.int64)
    return x, np.where(l == -np.inf, 0, (w + 1) >> 1)


def position(u, s):
    t = math.floor(float(u) * float(s)) if u > 0 else 0
    return min(t, s - 1)


def pick(r, u):
    s = int(r.sum())
    if s == 0:
        return -1
    return int(np.searchsorted(np.cumsum(r), position(u, s), side="right"))


def residual(wp, wq):
    zp, zq = int(wp.sum()), int(wq.sum())
    if zq == 0:
        return wp
    f, e = math.frexp(float(zp) / float(zq))
    m, s = int(f * 2.0 ** 31), 31 - e
    r = np.array([max(0, int(a) - (int(b) * m >> s)) if a else 0 for a, b in zip(wp, wq)], dtype=np.int64)
    return r if r.any() else wp


def verify(target, draft, bonus, tokens, cu, u, u_next, inv_p, inv_q):
    """Per request (n_accept, next_token), per token (logp_target, logp_draft) in 64 bits."""
    verdict, logp = [], []
    for r in range(len(cu) - 1):
        n, out = 0, None
        for t in range(cu[r], cu[r + 1]):
            (xp, wp), (xq, wq), tok = weights(target[t], inv_p[r]), weights(draft[t], inv_q[r]), tokens[t]
            zp, zq = int(wp.sum()), int(wq.sum())
            inside = 0 <= tok < len(wp)
            logp.append([float(x[tok]) * math.log(2) - math.log(z * 2.0 ** -30) if z and inside else -math.inf if inside else math.nan
                         for x, z in ((xp, zp), (xq, zq))])
            if out is None:
                if inside and float(u[t]) * float(wq[tok]) * float(zp) < float(wp[tok]) * float(zq):
                    n += 1
                else:
                    out = pick(residual(wp, wq), u_next[r]) if zp else -1
        if out is None:
            out = -1 if bonus is None else pick(weights(bonus[r], inv_p[r])[1], u_next[r])
        verdict.append((n, out))
    return verdict, logp
