"""Where the six coefficients of the draws' whole-number weights come from (CPU only).

The weights of truncated sampling and of the verification of drafts evaluate 2^f as
P(f), f in [-1/2, 1/2], with a degree-5 P of constant term 1 (include/ipd.h at
ipd_sample_trunc, csrc/weights.cuh, and the definition in the tests each state the
coefficients).  P is the least-squares fit of 2^f, relative to 2^f, at Chebyshev nodes
of that interval, rounded to fp32.  This test redoes the fit with numpy and checks the
rounded coefficients in each place.
"""
import os
import re

import numpy as np

from tests import draft_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def fit_pow2_coefficients(n_nodes: int = 1000) -> tuple:
    """fp32 bit patterns, lowest degree first: P = 1 + f Q, Q of degree 4, least squares of
    (P(f) - 2^f) / 2^f at n Chebyshev nodes (first kind) of [-1/2, 1/2]."""
    f = 0.5 * np.cos((2 * np.arange(n_nodes) + 1) * np.pi / (2 * n_nodes))
    y = np.exp2(f)
    coef = np.linalg.lstsq(np.vander(f, 6, increasing=True)[:, 1:] / y[:, None], (y - 1) / y, rcond=None)[0]
    return tuple(int(w) for w in np.append(1.0, coef).astype(np.float32).view(np.uint32))


def test_fit_reproduces_the_coefficients():
    want = fit_pow2_coefficients()
    header = open(os.path.join(ROOT, "include", "ipd.h")).read()
    words = re.search(r"bit patterns, lowest degree first\) (3F800000[0-9A-F \s*]+)\n", header).group(1)
    assert tuple(int(w, 16) for w in re.findall(r"[0-9A-F]{8}", words)) == want
    source = open(os.path.join(ROOT, "paper_2609_36546_gb300", "csrc", "weights.cuh")).read()
    named = dict((int(i), int(h, 16)) for i, h in re.findall(r"\bc([1-5]) = __uint_as_float\(0x([0-9a-f]{8})u\)", source))
    assert tuple(named[i] for i in range(1, 6)) == want[1:]
    assert tuple(int(np.float32(c).view(np.uint32)) for c in draft_ref.POW2) == want


def test_the_rounded_fit_does_not_depend_on_the_node_count():
    for n in (64, 257, 4000):
        assert fit_pow2_coefficients(n) == fit_pow2_coefficients()


def test_the_fit_s_relative_error():
    """Below 1.9e-7 with the roundings of Horner's rule in fp32."""
    f = np.linspace(-0.5, 0.5, 200001).astype(np.float32)
    p = np.full_like(f, draft_ref.POW2[5])
    for c in draft_ref.POW2[4::-1]:
        p = (p * f).astype(np.float32)
        p = (p + c).astype(np.float32)
    assert float(np.abs(p.astype(np.float64) / np.exp2(f.astype(np.float64)) - 1).max()) < 1.9e-7
