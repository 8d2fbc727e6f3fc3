"""Bounds of the losses' gradients by the precision that D, the gradient with respect to the logits, has on a call's path:
float32, two bfloat16 parts (its rounding and what that loses, up to 128 tokens), or one.  Everything else as Problem.check() derives it."""
from __future__ import annotations

import numpy as np
import torch

from tests.losses import FLOAT, ROUND

# What D is off by, relative: a rounding to float32; the second part's rounding, 2^-8 of at most 2^-8 of D; one rounding to bfloat16.
D_FLOAT, D_TWO, D_ONE = 2.0 ** -24, 2.0 ** -16, 2.0 ** -8


def d_precision(p):
    return D_FLOAT if p.dtype == "f32" else D_TWO if p.T <= 128 else D_ONE


def exact_logits(p):
    """The problem with operands whose logits have no rounding in fp32, in any order of their sums: x in halves, w in 64ths."""
    for name, step in (("x", 0.5), ("w", 1.0 / 64)):
        full = np.round(getattr(p, name) / step) * step
        t = getattr(p, name + "t")
        setattr(p, name, full)
        setattr(p, name + "t", torch.from_numpy(full.astype(np.float32)).to(t.dtype))
    assert (np.abs(p.x) @ np.abs(p.w).T).max(initial=0.0) < 2.0 ** 16
    return p


def check_gradients(p, got, precision=None):
    """dx and dw of `got` (of a problem with exact logits) element by element.  u, exp, log: roundings of values up to |u|; lse: those and 2^-18 for its sum.  D: those errors times its
    two terms, its own precision, and 2^-126 where a bfloat16 part is below the smallest normal number.  The products' sums of n terms: fp32, no more than n / 4 additions one after the
    other (vector instructions; a matrix instruction adds 32 terms, with a few roundings) and 64 for ranges, parts and joining.  One rounding of the result."""
    loss, lse, d, dx, dw = p.expected()
    u = (p.x @ p.w.T) / p.tau
    du = 8 * FLOAT * (np.abs(u).max(axis=1) + 1)
    dl = 2 * du + 2.0 ** -18 + 4 * FLOAT * np.abs(lse)
    q = 0.0 if p.logits is None else 16 * FLOAT * (np.abs(p.logits[np.isfinite(p.logits)]).max(initial=0.0) / p.tau + 2)
    weights = np.ones(p.T) if p.weights is None else p.weights.astype(np.float64)
    there = ((p.ids >= 0) & (p.ids < p.V)).any(axis=1)
    share = np.exp(u - lse[:, None]) * (weights * there / p.tau)[:, None]
    terms = share + np.abs(d - share)
    r = d_precision(p) if precision is None else precision
    off = 1.01 * r * np.abs(d) + (2 * dl[:, None] + q + 16 * FLOAT) * terms + 2.0 ** -126
    for name, ref, a, big, b, n in (("dx", dx, off, np.abs(d), np.abs(p.w), p.V), ("dw", dw, off.T, np.abs(d).T, np.abs(p.x), p.T)):
        if name in got:
            most = 1.02 * (a @ b) + 1.01 * ROUND[p.dtype] * np.abs(ref) + (n / 4 + 64) * FLOAT * (big @ b) + 1e-38
            bad = ~(np.abs(got[name] - ref) <= most)
            assert not bad.any(), (name, int(bad.sum()), float((np.abs(got[name] - ref) / most)[bad].max()))
