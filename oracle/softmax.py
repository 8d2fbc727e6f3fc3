"""Losses over a vocabulary in float64, from their definitions: one token at a time, one target at a time."""
from __future__ import annotations

import math

import numpy as np


def shares(ids, logits, V: int, tau: float):
    """{entry: share} of one token's targets, and sum_k p_k log p_k; {} without any."""
    there = [k for k in range(len(ids)) if 0 <= ids[k] < V]
    q = [0.0 if logits is None else float(logits[k]) / tau for k in there]
    if not there or all(v == -math.inf for v in q):
        return {}, 0.0
    top = max(q)
    total = sum(math.exp(v - top) for v in q)
    p, entropy = {}, 0.0
    for k, v in zip(there, q):
        share = math.exp(v - top) / total
        p[int(ids[k])] = p.get(int(ids[k]), 0.0) + share
        if share > 0.0:
            entropy += share * ((v - top) - math.log(total))
    return p, entropy


def loss_and_gradients(x, w, ids, weights, logits=None, tau: float = 1.0):
    """x [T, M], w [V, M], ids [T, K], weights [T], all float64 or integers: loss [T], lse [T], D [T, V], dx [T, M], dw [V, M]."""
    T, V = x.shape[0], w.shape[0]
    u = (x @ w.T) / tau
    top = u.max(axis=1, keepdims=True) if T else u[:, :1]
    lse = (top + np.log(np.exp(u - top).sum(axis=1, keepdims=True)))[:, 0]
    d = np.exp(u - lse[:, None])
    loss = np.zeros(T)
    for t in range(T):
        p, entropy = shares(ids[t], None if logits is None else logits[t], V, tau)
        loss[t] = entropy - sum(s * (u[t, v] - lse[t]) for v, s in p.items() if s > 0.0)
        for v, s in p.items():
            d[t, v] -= s
        d[t] *= weights[t] / tau if p else 0.0
    return loss, lse, d, d @ w, d.T @ x
