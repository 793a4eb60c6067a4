"""CPU oracle for the router's auxiliary losses and gradients.

TEST INFRASTRUCTURE ONLY: the plain definitions in float64, token by token; shares no code with the HIP library.  Pins
(tests/test_router_grad_oracle_pins.py): even routing has balance loss 1; central differences of the losses and of the
gates; the product's gradients against differences.
"""
from __future__ import annotations

import numpy as np


def _softmax(row):
    e = np.exp(row - row.max())
    return e / e.sum()


def _lse(row):
    return row.max() + np.log(np.exp(row - row.max()).sum())


def balance_loss(logits, idx, mask=None):
    """-> (counts [E+1], mean_prob [E], balance, z)"""
    T, E = logits.shape
    k = idx.shape[1]
    counts, prob, z = np.zeros(E + 1, np.int64), np.zeros(E), 0.0
    for t in range(T):
        if mask is not None and mask[t] == 0:
            continue
        counts[E] += 1
        for e in idx[t]:
            if 0 <= e < E:
                counts[e] += 1
        prob += _softmax(logits[t])
        z += _lse(logits[t]) ** 2
    n = counts[E]
    if n == 0:
        return counts, prob, 0.0, 0.0
    return counts, prob / n, E / (k * n) * float(counts[:E] @ (prob / n)), z / n


def gates(row, picked, renorm):
    """Gate weights of one token's picked experts, in the order they are given."""
    p = _softmax(row)[picked]
    return p / p.sum() if renorm else p


def route_backward(logits, idx, d_topk_w, mask, counts, coef_balance, coef_z, renorm):
    """d_logits [T,E]: the Jacobian of each token's gates, and that of the losses, written out."""
    T, E = logits.shape
    k = idx.shape[1]
    out = np.zeros((T, E))
    n = max(int(counts[E]), 1) if counts is not None else 1
    for t in range(T):
        inside = mask is None or mask[t] != 0
        if d_topk_w is not None:
            p = _softmax(logits[t])
            w = gates(logits[t], idx[t], renorm)
            for j in range(k):
                for i in range(k):      # d w_j / d logit of the i-th picked expert
                    own = 1.0 if i == j else 0.0
                    if renorm:
                        out[t, idx[t, i]] += d_topk_w[t, j] * w[j] * (own - w[i])
                    else:
                        out[t, idx[t, i]] += d_topk_w[t, j] * w[j] * own
                if not renorm:
                    out[t] -= d_topk_w[t, j] * w[j] * p
        if inside and counts is not None:
            p = _softmax(logits[t])
            g = coef_balance * E / (k * n) * counts[:E] / n
            out[t] += p * g - p * float(p @ g)
            out[t] += coef_z * 2.0 * _lse(logits[t]) / n * p
    return out


def router_backward(x, w_router, d_logits, dx_in=None):
    """-> (dx [T,H], d_w_router [H,E])"""
    dx = d_logits @ w_router.T
    return dx if dx_in is None else dx + dx_in, x.T @ d_logits


def combine_backward(dy, y_perm, slot_row, k, y_shared=None, x=None, w_shared_gate=None):
    """-> (d_topk_w [T,k], d_shared_gate [T] or None)"""
    T = dy.shape[0]
    out = np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            row = int(slot_row[t * k + j])
            if row >= 0:
                out[t, j] = dy[t] @ y_perm[row]
    if y_shared is None:
        return out, None
    gate = 1.0 / (1.0 + np.exp(-(x @ w_shared_gate)))
    return out, gate * (1.0 - gate) * np.einsum("th,th->t", dy, y_shared)
