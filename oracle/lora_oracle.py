"""CPU oracle for low-rank adapters of many requests beside one projection.

TEST INFRASTRUCTURE ONLY: the plain definition in float64, row by row, from exactly converted inputs; shares no code with
the HIP library.  Pins (tests/test_lora_oracle_pins.py): the dense update x (A^T B^T) of one adapter; shard sums; the
gradients against central differences.
"""
from __future__ import annotations

import numpy as np


def forward(x, idx, a, b, scale, y_in=None):
    """x [T,K], idx [T], a [L,r,K], b [L,N,r], scale [L], y_in [T,N] or None -> (y_out [T,N], v [T,r])."""
    T, L, r, N = x.shape[0], a.shape[0], a.shape[1], b.shape[1]
    y = np.zeros((T, N)) if y_in is None else np.array(y_in, np.float64)
    v = np.zeros((T, r))
    for t in range(T):
        i = int(idx[t])
        if 0 <= i < L:
            v[t] = a[i] @ x[t]
            y[t] += scale[i] * (b[i] @ v[t])
    return y, v


def backward(x, dy, idx, a, b, scale, v, dx_in=None):
    """-> (dx [T,K], grad_a [L,r,K], grad_b [L,N,r])"""
    T, L = x.shape[0], a.shape[0]
    dx = np.zeros(x.shape) if dx_in is None else np.array(dx_in, np.float64)
    grad_a, grad_b = np.zeros(a.shape), np.zeros(b.shape)
    for t in range(T):
        i = int(idx[t])
        if 0 <= i < L:
            u = scale[i] * (b[i].T @ dy[t])
            dx[t] += a[i].T @ u
            grad_a[i] += np.outer(u, x[t])
            grad_b[i] += scale[i] * np.outer(dy[t], v[t])
    return dx, grad_a, grad_b
