"""Pins of the router losses' and gradients' oracle: closed forms and differences."""
import numpy as np
import pytest

from oracle import moe_oracle as M
from oracle import router_grad_oracle as O


def _routing(seed, T, E, k, renorm=False):
    g = np.random.default_rng(seed)
    logits = g.standard_normal((T, E)) * 1.3
    idx, _, _ = M.route_topk(logits.astype(np.float32), k, renorm)
    return logits.astype(np.float32).astype(np.float64), idx, g


def test_even_routing_has_balance_loss_one():
    E, k = 8, 2
    idx = np.array([[(2 * t) % E, (2 * t + 1) % E] for t in range(16)])
    counts, prob, balance, z = O.balance_loss(np.zeros((16, E)), idx)
    assert list(counts) == [4] * 8 + [16] and np.allclose(prob, 1 / E)
    assert abs(balance - 1.0) < 1e-15 and abs(z - np.log(E) ** 2) < 1e-14


def test_one_expert_for_all_has_balance_loss_e_over_k():
    E = 6
    logits = np.full((5, E), -1e30)
    logits[:, 3] = 2.0
    counts, prob, balance, z = O.balance_loss(logits, np.full((5, 1), 3))
    assert counts[3] == 5 and abs(balance - E) < 1e-12 and abs(z - 4.0) < 1e-12


def test_masked_tokens_are_as_if_they_were_not_there():
    logits, idx, _ = _routing(1, 20, 7, 3)
    mask = (np.arange(20) % 3 != 0).astype(np.uint8)
    some = O.balance_loss(np.where(mask[:, None] != 0, logits, np.nan), idx, mask)
    kept = O.balance_loss(logits[mask != 0], idx[mask != 0])
    assert np.array_equal(some[0], kept[0]) and np.allclose(some[1], kept[1]) and np.allclose(some[2:], kept[2:])
    nobody = O.balance_loss(logits, idx, np.zeros(20))
    assert not nobody[0].any() and not nobody[1].any() and nobody[2:] == (0.0, 0.0)


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("masked", [False, True])
def test_logit_gradient_against_differences(renorm, masked):
    T, E, k, cb, cz = 6, 7, 3, 0.7, 0.3
    logits, idx, g = _routing(2, T, E, k, renorm)
    mask = np.array([1, 1, 0, 1, 0, 1], np.uint8) if masked else None
    dw = g.standard_normal((T, k))
    counts = O.balance_loss(logits, idx, mask)[0]

    def objective(l):
        _, _, balance, z = O.balance_loss(l, idx, mask)
        return cb * balance + cz * z + sum(float(O.gates(l[t], idx[t], renorm) @ dw[t]) for t in range(T))

    grad = O.route_backward(logits, idx, dw, mask, counts, cb, cz, renorm)
    for t in range(T):
        for e in range(E):
            up, down = logits.copy(), logits.copy()
            up[t, e] += 1e-5
            down[t, e] -= 1e-5
            assert abs((objective(up) - objective(down)) / 2e-5 - grad[t, e]) < 1e-8


def test_product_and_gate_gradients_against_differences():
    g = np.random.default_rng(3)
    T, H, E, k = 5, 8, 4, 2
    x, w, dl = g.standard_normal((T, H)), g.standard_normal((H, E)), g.standard_normal((T, E))
    dx, dw = O.router_backward(x, w, dl)
    for i in range(H):
        step = np.zeros((H,))
        step[i] = 1e-4
        assert np.allclose((((x + step) @ w - (x - step) @ w) * dl).sum(1) / 2e-4, dx[:, i], atol=1e-9)
        up, down = w.copy(), w.copy()
        up[i, 1] += 1e-4
        down[i, 1] -= 1e-4
        assert abs((((x @ up) - (x @ down)) * dl).sum() / 2e-4 - dw[i, 1]) < 1e-9
    # the combine's gates: y is linear in topk_w, and sigmoid(x.w_s) scales the shared expert
    y_perm, slot = g.standard_normal((T * k, H)), np.arange(T * k)
    slot[3] = -1
    y_shared, ws, dy = g.standard_normal((T, H)), g.standard_normal(H), g.standard_normal((T, H))
    topk_w = g.uniform(0.1, 0.5, (T, k))
    d_topk, d_gate = O.combine_backward(dy, y_perm, slot, k, y_shared, x, ws)

    def loss(wts, z):
        y = np.zeros((T, H))
        for t in range(T):
            for j in range(k):
                if slot[t * k + j] >= 0:
                    y[t] += wts[t, j] * y_perm[slot[t * k + j]]
            y[t] += y_shared[t] / (1.0 + np.exp(-z[t]))
        return float((y * dy).sum())

    z = x @ ws
    for t in range(T):
        for j in range(k):
            up, down = topk_w.copy(), topk_w.copy()
            up[t, j] += 1e-4
            down[t, j] -= 1e-4
            assert abs((loss(up, z) - loss(down, z)) / 2e-4 - d_topk[t, j]) < 1e-8
        up, down = z.copy(), z.copy()
        up[t] += 1e-5
        down[t] -= 1e-5
        assert abs((loss(topk_w, up) - loss(topk_w, down)) / 2e-5 - d_gate[t]) < 1e-7
