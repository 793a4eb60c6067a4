"""Pins of the adapters' oracle: dense updates, shard sums, differences."""
import numpy as np
import pytest

from oracle import lora_oracle as O


def _case(seed=0, T=9, K=16, N=24, r=8, L=3):
    g = np.random.default_rng(seed)
    idx = np.array([0, 2, -1, 1, 2, L, 0, 1, -5][:T])
    return dict(x=g.standard_normal((T, K)), idx=idx, a=g.standard_normal((L, r, K)), b=g.standard_normal((L, N, r)),
                scale=g.uniform(0.5, 2.0, L)), g


def test_one_adapter_is_the_dense_update():
    c, g = _case()
    c["idx"] = np.full(9, 1)
    y_in = g.standard_normal((9, 24))
    y, v = O.forward(**c, y_in=y_in)
    assert np.allclose(y, y_in + c["scale"][1] * c["x"] @ (c["b"][1] @ c["a"][1]).T, atol=1e-12)
    assert np.allclose(v, c["x"] @ c["a"][1].T, atol=1e-12)


def test_rows_without_an_adapter_stay():
    c, g = _case()
    y_in = g.standard_normal((9, 24))
    c["x"][[2, 5, 8]] = np.nan
    y, v = O.forward(**c, y_in=y_in)
    assert np.array_equal(y[[2, 5, 8]], y_in[[2, 5, 8]]) and not v[[2, 5, 8]].any() and np.isfinite(y).all()


def test_slices_of_the_input_and_of_the_rank_add_up():
    c, _ = _case()
    whole, _ = O.forward(**c)
    by_k = sum(O.forward(**{**c, "x": c["x"][:, s], "a": c["a"][:, :, s]})[0] for s in (slice(0, 8), slice(8, 16)))
    by_r = sum(O.forward(**{**c, "a": c["a"][:, s], "b": c["b"][:, :, s]})[0] for s in (slice(0, 4), slice(4, 8)))
    assert np.allclose(whole, by_k, atol=1e-12) and np.allclose(whole, by_r, atol=1e-12)


@pytest.mark.parametrize("what", ["x", "a", "b"])
def test_gradients_against_differences(what):
    c, g = _case()
    dy = g.standard_normal((9, 24))
    _, v = O.forward(**c)
    grad = dict(zip(("x", "a", "b"), O.backward(c["x"], dy, c["idx"], c["a"], c["b"], c["scale"], v)))[what]
    for _ in range(12):
        at = tuple(g.integers(0, n) for n in c[what].shape)
        h = 1e-4
        up, down = ({**c, what: c[what].copy()} for _ in range(2))
        up[what][at] += h
        down[what][at] -= h
        d = ((O.forward(**up)[0] - O.forward(**down)[0]) * dy).sum() / (2 * h)   # bilinear: exact to rounding
        assert abs(d - grad[at]) < 1e-8 * max(1.0, abs(d))
