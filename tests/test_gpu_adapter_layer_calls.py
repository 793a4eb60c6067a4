"""Calls of a layer's forward and backward in other orders than a plain training step's.  Tolerances and the float64 chain are those of
test_gpu_adapter_layer.py."""
import pytest
import torch

from test_gpu_adapter_layer import DX, FP32, H, E, _batch, _chain, _layer, _rel, _weights

pytestmark = pytest.mark.gpu


def _compare(got, ref, names):
    for name in names:
        err = _rel(getattr(got, name), ref[name])
        print(name, err, flush=True)
        assert err <= (DX if name == "dx" else FP32), (name, err)


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("T", [3, 130])
def test_gradients_after_a_forward_of_given_logits(T, shared):
    """Such a forward does not read the router's weights: they have no gradient and dx has no part through them."""
    w = _weights()
    x, dy, idx, mask = _batch(T)
    mask[0] = 1
    layer = _layer(w, shared=shared)
    layer.forward(x, torch.randn(T, E, device="cuda"), adapter_idx=idx)
    got = layer.backward(x, dy, idx, mask, 0.5, 0.25)
    ref, _, _ = _chain(layer, {**w, "router": torch.zeros_like(w["router"])}, x, dy, idx, mask, 0.5, 0.25, shared, True)
    assert got.w_router is None
    _compare(got, ref, ["dx", "logits", "adapter_a", "adapter_b"] + ["w_shared_gate"] * shared)
    layer.forward(x, adapter_idx=idx)                # its own logits again
    got = layer.backward(x, dy, idx, mask, 0.5, 0.25)
    ref, _, _ = _chain(layer, w, x, dy, idx, mask, 0.5, 0.25, shared, True)
    _compare(got, ref, ["dx", "logits", "w_router"])


def test_dx_after_given_logits_where_nothing_else_reads_x():
    w = _weights()
    x, dy, _, _ = _batch(20)
    layer = _layer(w, shared=False, adapters=False)
    layer.forward(x, torch.randn(20, E, device="cuda"))
    assert layer.backward(x, dy).dx is None
    more = torch.randn(20, H, device="cuda").bfloat16()
    assert torch.equal(layer.backward(x, dy, dx_in=more).dx, more)
