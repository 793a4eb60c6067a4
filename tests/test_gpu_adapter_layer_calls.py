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


@pytest.mark.parametrize("T", [16, 200])
def test_a_forward_captured_alone_keeps_its_buffers(T):
    """Captured with torch.cuda.graph, not by layer.capture: a larger eager batch takes none of the graph's buffers away."""
    w = _weights()
    x, _, idx, _ = _batch(T)
    layer, eager = _layer(w), _layer(w)
    layer.forward(x, adapter_idx=idx)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = layer.forward(x, adapter_idx=idx)
    kept = {n: getattr(layer, n) for n in layer._BUFFERS if getattr(layer, n, None) is not None}
    big = _batch(T + 500)
    layer.forward(big[0], adapter_idx=big[2])
    for name, buffer in kept.items():
        assert getattr(layer, name) is buffer or any(buffer is r for r in layer._retired), name
    filler = [torch.full((1 << 20,), 1.0, device="cuda") for _ in range(8)]
    for seed in (1, 2, 3):
        new = _batch(T, seed)
        x.copy_(new[0]), idx.copy_(new[2])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager.forward(x, adapter_idx=idx))
    assert all(bool((f == 1).all()) for f in filler)


@pytest.mark.parametrize("T", [9, 200])
def test_the_modules_adapters_are_trained_beside_frozen_ones(T):
    """A layer that serves adapters of the shared expert's down projection too: all gradients but those, from the same ids."""
    w = _weights()
    x, dy, idx, mask = _batch(T)
    mask[0] = 1
    layer = _layer(w, down=True)
    layer.forward(x, adapter_idx=idx)
    with pytest.raises(ValueError):
        layer.backward(x, dy)                        # dx without the module's adapters would lack a part
    got = layer.backward(x, dy, idx, mask, 0.5, 0.25)
    ref, _, _ = _chain(layer, w, x, dy, idx, mask, 0.5, 0.25, True, True)
    _compare(got, ref, list(ref))
    only = layer.backward(x, dy, None, mask, need_dx=False)
    assert only.dx is None and only.adapter_a is None and only.w_router is not None


@pytest.mark.parametrize("overlap", [True, False])
@pytest.mark.parametrize("T", [5, 150])
def test_sliced_down_projections_adapters_add_up(T, overlap):
    """Two tensor-parallel shards: their columns of the down projection's A (112 of 224, padded to 128), whole B; half of the module's ranks."""
    w = _weights()
    x, _, idx, _ = _batch(T)
    want = _layer(w, down=True, out_f32=True, overlap_shared=overlap).forward(x, adapter_idx=idx).clone()
    without = _layer(w, out_f32=True, overlap_shared=overlap).forward(x, adapter_idx=idx)
    assert not torch.equal(without, want)
    total = sum(_layer(w, down=True, tp=2, p=p, out_f32=True, overlap_shared=overlap).forward(x, adapter_idx=idx).clone() for p in range(2))
    assert _rel(total, want) <= 1e-4        # as test_shards_add_up


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("T", [7, 160])
def test_a_step_on_a_stream_of_the_callers(T, given):
    """Forward, losses and backward with stream=: the same bits as on torch's current stream, which is busy meanwhile."""
    w = _weights()
    x, dy, idx, mask = _batch(T)
    logits = torch.randn(T, E, device="cuda") if given else None
    one, other = _layer(w, overlap_shared=False, max_tokens=T), _layer(w, overlap_shared=False, max_tokens=T)
    other._alloc_grad(T)
    other.logits.zero_()
    want = (one.forward(x, logits, adapter_idx=idx), *one.backward(x, dy, idx, mask, 0.5, 0.25), one.losses)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)
    got = (other.forward(x, logits, stream=stream, adapter_idx=idx), *other.backward(x, dy, idx, mask, 0.5, 0.25, stream=stream), other.losses)
    stream.synchronize()
    copies = []
    with torch.cuda.stream(stream):
        for t in got:
            copies.append(None if t is None else t.clone())
    torch.cuda.synchronize()
    for a, b in zip(copies, want):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
