"""What a layer keeps for a captured forward, and what it refuses while a graph is being captured; on the host, where the
calls into the library end at their first look at a tensor."""
import pytest
import torch

from paper_2508_19373_amd.layer import ExpertShardLayer

H, L, R = 64, 3, 8


def _layer(**kw):
    w = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    return ExpertShardLayer(n_experts=2, top_k=1, hidden=H, inter_full=64, inter_slice=64, w_gate=w(2, 64, H), w_up=w(2, 64, H),
                            w_down=w(2, H, 64), adapters=(w(L, R, H), w(L, H, R), torch.ones(L)), overlap_shared=False, device="cpu", **kw)


def _x(T):
    return torch.zeros((T, H), dtype=torch.bfloat16), torch.zeros(T, dtype=torch.int32)


def test_a_forward_that_is_captured_directly_keeps_its_buffers(monkeypatch):
    layer = _layer(max_tokens=4)
    kept = [layer.lora_v, layer.lora_ws, layer.y_out, layer.ffn_ws]
    x, idx = _x(4)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(ValueError):
        layer.forward(x, adapter_idx=idx)
    monkeypatch.undo()
    layer._alloc(100)
    assert all(any(t is r for r in layer._retired) for t in kept)


def test_no_workspace_grows_inside_a_capture(monkeypatch):
    layer = _layer(max_tokens=4)
    x, idx = _x(4)
    layer.lora_ws = small = layer.lora_ws[:16]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError):
        layer.forward(x, adapter_idx=idx)
    assert layer.lora_ws is small


def test_given_logits_are_copied_on_the_callers_stream(monkeypatch):
    """Not on torch's current one, beside which the caller's would read them half written."""
    layer, used = _layer(max_tokens=4), []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            used.append(self.stream)

        def __exit__(self, *_):
            used.append(None)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "stream", On)
    stream = object()
    with pytest.raises(ValueError):
        layer.forward(_x(4)[0], torch.ones(4, 2), stream=stream)
    assert used == [stream, None] and bool((layer.logits[:4] == 1).all())
