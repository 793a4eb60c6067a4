"""What a layer with adapters refuses, before anything reaches the device."""
import pytest
import torch

from paper_2508_19373_amd.layer import ExpertShardLayer

H, I, S, L, R = 64, 64, 96, 3, 8


def _ad(K, N=H, L=L, r=R, dtype=torch.bfloat16, scales=None):
    return (torch.zeros((L, r, K), dtype=dtype), torch.zeros((L, N, r), dtype=dtype), torch.ones(scales or L))


def _layer(shared=False, **kw):
    w = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    return ExpertShardLayer(n_experts=2, top_k=1, hidden=H, inter_full=I, inter_slice=I, w_gate=w(2, I, H), w_up=w(2, I, H),
                            w_down=w(2, H, I), shared=(w(1, S, H), w(1, S, H), w(1, H, S)) if shared else None,
                            inter_shared_full=S, inter_shared_slice=S, overlap_shared=False, device="cpu", **kw)


@pytest.mark.parametrize("given", [_ad(H + 8), _ad(H, N=H + 8), _ad(H, dtype=torch.float32), _ad(H, r=12), _ad(H, r=136),
                                   _ad(H, L=257), _ad(H, scales=2), (_ad(H)[0], _ad(H)[1], torch.ones(L, dtype=torch.float64))])
def test_adapters_of_other_shapes_and_types(given):
    with pytest.raises(ValueError):
        _layer(adapters=given)


def test_adapters_of_a_shared_expert():
    with pytest.raises(ValueError):
        _layer(shared_adapters=_ad(S))
    with pytest.raises(ValueError):
        _layer(shared=True, shared_adapters=_ad(H))
    layer = _layer(shared=True, shared_adapters=(torch.ones((L, R, S), dtype=torch.bfloat16), *_ad(S)[1:]))
    a = layer.shared_adapters.a      # padded with zeros as the slice is
    assert a.shape == (L, R, 128) and bool((a[:, :, :S] == 1).all()) and not bool(a[:, :, S:].any())


def test_forward_arguments():
    x, idx = torch.zeros((4, H), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        _layer().forward(x, adapter_idx=idx)
    for wrong in (idx.long(), idx[:3], idx[:, None]):
        with pytest.raises(ValueError):
            _layer(adapters=_ad(H)).forward(x, adapter_idx=wrong)


def test_backward_and_loss_arguments():
    x, idx = torch.zeros((4, H), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    layer, both = _layer(adapters=_ad(H)), _layer(shared=True, adapters=_ad(H), shared_adapters=_ad(S))
    for one in (layer, both):
        with pytest.raises(RuntimeError):
            one.backward(x, x)
        with pytest.raises(RuntimeError):
            one.router_losses()
        one._last_T = 4
    with pytest.raises(ValueError):      # the last forward was without ids
        layer.backward(x, x, idx)
    layer._has_v = both._has_v = True
    for wrong in (dict(dy=x.float()), dict(dy=x[:3]), dict(x=x[:, :32]), dict(adapter_idx=idx.long()), dict(adapter_idx=idx[:2]),
                  dict(dx_in=x.float()), dict(dx_in=x[:2]), dict(dx_in=x, need_dx=False),
                  dict(token_mask=torch.ones(4)),
                  dict(token_mask=torch.ones(5, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            layer.backward(**{**dict(x=x, dy=x), **wrong})
    with pytest.raises(ValueError):
        both.backward(x, x, idx)
    with pytest.raises(ValueError):
        layer.router_losses(torch.ones(4))
    with pytest.raises(ValueError):
        layer.router_losses(torch.ones(3, dtype=torch.uint8))
    plain = _layer()
    plain._last_T = 4
    with pytest.raises(ValueError):
        plain.backward(x, x, idx)
