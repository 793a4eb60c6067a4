"""Which ids a backward pass takes after which forward, before anything reaches the device."""
import pytest
import torch

from test_adapter_layer_boundary import H, S, _ad, _layer


@pytest.mark.parametrize("both", [False, True])
def test_dx_needs_the_ids_of_the_forward(both):
    x = torch.zeros((4, H), dtype=torch.bfloat16)
    layer = _layer(shared=both, adapters=_ad(H), shared_adapters=_ad(S) if both else None)
    layer._last_T, layer._has_v = 4, True
    with pytest.raises(ValueError, match="adapter_idx"):
        layer.backward(x, x)
    with pytest.raises(ValueError, match="device tensor"):      # accepted: the first call into the library looks at the tensors
        layer.backward(x, x, need_dx=False)
    with pytest.raises(ValueError, match="device tensor"):
        layer.backward(x, x, torch.zeros(4, dtype=torch.int32))
    layer._has_v = False
    with pytest.raises(ValueError, match="device tensor"):
        layer.backward(x, x)
    with pytest.raises(ValueError, match="without"):
        layer.backward(x, x, torch.zeros(4, dtype=torch.int32))
