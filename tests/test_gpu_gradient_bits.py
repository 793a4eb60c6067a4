"""How many bits of the narrow factors the bf16 results are made from.

Every result here is one product plus an addend that cancels the product's bf16 value, so that what is left shows the bits below it.

Tolerances, per element, of the product's size p.  The router's factors are both fp32: held in 24 bits, products of their parts below 2^-23 p
together may be left out, and six of them and the addend are joined, 2^-23 p each if an addition is truncated: 8 2^-23 p in all, then half a
step of the result, 2^-8 of it."""
import pytest
import torch

from paper_2508_19373_amd import binding as B

pytestmark = pytest.mark.gpu


def _normal(g, *shape):
    t = torch.randn(shape, generator=g, dtype=torch.float64)
    return t + torch.sign(t) * 0.25                          # away from zero, so that every product has its size


def _check(got, product, base, bits):
    got, ref = got.double().cpu(), product + base.double()
    bad = (got - ref).abs() > product.abs() * bits * 2.0 ** -23 + ref.abs() * 2.0 ** -8
    assert not bad.any(), (int(bad.sum()), bad.numel(), (got - ref)[bad][:4], product[bad][:4])


@pytest.mark.parametrize("T,H,E", [(1, 64, 1), (65, 520, 8), (300, 264, 20), (333, 2048, 60), (200, 1032, 64), (130, 520, 100), (65, 264, 200),
                                   (70, 136, 256)])
def test_routers_dx(T, H, E):
    print("case bits of the router's dx", T, H, E, flush=True)
    g = torch.Generator().manual_seed(T + E)
    at, value, w = torch.randint(0, E, (T,), generator=g), _normal(g, T).float(), _normal(g, H, E).float()
    d_logits = torch.zeros((T, E)).scatter_(1, at[:, None], value[:, None])
    product = value.double()[:, None] * w.double().T[at]
    base = (-product).bfloat16()
    d = [t.cuda() for t in (torch.zeros(T, H).bfloat16(), w, d_logits, base)]
    dx, dw = torch.empty_like(d[3]), torch.empty((H, E), device="cuda")
    ws = torch.empty(B.moe_router_backward_workspace_bytes(T, H, E), dtype=torch.uint8, device="cuda")
    B.moe_router_backward(*d[:3], T, H, E, d[3], dx, dw, ws)
    _check(dx, product, base, 8)
