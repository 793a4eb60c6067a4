"""How many bits of the narrow factors the bf16 results are made from.

Every result here is one product plus an addend that cancels the product's bf16 value, so that what is left shows the bits below it.

Tolerances, per element, of the product's size p.  v (or u before its scale) is one product of two bf16 numbers, exact; times the scale in
fp32 it is off by 2^-24 p.  Held in 24 bits it meets a bf16 number in three products, exact in fp32, that two additions join and a third adds
to the addend: 2^-23 p each if they are truncated.  4 2^-23 p in all, then half a step of the result, 2^-8 of it.  The router's
factors are both fp32: products of their parts below 2^-23 p together may be left out, and six of them are joined: 8 2^-23 p."""
import pytest
import torch

from paper_2508_19373_amd import binding as B

pytestmark = pytest.mark.gpu


def _normal(g, *shape):
    t = torch.randn(shape, generator=g, dtype=torch.float64)
    return t + torch.sign(t) * 0.25                          # away from zero, so that every product has its size


def _one_hot(g, T, n):
    """[T,n] with one value in each row, and its column."""
    at = torch.randint(0, n, (T,), generator=g)
    value = _normal(g, T).bfloat16()
    return torch.zeros((T, n), dtype=torch.bfloat16).scatter_(1, at[:, None], value[:, None]), at, value.double()


def _diagonal(m, rank):
    """Of each row of m [L][n][rank] the value in column row % rank."""
    keep = torch.arange(m.shape[1])[:, None] % rank == torch.arange(rank)
    return torch.where(keep, m, torch.zeros_like(m))


def _check(got, product, base, bits):
    got, ref = got.double().cpu(), product + base.double()
    bad = (got - ref).abs() > product.abs() * bits * 2.0 ** -23 + ref.abs() * 2.0 ** -8
    assert not bad.any(), (int(bad.sum()), bad.numel(), (got - ref)[bad][:4], product[bad][:4])


SIZES = [(1, 64, 264, 16, 2), (5, 2048, 512, 32, 3), (9, 4104, 520, 8, 2), (40, 72, 328, 64, 6), (64, 136, 264, 128, 5), (65, 1032, 264, 16, 3),
         (300, 264, 1032, 32, 4), (300, 520, 264, 64, 9), (200, 136, 520, 128, 4)]


@pytest.mark.parametrize("T,K,N,r,L", SIZES)
def test_adapters_result(T, K, N, r, L):
    print("case bits of y", T, K, N, r, L, flush=True)
    g = torch.Generator().manual_seed(T + r)
    x, at, value = _one_hot(g, T, K)
    a, b = _normal(g, L, r, K).bfloat16(), _diagonal(_normal(g, L, N, r).bfloat16(), r)
    scale, idx = (_normal(g, L).abs() + 0.5).float(), torch.randint(0, L, (T,), generator=g, dtype=torch.int32)
    i = idx.long()
    v = value[:, None] * a.double()[i, :, at]                                             # [T,r]
    product = scale.double()[i, None] * (v[:, None, :] * b.double()[i]).sum(2)            # [T,N], one term each
    base = (-product).bfloat16()
    d = [t.cuda() for t in (x, idx, a, b, scale, base)]
    y, ws = torch.empty_like(d[5]), torch.empty(B.moe_lora_workspace_bytes(T, K, N, r, L), dtype=torch.uint8, device="cuda")
    B.moe_lora_forward(d[0], d[1], T, K, N, r, L, *d[2:5], d[5], y, None, ws)
    _check(y, product, base, 4)


@pytest.mark.parametrize("T,K,N,r,L", SIZES)
def test_adapters_dx(T, K, N, r, L):
    print("case bits of dx", T, K, N, r, L, flush=True)
    g = torch.Generator().manual_seed(T + r + 1)
    dy, at, value = _one_hot(g, T, N)
    b, a = _normal(g, L, N, r).bfloat16(), _diagonal(_normal(g, L, K, r).bfloat16(), r).transpose(1, 2).contiguous()
    scale, idx = (_normal(g, L).abs() + 0.5).float(), torch.randint(0, L, (T,), generator=g, dtype=torch.int32)
    i = idx.long()
    u = scale.double()[i, None] * value[:, None] * b.double()[i, at]                      # [T,r]
    product = (u[:, :, None] * a.double()[i]).sum(1)                                      # [T,K], one term each
    base = (-product).bfloat16()
    d = [t.cuda() for t in (torch.zeros(T, K).bfloat16(), dy, idx, a, b, scale, torch.zeros(T, r), base)]
    dx, ga, gb = torch.empty_like(d[7]), torch.empty((L, r, K), device="cuda"), torch.empty((L, N, r), device="cuda")
    ws = torch.empty(B.moe_lora_workspace_bytes(T, K, N, r, L, True), dtype=torch.uint8, device="cuda")
    B.moe_lora_backward(*d[:3], T, K, N, r, L, *d[3:7], d[7], dx, ga, gb, ws)
    _check(dx, product, base, 4)


@pytest.mark.parametrize("T,H,E", [(1, 64, 1), (65, 520, 8), (300, 264, 20), (333, 2048, 60), (200, 1032, 64), (130, 520, 100), (65, 264, 200),
                                   (70, 136, 256), (2100, 1032, 100), (2500, 1032, 256)])
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
