"""The router's gradients where a formula that is right on paper loses its digits."""
import numpy as np
import pytest
import torch

import test_gpu_router_grad as whole
from paper_2508_19373_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_shared_gate_far_from_its_middle(sign, bf16):
    """The gate's logits are 8 to 60 on one side.  g (1 - g) follows its logit z with a relative slope of 1 at most: the relative error is
    that of z, a sum of H products of one sign, (H + 8) 2^-23 |z|, that of the products with y_shared, (H + 8) 2^-23 of their absolute
    sum, and 2^-20 for the exponential and what is made of it."""
    T, H, k = 53, 64, 2
    g = torch.Generator().manual_seed(4)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = (torch.rand((T, H), generator=g) + 0.5).bfloat16()
    w = torch.rand(H, generator=g) + 0.5
    z = torch.linspace(8.0, 60.0, T).double()
    x = (x.double() * (z / (x.double() @ w.double()))[:, None] * sign).bfloat16()
    dy, ys, y = torch.randn((T, H), generator=g).bfloat16(), torch.randn((T, H), generator=g).to(dt), torch.zeros((T * k, H), dtype=dt)
    d = [t.cuda() for t in (dy, y, torch.arange(T * k, dtype=torch.int32), ys, x, w)]
    dw, dg = torch.empty((T, k), device="cuda"), torch.empty(T, device="cuda")
    B.moe_combine_backward(d[0], d[1], d[2], T, k, H, *d[3:], dw, dg, B.MOE_Y_PERM_BF16 if bf16 else 0)
    z = (x.double() @ w.double()).numpy()
    slope = np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))) ** 2
    terms = (dy.double() * ys.double()).numpy()
    bound = slope * np.abs(terms).sum(1) * ((H + 8) * 2.0 ** -23 * (1 + np.abs(z)) + 2.0 ** -20)
    assert (np.abs(dg.double().cpu().numpy() - slope * terms.sum(1)) <= bound).all()


@pytest.mark.parametrize("T,E", [(1, 1), (70, 8), (300, 16), (65, 33), (200, 60), (3000, 64), (40, 130), (33, 256)])
def test_one_renormalised_gate_has_no_gradient(T, E):
    """A gate that is divided by itself is 1 whatever the logits are: its gradient is 0, not the last places of the one it is given."""
    g = torch.Generator().manual_seed(T + E)
    logits, dw = (torch.randn((T, E), generator=g) * 3).cuda(), (torch.randn((T, 1), generator=g) * 100).cuda()
    idx = logits.argmax(1, keepdim=True).int()
    d = torch.full((T, E), float("nan"), device="cuda")
    B.moe_route_backward(logits, idx, dw, None, None, T, E, 1, 0.0, 0.0, B.MOE_RENORM_TOPK, d)
    assert not d.any()


@pytest.mark.parametrize("T,E,k", [(130, 8, 2), (2000, 60, 4), (90, 200, 8)])
def test_data_parallel_devices_sum_their_counts(T, E, k):
    """Two devices' batches with the sums of their counts: row by row the gradients of the whole batch, bit for bit."""
    g = torch.Generator().manual_seed(T)
    logits, dw = torch.randn((T, E), generator=g).cuda(), torch.randn((T, k), generator=g).cuda()
    idx, mask = logits.topk(k, dim=1).indices.int().contiguous(), (torch.rand(T, generator=g) < 0.7).to(torch.uint8).cuda()
    ws = torch.empty(B.moe_balance_workspace_bytes(T, E), dtype=torch.uint8, device="cuda")

    def counted(rows):
        counts, prob, losses = torch.empty(E + 1, dtype=torch.int32, device="cuda"), torch.empty(E, device="cuda"), torch.empty(2, device="cuda")
        B.moe_balance_loss(logits[rows], idx[rows], mask[rows], rows.stop - rows.start, E, k, counts, prob, losses, ws)
        return counts

    def gradient(rows, counts):
        d = torch.full((rows.stop - rows.start, E), float("nan"), device="cuda")
        B.moe_route_backward(logits[rows], idx[rows], dw[rows], mask[rows], counts, rows.stop - rows.start, E, k, 0.5, 0.25, 0, d)
        return d
    cut = T // 3
    parts, whole = [slice(0, cut), slice(cut, T)], slice(0, T)
    total = counted(parts[0]) + counted(parts[1])
    assert torch.equal(total, counted(whole)) and int(total[E]) == int(mask.sum())
    assert torch.equal(torch.cat([gradient(p, total) for p in parts]), gradient(whole, total))


@pytest.mark.parametrize("T,H,E", [(2, 262144, 8), (70, 262144, 64), (65, 262144, 1), (33, 8, 256)])
def test_routers_product_at_the_limits(T, H, E):
    whole.test_router_backward(T, H, E)


@pytest.mark.parametrize("T,H,k,bf16,shared", [(2, 262144, 16, False, True), (3, 262144, 1, True, True)])
def test_combines_gates_at_the_limits(T, H, k, bf16, shared):
    whole.test_combine_backward(T, H, k, bf16, shared)
