"""The layer's adapters, losses and backward pass as they are used together, against a float64 chain of torch operations.

Tolerances.  The reference takes the device's logits and experts' outputs as they are (their own tests are elsewhere), so what differs
are the sums of the backward pass.  fp32 gradients: sums of 512 fp32 products, off by sqrt(520) 2^-23 = 2.7e-6 of their terms' norm if
the errors are independent; three such sums follow one another, and the differences between gates cancel, a factor of ten at these sizes: rel-L2
1e-4.  The bf16 dx is rounded after each of the three branches, half a step of 2^-8 each and two parts of 8 bits before: rel-L2 3 2^-8.  An fp32
output with adapters: 3 parts of 8 bits of v and sums of 512 + 16: rel-L2 1e-5 of the update (as in the adapters' own tests)."""
import numpy as np
import pytest
import torch

from guards import Guards
from paper_2508_19373_amd.binding import MoeError
from paper_2508_19373_amd.layer import ExpertShardLayer

pytestmark = pytest.mark.gpu

H, E, K, I, S, L, R = 512, 8, 2, 256, 224, 3, 16
FP32, DX = 1e-4, 3 * 2.0 ** -8


def _weights(seed=3):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, by=1.0: torch.randn(s, generator=g) * by  # noqa: E731
    w = dict(gate=n(E, I, H, by=H ** -0.5), up=n(E, I, H, by=H ** -0.5), down=n(E, H, I, by=I ** -0.5), sg=n(1, S, H, by=H ** -0.5),
             su=n(1, S, H, by=H ** -0.5), sd=n(1, H, S, by=S ** -0.5), a=n(L, R, H, by=H ** -0.5), b=n(L, H, R, by=R ** -0.5),
             sa=n(L, R, S, by=S ** -0.5), sb=n(L, H, R, by=R ** -0.5))
    w = {k: v.bfloat16().cuda() for k, v in w.items()}
    w.update(router=n(H, E, by=H ** -0.5).cuda(), wsg=n(H, by=H ** -0.5).cuda(), scale=torch.tensor([0.5, 1.0, 2.0]).cuda())
    return w


def _layer(w, *, shared=True, renorm=True, adapters=True, down=False, tp=1, p=0, ep=1, q=0, **kw):
    n, i, s, r = E // ep, I // tp, S // tp, R // tp
    es, cs, ss, rs = slice(q * n, q * n + n), slice(p * i, p * i + i), slice(p * s, p * s + s), slice(p * r, p * r + r)
    c = lambda t: t.contiguous()  # noqa: E731
    shared = shared and q == 0
    return ExpertShardLayer(
        n_experts=E, top_k=K, hidden=H, inter_full=I, inter_slice=i, n_local_experts=n, expert_offset=q * n, renorm=renorm,
        w_router=w["router"], w_gate=c(w["gate"][es, cs]), w_up=c(w["up"][es, cs]), w_down=c(w["down"][es, :, cs]),
        shared=(c(w["sg"][:, ss]), c(w["su"][:, ss]), c(w["sd"][:, :, ss])) if shared else None,
        w_shared_gate=w["wsg"] if shared else None, inter_shared_full=S, inter_shared_slice=s,
        adapters=(c(w["a"][:, rs]), c(w["b"][:, :, rs]), w["scale"]) if adapters and q == 0 else None,
        shared_adapters=(c(w["sa"][:, :, ss]), w["sb"], w["scale"]) if down and shared else None, **kw)


def _batch(T, seed=1):
    g = torch.Generator().manual_seed(seed)
    x, dy = (torch.randn((T, H), generator=g).bfloat16().cuda() for _ in range(2))
    idx = torch.randint(-1, L + 1, (T,), generator=g, dtype=torch.int32).cuda()
    mask = (torch.rand(T, generator=g) < 0.8).to(torch.uint8).cuda()
    return x, dy, idx, mask


def _rel(got, ref):
    got, ref = got.double().cpu(), ref.double().cpu()
    return float((got - ref).norm() / ref.norm().clamp_min(1e-30))


def _update(x, idx, a, b, scale):
    """scale_i B_i A_i x of each row in float64, on the CPU."""
    x, a, b, scale = (t.double().cpu() for t in (x, a, b, scale))
    y = torch.zeros(x.shape[0], b.shape[1], dtype=torch.float64)
    for t, i in enumerate(idx.tolist()):
        if 0 <= i < a.shape[0]:
            y[t] = scale[i] * (b[i] @ (a[i] @ x[t]))
    return y


@pytest.mark.parametrize("overlap", [True, False])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("T", [1, 7, 64, 65, 300])
def test_forward_with_adapters(T, bf16, overlap):
    w = _weights()
    x, _, idx, _ = _batch(T)
    plain = _layer(w, adapters=False, out_f32=True, y_perm_bf16=bf16, overlap_shared=overlap)
    y0 = plain.forward(x).clone()
    layer = _layer(w, down=True, out_f32=True, y_perm_bf16=bf16, overlap_shared=overlap, max_tokens=T)
    guards = Guards().wrap_layer(layer)
    assert torch.equal(layer.forward(x), y0)     # without ids: the layer without adapters, bit for bit
    y = layer.forward(x, adapter_idx=idx).clone()
    guards.check()
    h = layer.h_sh[:T]
    f = lambda t: t.double().cpu()  # noqa: E731
    g, u = f(x) @ f(w["sg"][0]).T, f(x) @ f(w["su"][0]).T
    hr = g / (1 + torch.exp(-g)) * u
    assert bool(((f(h)[:, :S] - hr).abs() <= 2.0 ** -7 * hr.abs() + 1e-4).all())
    gate = torch.sigmoid(f(x) @ f(w["wsg"]))[:, None]
    update = _update(x, idx, w["a"], w["b"], w["scale"]) + gate * _update(h[:, :S], idx, w["sa"], w["sb"], w["scale"])
    has = ((idx >= 0) & (idx < L)).cpu()
    assert torch.equal(y[~has.cuda()], y0[~has.cuda()])
    if bool(has.any()):
        # y_shared is rounded once more where it is bf16: half a step of it and of the layer's without
        tol = 1e-5 * 2 + (2 * 2.0 ** -8 if bf16 else 0)
        d = (y - y0).double().cpu()
        size = float(update.norm()) + float(y0.double().norm())     # (y itself is rounded to fp32)
        assert float((d - update).norm()) <= tol * size
        if not bf16:
            assert float((d - update)[has].abs().max()) <= 2e-5 * (1 + float(y0.abs().max()) + float(update.abs().max()))


def _chain(layer, w, x, dy, idx, mask, cb, cz, shared, renorm):
    """float64 gradients; the values of the logits and of the experts' outputs are the device's."""
    T = x.shape[0]
    leaf = lambda t: t.double().cpu().requires_grad_(True)  # noqa: E731
    xd, wr, ws, a, b = leaf(x), leaf(w["router"]), leaf(w["wsg"]), leaf(w["a"]), leaf(w["b"])
    dyd, scale, idx, mask = dy.double().cpu(), w["scale"].double().cpu(), idx.cpu(), mask.cpu().bool()
    prod = xd @ wr
    logits = layer.logits[:T].double().cpu() + (prod - prod.detach())
    logits.retain_grad()
    prob = torch.softmax(logits, 1)
    topk = layer.topk_idx[:T].cpu().long()
    gates = prob.gather(1, topk)
    if renorm:
        gates = gates / gates.sum(1, keepdim=True)
    slot = layer.slot_row[:T * K].cpu().long()
    rows = layer.y_perm.double().cpu()[slot.clamp_min(0)] * (slot >= 0)[:, None]
    y = (gates.reshape(-1, 1) * rows).view(T, K, H).sum(1)
    if shared:
        y = y + torch.sigmoid(xd @ ws)[:, None] * layer.y_shared[:T].double().cpu()
    y = y + torch.stack([scale[i] * (b[i] @ (a[i] @ xd[t])) if 0 <= i < L else torch.zeros(H, dtype=torch.float64)
                         for t, i in enumerate(idx.tolist())])
    loss = (y * dyd).sum()
    counts = torch.zeros(E, dtype=torch.float64)
    for row in topk[mask]:
        counts[row] += 1
    n = max(int(mask.sum()), 1)
    balance = E / (K * n) * (counts * prob[mask].sum(0) / n).sum()
    z = (torch.logsumexp(logits[mask], 1) ** 2).sum() / n
    (loss + cb * balance + cz * z).backward()
    return dict(dx=xd.grad, logits=logits.grad, w_router=wr.grad, w_shared_gate=ws.grad, adapter_a=a.grad, adapter_b=b.grad), balance, z


@pytest.mark.parametrize("shared,renorm,bf16", [(True, True, False), (True, False, True), (False, False, False), (False, True, True)])
@pytest.mark.parametrize("T", [1, 65, 333])
def test_backward(T, shared, renorm, bf16):
    w = _weights()
    x, dy, idx, mask = _batch(T, seed=T)
    mask[0] = 1
    layer = _layer(w, shared=shared, renorm=renorm, y_perm_bf16=bf16, max_tokens=T)
    layer.forward(x, adapter_idx=idx)
    layer._alloc_grad(T)
    for name in layer._GRAD_BUFFERS:
        getattr(layer, name).view(torch.uint8).fill_(255)
    got = layer.backward(x, dy, idx, mask, 0.5, 0.25)
    ref, balance, z = _chain(layer, w, x, dy, idx, mask, 0.5, 0.25, shared, renorm)
    assert np.allclose(layer.losses.cpu().numpy(), [float(balance.detach()), float(z.detach())], rtol=1e-5)
    for name, value in got._asdict().items():
        if name == "w_shared_gate" and not shared:
            assert value is None
            continue
        err = _rel(value, ref[name])
        print("T", T, name, err, flush=True)
        assert err <= (DX if name == "dx" else FP32), (name, err)
    only = layer.backward(x, dy, None, mask, need_dx=False)
    assert only.dx is None and only.adapter_a is None
    ref, _, _ = _chain(layer, w, x, dy, idx, mask, 0.0, 0.0, shared, renorm)
    assert _rel(only.w_router, ref["w_router"]) <= FP32


def test_dx_in_is_added():
    w = _weights()
    x, dy, idx, mask = _batch(70)
    layer = _layer(w)
    layer.forward(x, adapter_idx=idx)
    alone = layer.backward(x, dy, idx).dx.clone()
    more = torch.randn(70, H, device="cuda").bfloat16()
    both = layer.backward(x, dy, idx, dx_in=more).dx
    # each side is rounded three times
    assert float((both.float() - alone.float() - more.float()).norm()) <= DX * float(alone.float().norm() + both.float().norm())


def test_shards_add_up():
    """Two slices of the experts' columns by two halves of the experts: outputs and gradients are the unsharded layer's."""
    w = _weights()
    x, dy, idx, mask = _batch(130)
    full = _layer(w, out_f32=True)
    y = full.forward(x, adapter_idx=idx).clone()
    want = {k: v.clone() for k, v in full.backward(x, dy, idx, mask, 0.5, 0.25)._asdict().items()}
    total, grads = torch.zeros_like(y), {}
    parts = {"adapter_a": [], "adapter_b": []}
    for q in range(2):
        for p in range(2):
            layer = _layer(w, tp=2, p=p, ep=2, q=q, out_f32=True)
            ids = idx if q == 0 else None
            total += layer.forward(x, adapter_idx=ids)
            once = 1.0 if p == q == 0 else 0.0
            for name, value in layer.backward(x, dy, ids, mask, 0.5 * once, 0.25 * once)._asdict().items():
                if name in parts:
                    if q == 0:
                        parts[name].append(value.clone())
                elif value is not None:
                    grads[name] = grads.get(name, 0) + value.float()
    grads.update(adapter_a=torch.cat(parts["adapter_a"], 1), adapter_b=torch.cat(parts["adapter_b"], 2))
    assert _rel(total, y) <= 1e-4
    for name, value in want.items():
        assert _rel(grads[name], value) <= (4 * DX if name == "dx" else FP32), name     # (dx is rounded by each shard)


@pytest.mark.parametrize("T", [16, 200])
def test_a_captured_step_on_other_ids(T):
    """Forward, losses and backward in one graph; ids, rows and gradients are written in place between the replays."""
    w = _weights()
    x, dy, idx, mask = _batch(T)
    layer, eager = _layer(w, down=False), _layer(w, down=False)

    def step(one, *b):
        y = one.forward(b[0], adapter_idx=b[2])
        return (y, *one.backward(*b, 0.5, 0.25), one.losses)
    step(layer, x, dy, idx, mask)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step(layer, x, dy, idx, mask)
    for seed in (1, 2, 3, 4):
        new = _batch(T, seed)
        for old, value in zip((x, dy, idx, mask), new):
            old.copy_(value)
        graph.replay()
        want = step(eager, *new)
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
    step(layer, *_batch(T + 300))       # the layer allocates anew: the graph keeps its own buffers
    filler = torch.full((1 << 22,), 1.0, device="cuda")
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, want):
        assert torch.equal(a, b)
    assert bool((filler == 1).all())


def test_capture_reads_ids_in_place():
    w = _weights()
    x, _, idx, _ = _batch(24)
    layer, eager = _layer(w, down=True), _layer(w, down=True)
    graph, out = layer.capture(x, adapter_idx=idx)
    for seed in (5, 6, 7):
        idx.copy_(_batch(24, seed)[2])
        graph.replay()
        assert torch.equal(out, eager.forward(x, adapter_idx=idx))
        torch.cuda.synchronize()


def test_a_training_step_in_which_nothing_counts():
    """No token of the mask, no adapter, no gradient: the losses and all gradients are zeros.  A batch without tokens is refused, with
    and without ids."""
    w = _weights()
    x, dy, idx, mask = _batch(90)
    layer = _layer(w)
    y0 = layer.forward(x).clone()
    idx.fill_(-1), mask.zero_(), dy.zero_()
    assert torch.equal(layer.forward(x, adapter_idx=idx), y0)
    got = layer.backward(x, dy, idx, mask, 0.5, 0.25)
    assert not any(bool(t.any()) for t in (*got, layer.losses, layer.counts))
    for ids in (None, idx[:0]):
        with pytest.raises(MoeError):
            layer.forward(x[:0], adapter_idx=ids)
