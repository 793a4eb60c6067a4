"""GPU parity of the router's losses and gradients against the float64 oracle, through the C ABI.

Tolerances, per element.  A sum of n fp32 products in any order is off by at most (n + 8) 2^-23 of the sum of their absolute
values; exp and log are good to a few units in the last place, and a softmax of logits up to 20 apart rounds them by 20 * 2^-24 first: 2^-18 of
a probability covers both.  bf16 results add half a step, 2^-8, and the factors of their sums may be held in 16 bits."""
import numpy as np
import pytest
import torch

from guards import Guards
from oracle import moe_oracle as M
from oracle import router_grad_oracle as O
from paper_2508_19373_amd import binding as B

pytestmark = pytest.mark.gpu


def _f64(t):
    return t.double().cpu().numpy()


def _routing(seed, T, E, k, renorm):
    g = np.random.default_rng(seed)
    logits = (g.standard_normal((T, E)) * 1.5 + g.standard_normal(E)).astype(np.float32)
    if T:
        idx, _, _ = M.route_topk(logits, k, renorm)
    else:
        idx = np.zeros((0, k), np.int32)
    return logits, idx, g


LOSS_SIZES = [(0, 8, 2), (1, 1, 1), (1, 8, 2), (3, 5, 5), (64, 8, 2), (65, 16, 1), (130, 60, 4), (200, 64, 8), (257, 33, 3), (300, 130, 6),
              (111, 200, 16), (70, 256, 16), (1500, 8, 2), (5000, 60, 4)]


@pytest.mark.parametrize("T,E,k", LOSS_SIZES)
@pytest.mark.parametrize("mask_kind", ["none", "padded", "empty"])
def test_losses_and_logit_gradient(T, E, k, mask_kind):
    renorm = (T + E) % 2 == 1
    print("case router loss", T, E, k, mask_kind, renorm, flush=True)
    logits, idx, g = _routing(T + E, T, E, k, renorm)
    mask = {"none": None, "padded": (np.arange(T) % 7 < 5).astype(np.uint8) * 200, "empty": np.zeros(T, np.uint8)}[mask_kind]
    dw = g.standard_normal((T, k)).astype(np.float32)
    guard = Guards()
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    counts = guard.empty(E + 1, torch.int32, -5)
    prob, losses = guard.empty(E, torch.float32, float("nan")), guard.empty(2, torch.float32, float("nan"))
    ws = guard.empty(B.moe_balance_workspace_bytes(T, E), torch.uint8, 0xFF)
    seen = logits.copy()
    if mask is not None:
        seen[mask == 0] = np.nan       # padding may hold anything
    B.moe_balance_loss(dev(seen), dev(idx), dev(mask), T, E, k, counts, prob, losses, ws)
    guard.check()
    ref = O.balance_loss(logits.astype(np.float64), idx, mask)
    assert np.array_equal(counts.cpu().numpy(), ref[0])
    n = max(int(ref[0][E]), 1)
    assert (np.abs(_f64(prob) - ref[1]) <= ref[1] * (2.0 ** -18 + (n + 8) * 2.0 ** -23)).all()
    got = _f64(losses)
    for have, want in zip(got, ref[2:]):
        assert abs(have - want) <= want * (2.0 ** -17 + (n + E + 8) * 2.0 ** -23)
    # the gradient of the gates and of the losses together, of the losses alone (padding not read), of the gates alone
    cb, cz = 0.7 * n, 0.3 * n          # (so that neither part hides behind the other)
    d_logits = guard.empty((T, E), torch.float32, float("nan"))
    flags = B.MOE_RENORM_TOPK if renorm else 0
    top = logits.max(1, keepdims=True) if T else logits
    p = np.exp(logits.astype(np.float64) - top)
    p /= p.sum(1, keepdims=True)
    size = np.abs(dw).sum(1, keepdims=True) + cb * E / (k * n) * ref[0][:E].max() / n + cz * 2 * 20 / n
    for which in ("all", "losses", "gates"):
        d = None if which == "losses" else dw
        c = (0.0, 0.0) if which == "gates" else (cb, cz)
        source = seen if which == "losses" else logits
        B.moe_route_backward(dev(source), dev(idx), dev(d), dev(mask), None if which == "gates" else counts, T, E, k, *c, flags,
                             d_logits)
        guard.check()
        want = O.route_backward(logits.astype(np.float64), idx, d, mask, None if which == "gates" else ref[0], *c, renorm)
        # every term is a probability (of all experts or of the picked ones) times a factor bounded by `size`
        w = p.copy()
        if renorm and T:
            for t in range(T):
                w[t, idx[t]] = p[t, idx[t]] / p[t, idx[t]].sum()
        assert (np.abs(_f64(d_logits) - want) <= (w + p) * size * 2.0 ** -16 + 1e-30).all(), which


def test_excluded_experts_and_invalid_ids():
    """-inf keeps an expert out of a token's softmax; ids outside the experts are not counted."""
    logits = np.array([[0.0, -np.inf, 1.0, -np.inf], [-np.inf, 2.0, -np.inf, -np.inf], [0.5, 0.25, -1.0, 3.0]], np.float32)
    idx = np.array([[2, 0], [1, 7], [-3, 3]], np.int32)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    counts, prob = torch.empty(5, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda")
    losses, ws = torch.empty(2, device="cuda"), torch.empty(B.moe_balance_workspace_bytes(3, 4), dtype=torch.uint8, device="cuda")
    B.moe_balance_loss(dev(logits), dev(idx), None, 3, 4, 2, counts, prob, losses, ws)
    with np.errstate(invalid="ignore"):
        ref = O.balance_loss(logits.astype(np.float64), idx)
    assert counts.tolist() == list(ref[0]) == [1, 1, 1, 1, 3]
    assert np.allclose(_f64(prob), ref[1], rtol=1e-5) and np.allclose(_f64(losses), ref[2:], rtol=1e-5)
    d = torch.empty((3, 4), device="cuda")
    B.moe_route_backward(dev(logits), dev(idx), None, None, counts, 3, 4, 2, 0.5, 0.5, 0, d)
    want = O.route_backward(logits.astype(np.float64), idx, None, None, ref[0], 0.5, 0.5, False)
    assert np.allclose(_f64(d), want, rtol=1e-5, atol=1e-7) and not _f64(d)[np.isinf(logits)].any()


ROUTER_SIZES = [(0, 64, 8), (1, 8, 1), (1, 2048, 60), (5, 72, 3), (64, 512, 8), (65, 200, 16), (100, 1000, 60), (333, 520, 64), (257, 264, 130),
                (700, 136, 256), (2100, 1032, 8), (4100, 256, 60),
                (5000, 2048, 60), (3000, 1032, 200), (2600, 2048, 100), (2600, 2048, 20)]


@pytest.mark.parametrize("T,H,E", ROUTER_SIZES)
def test_router_backward(T, H, E):
    print("case router backward", T, H, E, flush=True)
    g = torch.Generator().manual_seed(T + H + E)
    t = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x, w, dl, dx_in = t(T, H).bfloat16(), t(H, E), t(T, E), t(T, H).bfloat16()
    d, guard = [v.cuda() for v in (x, w, dl, dx_in)], Guards()
    ws = guard.empty(B.moe_router_backward_workspace_bytes(T, H, E), torch.uint8, 0xFF)
    runs = []
    for mode in ("apart", "in place", "no dx", "fresh"):
        dw = guard.empty((H, E), torch.float32, float("nan"))
        dx = None if mode == "no dx" else guard.empty((T, H), torch.bfloat16, float("nan"))
        if mode == "in place":
            dx.copy_(d[3])
        B.moe_router_backward(d[0], None if mode == "no dx" else d[1], d[2], T, H, E, {"apart": d[3], "in place": dx}.get(mode), dx, dw, ws)
        guard.check()
        runs.append((dx, dw))
    x, w, dl, dx_in = (_f64(v) for v in (x, w, dl, dx_in))
    for (dx, dw), base in zip(runs, (dx_in, dx_in, None, None)):
        ref_x, ref_w = O.router_backward(x, w, dl, base)
        terms_x, terms_w = O.router_backward(np.abs(x), np.abs(w), np.abs(dl), None if base is None else np.abs(base))
        assert torch.equal(dw, runs[0][1])
        assert (np.abs(_f64(dw) - ref_w) <= terms_w * (T + 8) * 2.0 ** -23 + 1e-37).all()
        if T:
            assert np.linalg.norm(_f64(dw) - ref_w) / np.linalg.norm(ref_w) < 1e-5
        if dx is not None:
            tol = terms_x * ((E + 8) * 2.0 ** -23 + 3 * 2.0 ** -16) + np.abs(ref_x) * 2.0 ** -8 * 1.01
            assert (np.abs(_f64(dx) - ref_x) <= tol).all()


@pytest.mark.parametrize("T,H,k,bf16,shared", [(0, 64, 2, False, True), (1, 8, 1, False, True), (1, 4096, 2, True, False), (5, 72, 3, True, True),
                                               (33, 2048, 4, False, True), (64, 3584, 8, True, True), (7, 200, 16, False, False),
                                               (300, 520, 5, False, True), (20, 8200, 2, True, False)])
def test_combine_backward(T, H, k, bf16, shared):
    print("case combine backward", T, H, k, bf16, shared, flush=True)
    g = torch.Generator().manual_seed(T + H + k)
    dt = torch.bfloat16 if bf16 else torch.float32
    rows = max(T * k, 1)
    y = torch.randn((rows, H), generator=g).to(dt)
    dy, x = torch.randn((T, H), generator=g).bfloat16(), torch.randn((T, H), generator=g).bfloat16()
    ys, ws = torch.randn((T, H), generator=g).to(dt), torch.randn(H, generator=g) * 0.05
    slot = torch.randperm(rows, generator=g)[:T * k].int()
    slot[torch.rand(T * k, generator=g) < 0.3] = -1
    y[sorted(set(range(rows)) - set(slot.tolist()))] = float("nan")      # rows nobody points at are not read
    d, guard = [v.cuda() for v in (dy, y, slot, ys, x, ws)], Guards()
    dw, dg = guard.empty((T, k), torch.float32, float("nan")), guard.empty(T, torch.float32, float("nan")) if shared else None
    B.moe_combine_backward(d[0], d[1], d[2], T, k, H, *(d[3:] if shared else (None,) * 3), dw, dg, B.MOE_Y_PERM_BF16 if bf16 else 0)
    guard.check()
    a = [_f64(v) for v in (dy, y, slot.float(), ys, x, ws)]
    slot = slot.numpy()
    ref = O.combine_backward(a[0], a[1], slot, k, *(a[3:] if shared else ()))
    terms = O.combine_backward(np.abs(a[0]), np.abs(a[1]), slot, k)[0]
    assert (np.abs(_f64(dw) - ref[0]) <= terms * (H + 8) * 2.0 ** -23 + 1e-37).all()
    assert not _f64(dw)[slot.reshape(T, k) < 0].any()
    if shared:
        size = 0.25 * np.einsum("th,th->t", np.abs(a[0]), np.abs(a[3]))
        wide = (np.abs(a[4]) @ np.abs(a[5])) * (H + 8) * 2.0 ** -23          # error of x . w_s, which moves g (1 - g) by at most a tenth of it
        assert (np.abs(_f64(dg) - ref[1]) <= size * ((H + 16) * 2.0 ** -23 + 4 * wide)).all()


def test_offsets_beyond_32_bits():
    """More than 2^31 elements in y_perm: the far rows' products are those of a small call."""
    T, k, H = 140_000, 2, 8192
    y = torch.zeros((T * k, H), dtype=torch.bfloat16, device="cuda")
    y[-4:] = torch.randn((4, H), device="cuda").bfloat16()
    dy = torch.randn((T, H), dtype=torch.bfloat16, device="cuda")
    slot = torch.arange(T * k, dtype=torch.int32, device="cuda")
    dw = torch.empty((T, k), device="cuda")
    B.moe_combine_backward(dy, y, slot, T, k, H, None, None, None, dw, None, B.MOE_Y_PERM_BF16)
    want = (dy[-2:].double().unsqueeze(1) * y[-4:].double().view(2, k, H)).sum(2)
    size = (dy[-2:].double().unsqueeze(1) * y[-4:].double().view(2, k, H)).abs().sum(2)
    assert ((dw[-2:].double() - want).abs() <= size * (H + 8) * 2.0 ** -23).all() and not dw[:-2].any()


def test_chain_is_the_same_in_a_graph():
    """dy to the router's weights in one captured chain, replayed with eager work in between."""
    T, H, E, k = 200, 512, 60, 4
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, w, dy, y_perm = rnd(T, H).bfloat16(), rnd(H, E) * 0.05, rnd(T, H).bfloat16(), rnd(T * k, H)
    logits = x.float() @ w
    idx = logits.topk(k, dim=1).indices.int().contiguous()
    slot = torch.randperm(T * k, generator=g, device="cuda").int()
    mask = (torch.arange(T, device="cuda") < 150).to(torch.uint8)

    def new():
        return dict(dtw=torch.empty((T, k), device="cuda"), counts=torch.empty(E + 1, dtype=torch.int32, device="cuda"),
                    prob=torch.empty(E, device="cuda"), losses=torch.empty(2, device="cuda"), dl=torch.empty((T, E), device="cuda"),
                    dx=torch.empty_like(x), dw=torch.empty((H, E), device="cuda"),
                    ws=torch.empty(max(B.moe_balance_workspace_bytes(T, E), B.moe_router_backward_workspace_bytes(T, H, E)), dtype=torch.uint8, device="cuda"))

    def step(o):
        B.moe_balance_loss(logits, idx, mask, T, E, k, o["counts"], o["prob"], o["losses"], o["ws"])
        B.moe_combine_backward(dy, y_perm, slot, T, k, H, None, None, None, o["dtw"])
        B.moe_route_backward(logits, idx, o["dtw"], mask, o["counts"], T, E, k, 0.01, 0.001, 0, o["dl"])
        B.moe_router_backward(x, w, o["dl"], T, H, E, None, o["dx"], o["dw"], o["ws"])
    eager, captured = new(), new()
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for turn in range(4):
        captured["ws"].random_(0, 256)
        for n in ("dtw", "counts", "prob", "losses", "dl", "dx", "dw"):
            captured[n].zero_()
        if turn == 2:
            dy.mul_(-2.0)
            mask.fill_(1)
            step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for n in ("dtw", "counts", "prob", "losses", "dl", "dx", "dw"):
            assert torch.equal(eager[n], captured[n]), n


def test_more_tiles_than_a_grid_has_rows():
    """4.4 million tokens: over 65536 tiles of 64.  Values are small integers, so that every sum is exact."""
    T, H, E = 4_400_001, 8, 4
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randint(-1, 2, (T, H), generator=g, device="cuda").bfloat16()
    w = torch.randint(-2, 3, (H, E), generator=g, device="cuda").float()
    dl = torch.randint(-1, 2, (T, E), generator=g, device="cuda").float()
    dx, dw = torch.empty((T, H), dtype=torch.bfloat16, device="cuda"), torch.empty((H, E), device="cuda")
    ws = torch.empty(B.moe_router_backward_workspace_bytes(T, H, E), dtype=torch.uint8, device="cuda")
    B.moe_router_backward(x, w, dl, T, H, E, None, dx, dw, ws)
    assert torch.equal(dx.float(), dl @ w.T)
    assert torch.equal(dw.double(), x.double().T @ dl.double())
