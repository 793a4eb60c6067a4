"""GPU parity of the adapters' kernels against the float64 oracle, through the C ABI.

Tolerances, per element.  A sum of n fp32 products in any order is off by at most (n + 8) 2^-23 of the sum of their absolute
values (one rounding to nearest or a truncation for every term, and a few more for the factors).  Where the result is bf16 the kernels may
hold the small factor (v or u) in 16 bits or more: 2^-16 of the same sum; where it is fp32, in 24.  Then half a step of the
result's type: 2^-8 of a bf16 value, 2^-24 of an fp32 one.  Over all elements the errors of the fp32 results are independent: rel-L2 1e-5
(sqrt(8192) 2^-24 = 5.4e-6 for the longest sum here)."""
import numpy as np
import pytest
import torch

from guards import Guards
from oracle import lora_oracle as O
from paper_2508_19373_amd import binding as B

pytestmark = pytest.mark.gpu


def _ids(g, kind, T, L):
    if kind == "mixed":            # any order, some without, some out of range on either side
        idx = g.integers(0, L, T)
        bare = g.random(T) < 0.2
        idx[bare] = g.choice([-1, -7, L, L + 3, 2 ** 31 - 1, -2 ** 31], T)[bare]
    elif kind == "runs":           # requests behind each other
        idx = np.sort(g.integers(0, L, T))[::-1] if T else np.zeros(0, np.int64)
    elif kind == "one":
        idx = np.full(T, L - 1)
    else:                          # nobody has one
        idx = np.full(T, -1)
    return np.ascontiguousarray(idx).astype(np.int32)


def _make(seed, T, K, N, r, L, kind):
    g = np.random.default_rng(seed)
    t = lambda *s: torch.from_numpy(g.standard_normal(s)).float()  # noqa: E731
    d = dict(T=T, K=K, N=N, r=r, L=L, idx=torch.from_numpy(_ids(g, kind, T, L)), x=t(T, K).bfloat16(),
             a=(t(L, r, K) * K ** -0.5).bfloat16(), b=(t(L, N, r) * r ** -0.5).bfloat16(),
             scale=torch.from_numpy(g.uniform(0.5, 2.0, L)).float(), y_in=t(T, N), dy=t(T, N).bfloat16(),
             dx_in=t(T, K).bfloat16())
    none = (d["idx"] < 0) | (d["idx"] >= L)
    d["x"][none] = float("nan")     # the rows of requests without an adapter may hold anything
    d["dy"][none] = float("inf")
    return d


def _f64(t):
    return t.double().cpu().numpy()


def _cuda(d):
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in d.items()}


def _check(got, ref, terms, n, *, bf16, factor16):
    """terms: the sum of the products' absolute values, n: how many there are."""
    got = _f64(got)
    assert np.isfinite(got).all()
    tol = terms * ((n + 8) * 2.0 ** -23 + (2.0 ** -16 if factor16 else 0.0)) + np.abs(ref) * (2.0 ** -8 if bf16 else 2.0 ** -24) * 1.01
    bad = np.abs(got - ref) > tol + 1e-37
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])
    if not bf16 and np.linalg.norm(ref) > 0:
        assert np.linalg.norm(got - ref) / np.linalg.norm(ref) < 1e-5


def _abs(d):
    o = {k: np.abs(_f64(d[k])) for k in ("x", "a", "b", "scale", "dy")}
    none = ((d["idx"] < 0) | (d["idx"] >= d["L"])).numpy()
    o["x"][none], o["dy"][none] = 0.0, 0.0
    return o


SIZES = [  # T, K, N, rank, adapters, order of the ids
    (1, 64, 64, 8, 1, "one"), (1, 4096, 1408, 16, 8, "mixed"), (2, 72, 8, 24, 3, "mixed"), (16, 520, 200, 16, 5, "mixed"),
    (17, 8, 264, 64, 40, "mixed"), (48, 1024, 512, 16, 256, "mixed"), (63, 200, 1000, 128, 2, "one"), (64, 136, 72, 8, 64, "mixed"),
    (65, 136, 72, 40, 4, "runs"), (64, 512, 512, 32, 3, "none"), (200, 712, 328, 16, 7, "mixed"), (333, 512, 1024, 48, 12, "runs"),
    (777, 256, 520, 112, 3, "mixed"), (1000, 1000, 136, 64, 256, "mixed"), (2049, 128, 192, 16, 9, "mixed"),
    (2500, 72, 264, 8, 1, "one"), (300, 64, 64, 128, 5, "none"),
    (33, 2048, 1032, 32, 20, "mixed"), (64, 4096, 520, 8, 6, "runs"), (20, 4104, 264, 16, 4, "mixed"), (600, 264, 392, 32, 5, "mixed"),
    (25000, 64, 72, 64, 3, "runs"), (48, 4096, 4104, 16, 32, "mixed"), (64, 2048, 2056, 24, 64, "mixed"), (60, 2000, 2600, 8, 64, "mixed"),
    (700, 1024, 1024, 128, 6, "mixed"), (600, 1032, 2056, 32, 9, "mixed"),
]


@pytest.mark.parametrize("T,K,N,r,L,kind", SIZES)
@pytest.mark.parametrize("f32", [False, True])
def test_forward(T, K, N, r, L, kind, f32):
    print("case lora forward", T, K, N, r, L, kind, f32, flush=True)
    host = _make(T * 7 + K, T, K, N, r, L, kind)
    dt = torch.float32 if f32 else torch.bfloat16
    host["y_in"] = host["y_in"].to(dt)
    d, guard = _cuda(host), Guards()
    ref, ref_v = O.forward(_f64(host["x"]), host["idx"].numpy(), _f64(host["a"]), _f64(host["b"]), _f64(host["scale"]), _f64(host["y_in"]))
    p = _abs(host)
    terms, terms_v = O.forward(p["x"], host["idx"].numpy(), p["a"], p["b"], p["scale"], np.abs(_f64(host["y_in"])))
    ws = guard.empty(B.moe_lora_workspace_bytes(T, K, N, r, L), torch.uint8, 0xFF)
    flags = B.MOE_OUT_F32 if f32 else 0
    runs = {}
    for mode in ("apart", "in place", "delta"):
        v = guard.empty((T, r), torch.float32, float("nan")) if mode != "delta" else None
        out = guard.empty((T, N), dt, float("nan"))
        if mode == "in place":
            out.copy_(d["y_in"])
        y_in = {"apart": d["y_in"], "in place": out, "delta": None}[mode]
        B.moe_lora_forward(d["x"], d["idx"], T, K, N, r, L, d["a"], d["b"], d["scale"], y_in, out, v, ws, flags)
        guard.check()
        runs[mode] = out, v
    _check(runs["apart"][0], ref, terms, K + r, bf16=not f32, factor16=not f32)
    _check(runs["apart"][1], ref_v, terms_v, K, bf16=False, factor16=False)
    for a, b in zip(runs["apart"], runs["in place"]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    delta = ref - _f64(host["y_in"])
    _check(runs["delta"][0], delta, terms - np.abs(_f64(host["y_in"])) + np.abs(delta) * 1e-6, K + r, bf16=not f32, factor16=not f32)
    none = (host["idx"] < 0) | (host["idx"] >= L)
    assert torch.equal(runs["apart"][0][none.cuda()], d["y_in"][none.cuda()])   # bit for bit
    assert not runs["apart"][1][none.cuda()].any() and not runs["delta"][0][none.cuda()].any()


@pytest.mark.parametrize("T,K,N,r,L,kind", SIZES + [(0, 64, 64, 16, 4, "none")])
def test_backward(T, K, N, r, L, kind):
    print("case lora backward", T, K, N, r, L, kind, flush=True)
    host = _make(T * 5 + N, T, K, N, r, L, kind)
    d, guard = _cuda(host), Guards()
    idx = host["idx"].numpy()
    v = O.forward(np.nan_to_num(_f64(host["x"])), idx, _f64(host["a"]), _f64(host["b"]), _f64(host["scale"]))[1].astype(np.float32)
    none = (idx < 0) | (idx >= L)
    v_dev = torch.from_numpy(v)
    v_dev[torch.from_numpy(none)] = float("nan")
    v_dev = v_dev.cuda()
    args = (_f64(host["x"]), _f64(host["dy"]), idx, _f64(host["a"]), _f64(host["b"]), _f64(host["scale"]), v.astype(np.float64))
    ref = O.backward(*args, _f64(host["dx_in"]))
    p = _abs(host)
    terms = O.backward(p["x"], p["dy"], idx, p["a"], p["b"], p["scale"], np.abs(v).astype(np.float64), np.abs(_f64(host["dx_in"])))
    ws = guard.empty(B.moe_lora_workspace_bytes(T, K, N, r, L, True), torch.uint8, 0xFF)
    f = lambda *s, dt=torch.float32: guard.empty(s, dt, float("nan"))  # noqa: E731
    runs = []
    for mode in ("apart", "in place", "no dx"):
        dx = None if mode == "no dx" else f(T, K, dt=torch.bfloat16)
        dx_in = {"apart": d["dx_in"], "in place": dx, "no dx": None}[mode]
        if mode == "in place":
            dx.copy_(d["dx_in"])
        ga, gb = f(L, r, K), f(L, N, r)
        B.moe_lora_backward(d["x"], d["dy"], d["idx"], T, K, N, r, L, d["a"], d["b"], d["scale"], v_dev, dx_in, dx, ga, gb, ws)
        guard.check()
        runs.append((dx, ga, gb))
    dx, ga, gb = runs[0]
    _check(dx, ref[0], terms[0], N + r, bf16=True, factor16=True)
    _check(ga, ref[1], terms[1], N + T, bf16=False, factor16=False)
    _check(gb, ref[2], terms[2], T + 2, bf16=False, factor16=False)
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert b is None or torch.equal(a, b)
    assert torch.equal(dx[torch.from_numpy(none).cuda()], d["dx_in"][torch.from_numpy(none).cuda()])


def test_gradients_against_differences_of_the_forward_call():
    """The loss sum(dy * y) is linear in A and in B, so a difference of two forward calls in fp32 is its derivative."""
    T, K, N, r, L = 40, 128, 96, 16, 3
    host = _make(11, T, K, N, r, L, "runs")
    d = _cuda(host)
    ws = torch.empty(B.moe_lora_workspace_bytes(T, K, N, r, L, True), dtype=torch.uint8, device="cuda")
    v = torch.empty((T, r), device="cuda")

    def y(a, b):
        out = torch.empty((T, N), device="cuda")
        B.moe_lora_forward(d["x"], d["idx"], T, K, N, r, L, a, b, d["scale"], None, out, v, ws, B.MOE_OUT_F32)
        return out.double()
    y(d["a"], d["b"])
    ga, gb, dx = torch.empty((L, r, K), device="cuda"), torch.empty((L, N, r), device="cuda"), torch.empty_like(d["x"])
    B.moe_lora_backward(d["x"], d["dy"], d["idx"], T, K, N, r, L, d["a"], d["b"], d["scale"], v, None, dx, ga, gb, ws)
    g = np.random.default_rng(1)
    for name, grad in (("a", ga), ("b", gb)):
        for _ in range(4):
            step = torch.from_numpy(g.choice([-1.0, 0.0, 1.0], d[name].shape)).bfloat16().cuda()
            big, small = d[name].clone(), d[name].clone()
            big += step
            small -= step
            moved = (big.double() - small.double())          # what the rounding of the sums left of 2 step
            hi, lo = ({"a": d["a"], "b": d["b"], name: t} for t in (big, small))
            diff = float(((y(hi["a"], hi["b"]) - y(lo["a"], lo["b"])) * d["dy"].double()).sum())
            want = float((grad.double() * moved).sum())
            size = float((grad.double() * moved).abs().sum())
            assert abs(diff - want) < 1e-5 * size, name


def test_the_same_call_gives_the_same_bits_on_another_stream_and_in_a_graph():
    T, K, N, r, L = 300, 520, 264, 32, 9
    host = _make(21, T, K, N, r, L, "mixed")
    d = _cuda(host)
    for n in ("x", "dy"):              # finite everywhere: further down every row gets an adapter once
        d[n].nan_to_num_(0.0, 0.0, 0.0)
    new = lambda: dict(ws=torch.empty(B.moe_lora_workspace_bytes(T, K, N, r, L, True), dtype=torch.uint8, device="cuda"),  # noqa: E731
                       y=torch.empty((T, N), device="cuda"), v=torch.empty((T, r), device="cuda"), dx=torch.empty_like(d["x"]),
                       ga=torch.empty((L, r, K), device="cuda"), gb=torch.empty((L, N, r), device="cuda"))

    def step(o):
        B.moe_lora_forward(d["x"], d["idx"], T, K, N, r, L, d["a"], d["b"], d["scale"], None, o["y"], o["v"], o["ws"], B.MOE_OUT_F32)
        B.moe_lora_backward(d["x"], d["dy"], d["idx"], T, K, N, r, L, d["a"], d["b"], d["scale"], o["v"], None, o["dx"], o["ga"], o["gb"], o["ws"])

    def same(p, q):
        return all(torch.equal(p[n], q[n]) for n in ("y", "v", "dx", "ga", "gb"))
    first, other, captured = new(), new(), new()
    step(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(other)                    # beside a second call on the main stream, each with its own workspace
    again = new()
    step(again)
    torch.cuda.synchronize()
    assert same(first, other) and same(first, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    before = {n: t.clone() for n, t in first.items()}
    for turn in range(4):
        for n in ("y", "v", "dx", "ga", "gb"):
            captured[n].fill_(float("nan"))
        captured["ws"].random_(0, 256)
        if turn == 2:                  # other adapters for the same captured call
            d["idx"].copy_(torch.roll(d["idx"], 5))
        graph.replay()
        torch.cuda.synchronize()
        step(first)
        torch.cuda.synchronize()
        assert same(first, captured)
        assert same(first, before) == (turn < 2)


def test_offsets_beyond_32_bits():
    """More than 2^31 elements in x, y and dx: rows at the far end are those of a small call."""
    T, W, r, L = (1 << 18) + 77, 8200, 8, 2
    idx = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    some = torch.tensor([0, 5, 200_000, T - 3, T - 1], device="cuda")
    idx[some] = torch.tensor([0, 1, 1, 0, 1], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    big = torch.zeros((T, W), dtype=torch.bfloat16, device="cuda")
    big[some] = torch.randn((5, W), generator=g, device="cuda").bfloat16()
    a = torch.randn((L, r, W), generator=g, device="cuda").bfloat16()
    b = torch.randn((L, W, r), generator=g, device="cuda").bfloat16()
    scale = torch.ones(L, device="cuda")
    out = torch.empty((T, W), dtype=torch.bfloat16, device="cuda")
    v = torch.empty((T, r), device="cuda")
    ws = torch.empty(B.moe_lora_workspace_bytes(T, W, W, r, L, True), dtype=torch.uint8, device="cuda")
    B.moe_lora_forward(big, idx, T, W, W, r, L, a, b, scale, None, out, v, ws)
    few, few_idx = big[some].contiguous(), idx[some].contiguous()
    out_few, v_few = torch.empty_like(few), torch.empty((5, r), device="cuda")
    B.moe_lora_forward(few, few_idx, 5, W, W, r, L, a, b, scale, None, out_few, v_few, ws)
    torch.cuda.synchronize()
    assert torch.allclose(v[some], v_few, rtol=1e-4, atol=1e-3)          # K 2^-23 of sums of 8200 products of order one
    assert torch.allclose(out[some].float(), out_few.float(), rtol=2.0 ** -7, atol=0.05)
    assert not out[some[2] + 1].any() and not out[T - 2].any()
    ga, gb = torch.empty((L, r, W), device="cuda"), torch.empty((L, W, r), device="cuda")
    ga_few, gb_few = torch.empty_like(ga), torch.empty_like(gb)
    B.moe_lora_backward(big, big, idx, T, W, W, r, L, a, b, scale, v, None, out, ga, gb, ws)
    B.moe_lora_backward(few, few, few_idx, 5, W, W, r, L, a, b, scale, v_few, None, out_few, ga_few, gb_few, ws)
    torch.cuda.synchronize()
    assert torch.allclose(out[some].float(), out_few.float(), rtol=2.0 ** -7, atol=0.05)
    assert torch.allclose(ga, ga_few, rtol=1e-4, atol=0.02) and torch.allclose(gb, gb_few, rtol=1e-4, atol=0.02)
    assert not out[T - 2].any()


def test_more_tiles_than_a_grid_has_rows():
    """4.4 million rows: over 65536 tiles of 64.  Values are small integers, so that every sum is exact in fp32 and bf16."""
    T, K, N, r, L = 4_400_001, 8, 8, 8, 3
    g = torch.Generator(device="cuda").manual_seed(5)
    ints = lambda n, *s: torch.randint(-n, n + 1, s, generator=g, device="cuda").float()  # noqa: E731
    x, a, b = ints(1, T, K).bfloat16(), ints(1, L, r, K).bfloat16(), ints(1, L, N, r).bfloat16()
    scale = torch.tensor([1.0, 2.0, 0.5], device="cuda")
    idx = torch.randint(-1, L, (T,), generator=g, device="cuda", dtype=torch.int32)
    y, v = torch.full((T, N), 7.0, device="cuda"), torch.empty((T, r), device="cuda")
    ws = torch.empty(B.moe_lora_workspace_bytes(T, K, N, r, L), dtype=torch.uint8, device="cuda")
    B.moe_lora_forward(x, idx, T, K, N, r, L, a, b, scale, None, y, v, ws, B.MOE_OUT_F32)
    ref_v, ref_y = torch.zeros_like(v), torch.zeros_like(y)
    for e in range(L):
        one = (idx == e)[:, None].float()
        ve = (x.float() @ a[e].float().T) * one
        ref_v += ve
        ref_y += scale[e] * (ve @ b[e].float().T)
    assert torch.equal(v, ref_v) and torch.equal(y, ref_y)
