"""The adapters' sums at the lengths that prompts and long batches have: the first product's cut into six to eight slices, added where
the second product reads them or packed before it, and groups of rows cut into pieces of more than 256.

Tolerances as in test_gpu_lora.py, with all 24 bits of the narrow factor.  The reference is the definition in float64, adapter by adapter."""
import numpy as np
import pytest
import torch

from guards import Guards
from paper_2508_19373_amd import binding as B
from test_gpu_lora import _check, _make

pytestmark = pytest.mark.gpu


def _reference(d, v=None):
    """y without y_in, v and, for a given v, (dx without dx_in, grad_a, grad_b)."""
    x, a, b, scale, dy = (d[n].double() for n in ("x", "a", "b", "scale", "dy"))
    (T, K), (L, N, r) = x.shape, b.shape
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device="cuda")  # noqa: E731
    out = [z(T, N), z(T, r)] if v is None else [z(T, K), z(L, r, K), z(L, N, r)]
    for i in range(L):
        rows = torch.nonzero(d["idx"] == i).flatten()
        if v is None:
            out[1][rows] = x[rows] @ a[i].t()
            out[0][rows] = scale[i] * (out[1][rows] @ b[i].t())
        else:
            u = scale[i] * (dy[rows] @ b[i])
            out[0][rows] = u @ a[i]
            out[1][i] = u.t() @ x[rows]
            out[2][i] = scale[i] * (dy[rows].t() @ v[rows].double())
    return out


def _abs(d):
    o = {n: t.abs() if torch.is_tensor(t) and n != "idx" else t for n, t in d.items()}
    none = (d["idx"] < 0) | (d["idx"] >= d["L"])
    o["x"][none], o["dy"][none] = 0.0, 0.0
    return o


def _np(t):
    return t.double().cpu().numpy()


def _forward(d, f32):
    T, K, N, r, L = (d[n] for n in ("T", "K", "N", "r", "L"))
    dt, guard = torch.float32 if f32 else torch.bfloat16, Guards()
    y_in = d["y_in"].to(dt)
    y, v = guard.empty((T, N), dt, float("nan")), guard.empty((T, r), torch.float32, float("nan"))
    ws = guard.empty(B.moe_lora_workspace_bytes(T, K, N, r, L), torch.uint8, 0xFF)
    B.moe_lora_forward(d["x"], d["idx"], T, K, N, r, L, d["a"], d["b"], d["scale"], y_in, y, v, ws, B.MOE_OUT_F32 if f32 else 0)
    guard.check()
    (ref, ref_v), (terms, terms_v) = _reference(d), _reference(_abs(d))
    _check(y, _np(ref + y_in.double()), _np(terms + y_in.double().abs()), K + r, bf16=not f32, factor16=False)
    _check(v, _np(ref_v), _np(terms_v), K, bf16=False, factor16=False)
    return v


def _backward(d, v):
    T, K, N, r, L = (d[n] for n in ("T", "K", "N", "r", "L"))
    guard = Guards()
    f = lambda *s, dt=torch.float32: guard.empty(s, dt, float("nan"))  # noqa: E731
    dx, ga, gb = f(T, K, dt=torch.bfloat16), f(L, r, K), f(L, N, r)
    ws = guard.empty(B.moe_lora_workspace_bytes(T, K, N, r, L, True), torch.uint8, 0xFF)
    B.moe_lora_backward(d["x"], d["dy"], d["idx"], T, K, N, r, L, d["a"], d["b"], d["scale"], v, d["dx_in"], dx, ga, gb, ws)
    guard.check()
    ref, terms = _reference(d, v), _reference(_abs(d), v.abs())
    _check(dx, _np(ref[0] + d["dx_in"].double()), _np(terms[0] + d["dx_in"].double().abs()), N + r, bf16=True, factor16=False)
    _check(ga, _np(ref[1]), _np(terms[1]), N + T, bf16=False, factor16=False)
    _check(gb, _np(ref[2]), _np(terms[2]), T + 2, bf16=False, factor16=False)


SLICED = [  # T, K, N, rank, adapters, order: slices of the forward's and of the backward's first product
    (130, 4104, 264, 16, 5, "mixed"),     # 8, 1
    (300, 4096, 136, 64, 4, "mixed"),     # 8, 1
    (4096, 4096, 72, 64, 3, "runs"),      # 8 packed, 1
    (1500, 3080, 136, 128, 3, "runs"),    # 7 packed, 1
    (5000, 4096, 264, 32, 5, "mixed"),    # 7, 1
    (200, 136, 4104, 128, 4, "mixed"),    # 1, 8
    (333, 520, 3080, 48, 40, "mixed"),    # 2, 7
    (8192, 2048, 4096, 24, 6, "runs"),    # 4, 4
]


@pytest.mark.parametrize("T,K,N,r,L,kind", SLICED)
def test_sliced_sums(T, K, N, r, L, kind):
    print("case slices", T, K, N, r, L, kind, flush=True)
    host = _make(T + K, T, K, N, r, L, kind)
    d = {n: t.cuda() if torch.is_tensor(t) else t for n, t in host.items()}
    _forward(d, True)
    _backward(d, _forward(d, False))


@pytest.mark.parametrize("K,N,r,counts", [(2048, 2048, 128, [5000, 1281, 1280, 639]), (4096, 4096, 64, [0, 769, 3000, 768, 1463]),
                                          (2048, 1032, 64, [2600, 1, 512, 513, 255])])
def test_groups_cut_into_long_pieces(K, N, r, counts):
    """Pieces of 1280, 768 and 256 rows: groups of several, of exactly one, of one row more, of none."""
    T, L = sum(counts), len(counts)
    print("case pieces", T, K, N, r, counts, flush=True)
    host = _make(T, T, K, N, r, L, "one")
    host["idx"] = torch.repeat_interleave(torch.arange(L), torch.tensor(counts)).int()
    d = {n: t.cuda() if torch.is_tensor(t) else t for n, t in host.items()}
    v = torch.from_numpy(np.random.default_rng(T).standard_normal((T, r))).float().cuda()
    _backward(d, v)


@pytest.mark.parametrize("T,K,N,r", [(6, 520, 264, 16), (48, 4096, 264, 64), (150, 136, 264, 16), (700, 1032, 520, 72), (9000, 136, 72, 8)])
def test_slots_without_an_adapter_may_hold_anything(T, K, N, r):
    """Of five slots three are in use; what lies in the others, NaN here, reaches nothing, and their gradients are zeros."""
    L = 5
    host = _make(T, T, K, N, r, L, "one")
    host["idx"] = torch.tensor([1, 3, 2])[torch.arange(T) % 3].int()
    d = {n: t.cuda() if torch.is_tensor(t) else t for n, t in host.items()}
    clean = {n: t.clone() if torch.is_tensor(t) else t for n, t in d.items()}
    for n in ("a", "b", "scale"):
        d[n][0] = d[n][4] = float("nan")

    def step(one):
        y, v = torch.empty((T, N), device="cuda"), torch.empty((T, r), device="cuda")
        dx, ga, gb = torch.empty_like(one["x"]), torch.empty((L, r, K), device="cuda"), torch.empty((L, N, r), device="cuda")
        ws = torch.empty(max(B.moe_lora_workspace_bytes(T, K, N, r, L, back) for back in (False, True)), dtype=torch.uint8, device="cuda")
        B.moe_lora_forward(one["x"], one["idx"], T, K, N, r, L, one["a"], one["b"], one["scale"], None, y, v, ws, B.MOE_OUT_F32)
        B.moe_lora_backward(one["x"], one["dy"], one["idx"], T, K, N, r, L, one["a"], one["b"], one["scale"], v, None, dx, ga, gb, ws)
        return y, v, dx, ga, gb
    got, want = step(d), step(clean)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert not any(t[i].any() for t in got[3:] for i in (0, 4))


@pytest.mark.parametrize("T,K,N,r,L,kind", [(3, 262144, 262144, 8, 2, "one"), (70, 262144, 1032, 16, 2, "mixed"), (70, 1032, 262144, 24, 2, "mixed"),
                                            (2, 8, 8, 8, 256, "mixed"), (64, 8, 8, 128, 256, "mixed"), (300, 8, 8, 120, 256, "mixed"),
                                            (8193, 64, 64, 16, 256, "mixed"), (9000, 64, 64, 16, 255, "runs")])
def test_at_the_limits(T, K, N, r, L, kind):
    """The most columns, the fewest, the most adapters, on either side of the rows that one sort keeps in registers."""
    print("case limits", T, K, N, r, L, kind, flush=True)
    host = _make(T, T, K, N, r, L, kind)
    d = {n: t.cuda() if torch.is_tensor(t) else t for n, t in host.items()}
    _forward(d, True)
    _backward(d, _forward(d, False))
