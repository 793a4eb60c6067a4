"""The C ABI of the adapters and of the router's gradients: exported symbols, and refusals on the host before any
device call."""
import os
import re

import pytest

from paper_2508_19373_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000   # a fake, aligned, non-null "device pointer": validation must fail before it is touched
W = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B._LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return B.lib()


@pytest.mark.parametrize("header,exports", [("moe_lora.h", "LORA_EXPORTS"), ("moe_router_grad.h", "ROUTER_GRAD_EXPORTS")])
def test_every_declared_symbol_is_exported(lib, header, exports):
    src = open(os.path.join(ROOT, "include", header)).read()
    names = set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", src, flags=re.S)))
    assert names == set(getattr(B, exports))
    assert all(getattr(lib, n) is not None for n in names)
    for name, value in re.findall(r"#define (MOE_LORA_MAX_[A-Z]+) (\d+)", src):
        assert getattr(B, name) == int(value)


def _call(f, args, **change):
    """args: ordered dict of defaults."""
    assert set(change) <= set(args)
    return f(*{**args, **change}.values())


FORWARD = dict(x=P, idx=P, T=4, K=64, N=128, rank=16, L=3, a=P, b=P, scale=P, y_in=P, y_out=P, v=P, ws=P, nbytes=W, flags=0,
               stream=None)
BACKWARD = dict(x=P, dy=P, idx=P, T=4, K=64, N=128, rank=16, L=3, a=P, b=P, scale=P, v=P, dx_in=P, dx=P, ga=P, gb=P, ws=P,
                nbytes=W, stream=None)


@pytest.mark.parametrize("name,args", [("moe_lora_forward", FORWARD), ("moe_lora_backward", BACKWARD)])
def test_lora_refusals(lib, name, args):
    f = getattr(lib, name)
    invalid, shape, space = B.MOE_ERR_INVALID_ARG, B.MOE_ERR_UNSUPPORTED_SHAPE, B.MOE_ERR_WORKSPACE
    for change in (dict(T=-1), dict(T=1 << 24), dict(K=0), dict(N=4), dict(rank=0), dict(L=0), dict(L=257), dict(K=(1 << 18) + 8),
                   dict(N=(1 << 18) + 8)):
        assert _call(f, args, **change) == invalid, change
    for change in (dict(K=60), dict(N=100), dict(rank=12), dict(rank=136)):
        assert _call(f, args, **change) == shape, change
    optional = ("y_in", "v") if name == "moe_lora_forward" else ("dx_in",)
    for key, value in args.items():
        if value == P and key not in optional + ("ws", "dx"):
            assert _call(f, args, **{key: None}) == invalid, key
        if value == P and key not in ("idx", "scale", "ws"):
            assert _call(f, args, **{key: P + 8}) == invalid, key
    need = B.moe_lora_workspace_bytes(4, 64, 128, 16, 3, name == "moe_lora_backward")
    assert need > 0
    assert _call(f, args, nbytes=need - 1) == space and _call(f, args, ws=None) == space and _call(f, args, ws=P + 8) == space
    if name == "moe_lora_forward":
        assert _call(f, args, flags=1) == invalid and _call(f, args, flags=B.MOE_OUT_F32 | 1 << 9) == invalid
        assert _call(f, args, T=0) == B.MOE_OK     # nothing to launch
    else:
        assert _call(f, args, dx=None) == invalid  # dx_in without dx
    assert B.moe_lora_workspace_bytes(4, 60, 128, 16, 3) == 0


BALANCE = dict(logits=P, idx=P, mask=P, T=4, E=8, k=2, counts=P, prob=P, losses=P, ws=P, nbytes=W, stream=None)
ROUTE = dict(logits=P, idx=P, dw=P, mask=P, counts=P, T=4, E=8, k=2, cb=0.1, cz=0.1, flags=0, dl=P, stream=None)


def test_balance_and_route_backward_refusals(lib):
    invalid = B.MOE_ERR_INVALID_ARG
    for f, args in ((lib.moe_balance_loss, BALANCE), (lib.moe_route_backward, ROUTE)):
        for change in (dict(T=-1), dict(E=0), dict(E=257), dict(k=0), dict(k=9), dict(E=64, k=17), dict(T=1 << 23, k=2)):
            assert _call(f, args, **change) == invalid, change
        for key in ("logits", "idx", "counts"):
            assert _call(f, args, **{key: None}) == invalid, key
    f = lib.moe_balance_loss
    assert _call(f, BALANCE, prob=None) == invalid and _call(f, BALANCE, losses=None) == invalid
    need = B.moe_balance_workspace_bytes(4, 8)
    assert need > 0 and B.moe_balance_workspace_bytes(4, 300) == 0
    for change in (dict(nbytes=need - 1), dict(ws=None), dict(ws=P + 4)):
        assert _call(f, BALANCE, **change) == B.MOE_ERR_WORKSPACE
    f = lib.moe_route_backward
    assert _call(f, ROUTE, dl=None) == invalid
    assert _call(f, ROUTE, flags=B.MOE_LOGITS_GIVEN) == invalid
    assert _call(f, ROUTE, counts=None, cb=0.0) == invalid and _call(f, ROUTE, counts=None, cz=0.0) == invalid
    assert _call(f, ROUTE, T=0, counts=None, cb=0.0, cz=0.0) == B.MOE_OK
    assert _call(f, ROUTE, cb=float("nan")) == invalid and _call(f, ROUTE, cz=float("inf")) == invalid


ROUTER = dict(x=P, w=P, dl=P, T=4, H=64, E=8, dx_in=P, dx=P, dw=P, ws=P, nbytes=W, stream=None)
COMBINE = dict(dy=P, y=P, slot=P, T=4, k=2, H=64, ys=P, x=P, ws=P, dw=P, dg=P, flags=0, stream=None)


def test_router_and_combine_backward_refusals(lib):
    invalid, shape = B.MOE_ERR_INVALID_ARG, B.MOE_ERR_UNSUPPORTED_SHAPE
    f = lib.moe_router_backward
    for change in (dict(T=-1), dict(T=1 << 24), dict(H=0), dict(H=(1 << 18) + 8), dict(E=0), dict(E=257), dict(x=None),
                   dict(dl=None), dict(dw=None), dict(w=None), dict(dx=None), dict(x=P + 8), dict(dw=P + 8), dict(dx=P + 8), dict(dx_in=P + 8)):
        assert _call(f, ROUTER, **change) == invalid, change
    assert _call(f, ROUTER, H=60) == shape
    need = B.moe_router_backward_workspace_bytes(4, 64, 8)
    assert need > 0 and B.moe_router_backward_workspace_bytes(4, 60, 8) == 0
    for change in (dict(nbytes=need - 1), dict(ws=None), dict(ws=P + 4)):
        assert _call(f, ROUTER, **change) == B.MOE_ERR_WORKSPACE
    f = lib.moe_combine_backward
    for change in (dict(T=-1), dict(T=1 << 24), dict(k=0), dict(k=17), dict(H=0), dict(H=(1 << 18) + 8),
                   dict(dy=None), dict(y=None), dict(slot=None), dict(dw=None),
                   dict(ys=None), dict(x=None), dict(ws=None), dict(dg=None), dict(flags=B.MOE_OUT_F32), dict(dy=P + 8),
                   dict(y=P + 8), dict(ys=P + 8), dict(x=P + 8), dict(ws=P + 8)):
        assert _call(f, COMBINE, **change) == invalid, change
    assert _call(f, COMBINE, H=60) == shape
    assert _call(f, COMBINE, T=0) == B.MOE_OK


def test_binding_refuses_host_tensors(lib):
    import torch
    t = torch.zeros((8, 8), dtype=torch.bfloat16)
    f, i = torch.zeros((8, 8)), torch.zeros(8, dtype=torch.int32)
    for call in (lambda: B.moe_lora_forward(t, i, 8, 8, 8, 8, 1, t, t, f, t, t, None, f),
                 lambda: B.moe_lora_backward(t, t, i, 8, 8, 8, 8, 1, t, t, f, f, None, t, f, f, f),
                 lambda: B.moe_balance_loss(f, i, None, 8, 8, 1, i, f, f, f),
                 lambda: B.moe_route_backward(f, i, f, None, i, 8, 8, 1, 0.0, 0.0, 0, f),
                 lambda: B.moe_router_backward(t, f, f, 8, 8, 8, None, t, f, f),
                 lambda: B.moe_combine_backward(t, f, i, 8, 1, 8, None, None, None, f)):
        with pytest.raises(ValueError):
            call()
