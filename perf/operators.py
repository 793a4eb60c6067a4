"""The operators around the Expert module that a fine-tune and a server with many adapters need, as measurable cases:
low-rank adapters of many requests beside one projection (moe_lora_forward / moe_lora_backward), the router's balance and
z loss with per-expert counts and its gradient (moe_balance_loss / moe_route_backward), the gradient of the router's
product (moe_router_backward) and that of the combine's gates (moe_combine_backward).

`run` computes an operator in its plain form or, where `own` is set, by the library.  Sizes are those of
`paper_2508_19373_amd.inputs` (hidden 2048, 3584, 4096; 8, 60 or 64 experts; top 2, 4 or 8) and free token counts
between one and a long prompt batch, odd ones included; adapter ranks are 8 to 128.
"""
import math

import torch

own = False

MODELS = {  # hidden, experts, top k, renormalised gates, shared expert's intermediate size
    "tiny": (512, 8, 2, True, 0),
    "mixtral": (4096, 8, 2, True, 0),
    "qwen": (2048, 60, 4, False, 5632),
    "qwen2_57b": (3584, 64, 8, False, 20480),
}
COEF_BALANCE, COEF_Z = 0.01, 0.001


def _lora(op, tokens, K, N, rank, adapters, *, requests, bare=0.0, out_f32=False, save=False):
    """requests: how many runs of rows the batch has (0: every row a request of its own); bare: share without an adapter."""
    case = dict(op=op, tokens=tokens, K=K, N=N, rank=rank, adapters=adapters, requests=requests, bare=bare)
    return dict(case, out_f32=out_f32, save=save) if op == "lora" else case


def listed():
    return [
        # one token of one request: two short kernels, bound by launches and latency
        dict(_lora("lora", 1, 4096, 4096, 16, 8, requests=0), name="lora_decode_1"),
        # a decoding step of a full batch, adapters in any order: every active adapter is read once
        dict(_lora("lora", 48, 4096, 4096, 16, 32, requests=0, bare=0.1), name="lora_decode_48"),
        # prompts of a dozen requests beside the unsharded layer
        dict(_lora("lora", 4096, 4096, 4096, 32, 8, requests=12), name="lora_prompts_4096"),
        # training forward beside a shared expert's down projection: fp32 result, rows without an adapter, v kept
        dict(_lora("lora", 1111, 5632, 2048, 64, 6, requests=9, bare=0.2, out_f32=True, save=True),
             name="lora_shared_down_1111"),
        # a small training step of a few adapters on a narrow layer
        dict(_lora("lora_backward", 777, 2048, 2048, 8, 4, requests=7, bare=0.1), name="lora_backward_777"),
        # a full training batch of eight adapters
        dict(_lora("lora_backward", 8192, 4096, 4096, 64, 8, requests=16), name="lora_backward_8192"),
        # the loss of a small batch and its gradient: latency
        dict(op="router_loss", model="tiny", tokens=64, padded=False, name="router_loss_64"),
        # that of a long padded batch of the model with the most experts
        dict(op="router_loss", model="qwen2_57b", tokens=16384, padded=True, name="router_loss_16384"),
        # gradient of the router's product: a ragged batch of many experts, ...
        dict(op="router_backward", model="qwen", tokens=333, chain=True, name="router_backward_333"),
        # ... and a full one
        dict(op="router_backward", model="qwen2_57b", tokens=8192, chain=False, name="router_backward_8192"),
        # gradient of the gates: a few tokens with a shared expert, ...
        dict(op="combine_backward", model="qwen", tokens=32, ep=1, y_perm_bf16=False, name="combine_backward_32"),
        # ... and a prompt batch of the widest rows
        dict(op="combine_backward", model="mixtral", tokens=4096, ep=1, y_perm_bf16=False, name="combine_backward_4096"),
    ]


def draw(rng):
    limit = max(_cost(c) for c in listed())

    def tokens(top):
        return int(2.0 ** rng.uniform(0.0, math.log2(top)))

    while True:
        op = rng.choice(["lora", "lora", "lora_backward", "router_loss", "router_backward", "combine_backward"])
        if op.startswith("lora"):
            T = tokens(8192)
            width = lambda: rng.choice([512, 1408, 2048, 3584, 4096, 5632, 8 * rng.randint(8, 700)])  # noqa: E731
            case = _lora(op, T, width(), width(), rng.choice([8, 16, 16, 24, 32, 48, 64, 128]), rng.randint(1, 40),
                         requests=rng.choice([0, rng.randint(1, 24)]), bare=rng.choice([0.0, 0.0, 0.1, 0.5]),
                         **(dict(out_f32=rng.random() < 0.4, save=rng.random() < 0.3) if op == "lora" else {}))
        else:
            model = rng.choice(["tiny", "mixtral", "qwen", "qwen2_57b"])
            if op == "router_loss":
                case = dict(op=op, model=model, tokens=tokens(16384), padded=rng.random() < 0.5)
            elif op == "router_backward":
                case = dict(op=op, model=model, tokens=tokens(8192), chain=rng.random() < 0.5)
            else:
                case = dict(op=op, model=model, tokens=tokens(8192), ep=rng.choice([1, 1, 2, 4]),
                            y_perm_bf16=rng.random() < 0.4)
        if _cost(case) <= limit:
            return case


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def _adapter_ids(case, g):
    """int32 [T]: runs of rows of one request each, or every row its own; -1 for requests without an adapter."""
    T, L, runs = case["tokens"], case["adapters"], case["requests"]
    n = T if runs == 0 else min(runs, T)
    ids = torch.randint(0, L, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids = torch.where(torch.rand((n,), generator=g, device="cuda") < case["bare"], torch.full_like(ids, -1), ids)
    if runs == 0:
        return ids
    ends = torch.sort(torch.randint(0, T + 1, (n - 1,), generator=g, device="cuda")).values
    return ids[torch.searchsorted(ends, torch.arange(T, device="cuda"), right=True)].contiguous()


def prepare_lora(case, seed):
    g, T, K, N, r, L = _generator(seed), case["tokens"], case["K"], case["N"], case["rank"], case["adapters"]
    dt = torch.float32 if case.get("out_f32") else torch.bfloat16
    s = dict(case, x=_normal(g, (T, K), 1.0, torch.bfloat16), idx=_adapter_ids(case, g),
             a=_normal(g, (L, r, K), K ** -0.5, torch.bfloat16), b=_normal(g, (L, N, r), 0.05, torch.bfloat16),
             scale=torch.empty((L,), device="cuda").uniform_(0.5, 2.0, generator=g))
    if case["op"] == "lora":
        s["y"] = _normal(g, (T, N), 1.0, dt)
        s["out"] = torch.empty((T, N), dtype=dt, device="cuda")
        s["v"] = torch.empty((T, r), device="cuda") if case["save"] else None
    else:
        s["dy"] = _normal(g, (T, N), 1.0 / T, torch.bfloat16)
        s["v"] = _normal(g, (T, r))  # of the order that x and A above give
        s["v"] *= (s["idx"] >= 0).unsqueeze(1)
        s["dx"] = torch.empty((T, K), dtype=torch.bfloat16, device="cuda")
        s["grad_a"] = torch.empty((L, r, K), device="cuda")
        s["grad_b"] = torch.empty((L, N, r), device="cuda")
    return s


def prepare(case, seed):
    if case["op"].startswith("lora"):
        return prepare_lora(case, seed)
    g, T = _generator(seed), case["tokens"]
    H, E, k, renorm, shared = MODELS[case["model"]]
    s = dict(case, H=H, E=E, k=k, renorm=renorm)
    if case["op"] == "router_loss":
        s["logits"] = _normal(g, (T, E), 1.3) + _normal(g, (E,), 0.5)  # some experts are liked better
        s["topk_idx"] = torch.topk(s["logits"], k, dim=1).indices.int()
        s["d_topk_w"] = _normal(g, (T, k), 0.01 / T)
        s["mask"] = None
        if case["padded"]:  # sequences of 256 rows at most, padded on the right
            length = torch.randint(1, 257, ((T + 255) // 256,), generator=g, device="cuda")
            row = torch.arange(T, device="cuda")
            s["mask"] = (row % 256 < length[row // 256]).to(torch.uint8)
        s["counts"] = torch.empty((E + 1,), dtype=torch.int32, device="cuda")
        s["mean_prob"] = torch.empty((E,), device="cuda")
        s["losses"] = torch.empty((2,), device="cuda")
        s["d_logits"] = torch.empty((T, E), device="cuda")
    elif case["op"] == "router_backward":
        s["x"] = _normal(g, (T, H), 1.0, torch.bfloat16)
        s["w_router"] = _normal(g, (H, E), 0.02)
        s["d_logits"] = _normal(g, (T, E), 0.1 / T)
        s["dx_in"] = _normal(g, (T, H), 0.01 / T, torch.bfloat16) if case["chain"] else None
        s["dx"] = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
        s["d_w_router"] = torch.empty((H, E), device="cuda")
    else:
        dt = torch.bfloat16 if case["y_perm_bf16"] else torch.float32
        # where moe_permute puts the assignments of this device's experts: behind each other by expert, -1 for the others
        expert = torch.rand((T, E), generator=g, device="cuda").topk(k, dim=1).indices.reshape(-1)
        local = expert < E // case["ep"]
        order = torch.sort(torch.where(local, expert, E), stable=True).indices
        rows = torch.empty_like(order)
        rows[order] = torch.arange(T * k, device="cuda")
        s["slot_row"] = torch.where(local, rows, -1).int()
        s["y_perm"] = _normal(g, (T * k, H), 0.5, dt)
        s["dy"] = _normal(g, (T, H), 1.0 / T, torch.bfloat16)
        s["d_topk_w"] = torch.empty((T, k), device="cuda")
        s["y_shared"] = s["x"] = s["w_gate"] = s["d_gate"] = None
        if shared:
            s["y_shared"] = _normal(g, (T, H), 0.5, dt)
            s["x"] = _normal(g, (T, H), 1.0, torch.bfloat16)
            s["w_gate"] = _normal(g, (H,), 0.02)
            s["d_gate"] = torch.empty((T,), device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ the operators
def run(s):
    return (run_own if own else run_plain)(s)


def _workspace(s, size, *args):
    """The scratch buffer of these sizes, allocated once as a program that makes the call again keeps it."""
    if s.get("workspace") is None:
        s["workspace"] = torch.empty(max(size(*args), 256), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def run_own(s):
    from paper_2508_19373_amd import binding as B
    if s["op"].startswith("lora"):
        sizes = tuple(s[n] for n in ("tokens", "K", "N", "rank", "adapters"))
        ws = _workspace(s, B.moe_lora_workspace_bytes, *sizes, s["op"] == "lora_backward")
    if s["op"] == "lora":
        B.moe_lora_forward(s["x"], s["idx"], *sizes, s["a"], s["b"], s["scale"], s["y"], s["out"], s["v"], ws,
                           B.MOE_OUT_F32 if s["out_f32"] else 0)
        return {"y": s["out"], "v": s["v"]}
    if s["op"] == "lora_backward":
        B.moe_lora_backward(s["x"], s["dy"], s["idx"], *sizes, s["a"], s["b"], s["scale"], s["v"], None, s["dx"],
                            s["grad_a"], s["grad_b"], ws)
        return {"dx": s["dx"], "grad_a": s["grad_a"], "grad_b": s["grad_b"]}
    if s["op"] == "router_loss":
        B.moe_balance_loss(s["logits"], s["topk_idx"], s["mask"], s["tokens"], s["E"], s["k"], s["counts"],
                           s["mean_prob"], s["losses"], _workspace(s, B.moe_balance_workspace_bytes, s["tokens"], s["E"]))
        B.moe_route_backward(s["logits"], s["topk_idx"], s["d_topk_w"], s["mask"], s["counts"], s["tokens"], s["E"],
                             s["k"], COEF_BALANCE, COEF_Z, B.MOE_RENORM_TOPK if s["renorm"] else 0, s["d_logits"])
        return {n: s[n] for n in ("counts", "mean_prob", "losses", "d_logits")}
    if s["op"] == "router_backward":
        B.moe_router_backward(s["x"], s["w_router"], s["d_logits"], s["tokens"], s["H"], s["E"], s["dx_in"], s["dx"],
                              s["d_w_router"],
                              _workspace(s, B.moe_router_backward_workspace_bytes, s["tokens"], s["H"], s["E"]))
        return {"dx": s["dx"], "d_w_router": s["d_w_router"]}
    B.moe_combine_backward(s["dy"], s["y_perm"], s["slot_row"], s["tokens"], s["k"], s["H"], s["y_shared"], s["x"],
                           s["w_gate"], s["d_topk_w"], s["d_gate"], B.MOE_Y_PERM_BF16 if s["y_perm_bf16"] else 0)
    return {"d_topk_w": s["d_topk_w"], "d_gate": s["d_gate"]}


def run_plain(s):
    if s["op"].startswith("lora"):
        return plain_lora(s)
    if s["op"] == "router_loss":
        return plain_router_loss(s)
    if s["op"] == "router_backward":
        dl = s["d_logits"]
        dx = dl @ s["w_router"].t()
        if s["dx_in"] is not None:
            dx = dx + s["dx_in"].float()
        return {"dx": dx.bfloat16(), "d_w_router": s["x"].float().t() @ dl}
    T, k = s["tokens"], s["k"]
    dy, rows = s["dy"].float(), s["slot_row"].long()
    picked = s["y_perm"][rows.clamp(min=0)].float() * (rows >= 0).unsqueeze(1)
    d_topk_w = (picked.view(T, k, -1) * dy.unsqueeze(1)).sum(2)
    d_gate = None
    if s["y_shared"] is not None:
        gate = torch.sigmoid(s["x"].float() @ s["w_gate"])
        d_gate = gate * (1 - gate) * (dy * s["y_shared"].float()).sum(1)
    return {"d_topk_w": d_topk_w, "d_gate": d_gate}


def plain_lora(s):
    """All adapters as one wide product whose columns of other adapters are zeroed for each row."""
    T, K, N, r, L = s["tokens"], s["K"], s["N"], s["rank"], s["adapters"]
    mine = (s["idx"].unsqueeze(1) == torch.arange(L, device="cuda")).float()  # [T, L]
    x, a, b = s["x"].float(), s["a"].float().view(L * r, K), s["b"].float().transpose(1, 2).reshape(L * r, N)
    scaled = (mine * s["scale"]).repeat_interleave(r, dim=1)                     # [T, L r]
    if s["op"] == "lora":
        v = x @ a.t()
        y = (s["y"].float() + (v * scaled) @ b).to(s["out"].dtype)
        return {"y": y, "v": (v.view(T, L, r) * mine.unsqueeze(2)).sum(1) if s["save"] else None}
    dy = s["dy"].float()
    u = (dy @ b.t()) * scaled
    wide = s["v"].repeat(1, L) * scaled
    return {"dx": (u @ a).bfloat16(), "grad_a": (u.t() @ x).view(L, r, K),
            "grad_b": (wide.t() @ dy).view(L, r, N).transpose(1, 2).contiguous()}


def plain_router_loss(s):
    logits, idx, T, E, k = s["logits"], s["topk_idx"].long(), s["tokens"], s["E"], s["k"]
    valid = torch.ones((T, 1), device="cuda") if s["mask"] is None else (s["mask"] != 0).float().unsqueeze(1)
    picked = (idx.unsqueeze(2) == torch.arange(E, device="cuda")).float()       # [T, k, E]
    per_expert = (picked.sum(1) * valid).sum(0)
    n = valid.sum()
    counts = torch.cat([per_expert, n.view(1)]).round().int()
    top = logits.max(1, keepdim=True).values
    e = (logits - top).exp()
    total = e.sum(1, keepdim=True)
    p, lse = e / total, top + total.log()
    many = n.clamp(min=1.0)
    mean_prob = (p * valid).sum(0) / many
    losses = torch.stack([E / (k * many) * (per_expert * mean_prob).sum(), (lse.square() * valid).sum() / many])
    # gates: softmax over the picked logits alone where they are renormalised, over all of them else
    dw = (picked * s["d_topk_w"].unsqueeze(2)).sum(1)                           # [T, E]
    if s["renorm"]:
        w = e * picked.sum(1)
        w = w / w.sum(1, keepdim=True)
    else:
        w = p
    d = w * (dw - (w * dw).sum(1, keepdim=True))
    load = COEF_BALANCE * E / k * per_expert / many.square()
    aux = p * (load - (p * load).sum(1, keepdim=True)) + p * lse * (2 * COEF_Z / many)
    return {"counts": counts, "mean_prob": mean_prob, "losses": losses, "d_logits": d + aux * valid}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    s = {n: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for n, v in s.items()}
    if case["op"].startswith("lora"):
        return exact_lora(s)
    if case["op"] == "router_loss":
        return exact_router_loss(s)
    if case["op"] == "router_backward":
        dx = torch.matmul(s["w_router"], s["d_logits"].t()).t()
        return {"dx": dx if s["dx_in"] is None else dx + s["dx_in"], "d_w_router": torch.matmul(s["d_logits"].t(), s["x"]).t()}
    T, k = s["tokens"], s["k"]
    rows = s["slot_row"].long().view(T, k)
    out = torch.zeros((T, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        here = torch.nonzero(rows[:, j] >= 0).flatten()
        out[here, j] = torch.linalg.vecdot(s["dy"][here], s["y_perm"][rows[here, j]])
    if s["y_shared"] is None:
        return {"d_topk_w": out, "d_gate": None}
    z = torch.mv(s["x"], s["w_gate"])
    return {"d_topk_w": out, "d_gate": torch.linalg.vecdot(s["dy"], s["y_shared"]) / (2 + torch.exp(z) + torch.exp(-z))}


def exact_lora(s):
    r, forward = s["rank"], s["op"] == "lora"
    if forward:
        y, v = s["y"].clone(), torch.zeros((s["tokens"], r), dtype=torch.float64, device="cuda")
    else:
        dx, da, db = (torch.zeros(shape, dtype=torch.float64, device="cuda") for shape in (s["x"].shape, s["a"].shape, s["b"].shape))
    for i in range(s["adapters"]):
        rows = torch.nonzero(s["idx"] == i).flatten()
        a, b, c, x = s["a"][i], s["b"][i], s["scale"][i], s["x"][rows]
        if forward:
            v[rows] = torch.matmul(x, a.t())
            y[rows] += c * torch.matmul(v[rows], b.t())
        else:
            dy = s["dy"][rows]
            u = c * torch.matmul(dy, b)
            dx[rows] = torch.matmul(u, a)
            da[i] = torch.matmul(u.t(), x)
            db[i] = c * torch.matmul(dy.t(), s["v"][rows])
    return {"y": y, "v": v if s["save"] else None} if forward else {"dx": dx, "grad_a": da, "grad_b": db}


def exact_router_loss(s):
    """The gradient by torch's own differentiation of the scalar that a training step would minimise."""
    T, E, k, idx = s["tokens"], s["E"], s["k"], s["topk_idx"].long()
    valid = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"].bool()
    n = int(valid.sum())
    per_expert = torch.bincount(idx[valid].flatten(), minlength=E)
    logits = s["logits"].clone().requires_grad_(True)
    with torch.enable_grad():
        p = torch.softmax(logits, 1)
        gates = torch.gather(p, 1, idx)
        if s["renorm"]:
            gates = gates / gates.sum(1, keepdim=True)
        mean_prob = p[valid].sum(0) / max(n, 1)
        balance = E / (k * max(n, 1)) * torch.dot(per_expert.double(), mean_prob)
        z = torch.logsumexp(logits, 1)[valid].square().sum() / max(n, 1)
        (COEF_BALANCE * balance + COEF_Z * z + (gates * s["d_topk_w"]).sum()).backward()
    return {"counts": torch.cat([per_expert, torch.tensor([n], device="cuda")]).int(), "mean_prob": mean_prob.detach(),
            "losses": torch.stack([balance, z]).detach(), "d_logits": logits.grad}


# ------------------------------------------------------------------------------------------------ what cannot be done without
def work(case):
    T = case["tokens"]
    if case["op"].startswith("lora"):
        K, N, r, L = case["K"], case["N"], case["rank"], case["adapters"]
        rows, n = T * (1.0 - case["bare"]), case["requests"] or T
        active = L * (1.0 - (1.0 - (1.0 - case["bare"]) / L) ** min(n, T))     # expected
        weights = active * 2.0 * r * (K + N) + 4.0 * T
        if case["op"] == "lora":
            nbytes = 2.0 * rows * K + (4.0 if case["out_f32"] else 2.0) * 2.0 * T * N + weights
            return {"bytes": nbytes + (4.0 * T * r if case["save"] else 0.0), "flops": 2.0 * rows * r * (K + N)}
        nbytes = 2.0 * rows * (K + N) + 2.0 * T * K + 4.0 * rows * r + weights + 4.0 * L * r * (K + N)
        return {"bytes": nbytes, "flops": 4.0 * rows * r * (K + N)}
    H, E, k, _, shared = MODELS[case["model"]]
    if case["op"] == "router_loss":
        return {"bytes": 8.0 * T * E + 8.0 * T * k + 8.0 * E, "flops": 20.0 * T * E}
    if case["op"] == "router_backward":
        return {"bytes": (6.0 if case["chain"] else 4.0) * T * H + 4.0 * T * E + 8.0 * H * E, "flops": 4.0 * T * H * E}
    y = 2.0 if case["y_perm_bf16"] else 4.0
    nbytes = 2.0 * T * H + T * k / case["ep"] * H * y + 8.0 * T * k + (T * H * (y + 2.0) + 4.0 * H + 4.0 * T if shared else 0.0)
    return {"bytes": nbytes, "flops": 2.0 * T * H * (k / case["ep"] + (2 if shared else 0))}


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1e14
