"""Operators of a training step around the heads and the losses, each in its plain form and as the framework's call.

  norm_fwd / norm_bwd        layer norm of the kept rows ahead of the heads, and its derivatives
  balance_fwd / balance_bwd  the balance loss of a mixture-of-experts policy over its policy tokens, with per-expert counts
  orthogonalize              a matrix update made orthogonal by Newton-Schulz products

The plain form computes in fp32 with elementary torch operations and rounds once at the end.  Where `own` is true, `run` makes
the calls of ``paper_2506_15050_amd.binding``; the workspaces and output buffers that a training program keeps from step to
step are made by the first of them and live in the state.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS_NORM = 1e-5
STEPS, COEFFICIENTS, EPS_ORTHO = 5, (3.4445, -4.7750, 2.0315), 1e-7
BALANCE_COEFFICIENT = 0.01


def listed():
    return [
        # the smallest call: a handful of tokens of a toy model in fp32, launches and host time are all there is
        dict(name="norm_fwd_tiny_f32", kind="norm_fwd", B=3, ctx=16, win=21, H=64, dtype="f32", bias=True),
        # the benchmark's 32B-shaped batch: all kept tokens of an update, prompts skipped
        dict(name="norm_fwd_h5120", kind="norm_fwd", B=32, ctx=1024, win=2423, H=5120, dtype="bf16", bias=True),
        # hidden size, rows and leading dimension that no vector divides, without a bias, bf16 gradients throughout
        dict(name="norm_bwd_ragged_h1001", kind="norm_bwd", B=7, ctx=37, win=359, H=1001, dtype="bf16", grad_in="bf16",
             grad_out="bf16", bias=False),
        # the benchmark's small configuration in fp32
        dict(name="norm_bwd_h1024_f32", kind="norm_bwd", B=32, ctx=256, win=513, H=1024, dtype="f32", grad_in="f32",
             grad_out="f32", bias=True),
        # a micro-batch of the 32B-shaped batch: fp32 derivatives from the LM head, bf16 ones for the trunk
        dict(name="norm_bwd_h5120", kind="norm_bwd", B=8, ctx=1024, win=2423, H=5120, dtype="bf16", grad_in="f32",
             grad_out="bf16", bias=True),
        # a micro-batch's router of one layer: eight experts, two a token
        dict(name="balance_fwd_small_e8", kind="balance_fwd", B=2, ctx=16, win=73, E=8, k=2, dtype="f32", dead=0),
        # monitoring of one layer over a whole batch, router in fp32
        dict(name="balance_fwd_e256", kind="balance_fwd", B=32, ctx=1024, win=2423, E=256, k=8, dtype="f32", dead=0),
        # an odd number of experts with places that no expert fills (-inf logits), router in bf16
        dict(name="balance_bwd_odd_e67_bf16", kind="balance_bwd", B=7, ctx=37, win=701, E=67, k=4, dtype="bf16", dead=3),
        # the update of one layer over a whole batch
        dict(name="balance_bwd_e128", kind="balance_bwd", B=32, ctx=1024, win=2423, E=128, k=8, dtype="f32", dead=0),
        # a router's own weights, [E, H] of a small model: few products, all latency
        dict(name="ortho_router_64x1024", kind="orthogonalize", count=1, rows=64, cols=1024, dtype="f32", rank=16),
        # a stack of layers' tall matrices of sizes that no tile divides
        dict(name="ortho_stack_1000x333", kind="orthogonalize", count=8, rows=1000, cols=333, dtype="f32", rank=64),
        # a square matrix of the 32B-shaped model, gradients accumulated in fp32
        dict(name="ortho_5120", kind="orthogonalize", count=1, rows=5120, cols=5120, dtype="f32", rank=256),
    ]


def _log_between(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_fwd", "norm_bwd", "balance_fwd", "balance_bwd", "orthogonalize", "orthogonalize"])
    if kind == "orthogonalize":
        rows, cols = _log_between(rng, 8, 5120), _log_between(rng, 8, 5120)
        small, large = min(rows, cols), max(rows, cols)
        most = 5120 ** 3 // (small * small * large)
        count = min(_log_between(rng, 1, 12), max(1, most), max(1, (1 << 25) // (rows * cols)))
        return dict(kind=kind, count=count, rows=rows, cols=cols, dtype=rng.choice(["f32", "bf16"]),
                    rank=max(1, small // rng.choice([1, 4, 16])))
    B, ctx = _log_between(rng, 1, 32), rng.randint(1, 1024)
    win = _log_between(rng, 1, 2423)
    if kind in ("norm_fwd", "norm_bwd"):
        H = rng.choice([64 * rng.randint(1, 80), 8 * rng.randint(1, 640), _log_between(rng, 16, 5120)])
        c = dict(kind=kind, B=B, ctx=ctx, win=win, H=H, dtype=rng.choice(["bf16", "bf16", "f32"]), bias=rng.random() < 0.7)
        if kind == "norm_bwd":
            c["win"] = min(win, max(1, 19384 // B))
            types = [("f32", "f32")] if c["dtype"] == "f32" else [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")]
            c["grad_in"], c["grad_out"] = rng.choice(types)
        return c
    E = _log_between(rng, 4, 256)
    return dict(kind=kind, B=B, ctx=ctx, win=win, E=E, k=min(E, rng.randint(1, 8)), dtype=rng.choice(["f32", "bf16"]),
                dead=rng.choice([0, 0, E // 16]))


def _kept_rows(case):
    """Rows of the states that predict the window tokens of B packed sequences: the prompt's rows but its last are not among them."""
    B, ctx, win = case["B"], case["ctx"], case["win"]
    first = torch.arange(B, device="cuda", dtype=torch.int32)[:, None] * (ctx + win) + (ctx - 1)
    return (first + torch.arange(win, device="cuda", dtype=torch.int32)).reshape(-1).contiguous()


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0, dtype=torch.float32):
        return torch.randn(*shape, device="cuda", generator=g).mul_(scale).add_(shift).to(dtype)

    s = dict(case=case, kind=case["kind"])
    if case["kind"] == "orthogonalize":
        # momentum of a weight matrix: some directions that the batches share, and noise
        n, rows, cols, r = case["count"], case["rows"], case["cols"], case["rank"]
        shared = torch.bmm(normal(n, rows, r), normal(n, r, cols, scale=1e-3 / math.sqrt(r)))
        s["g"] = (shared + normal(n, rows, cols, scale=3e-4)).to(TYPES[case["dtype"]])
        return s
    n_rows, dt = case["B"] * (case["ctx"] + case["win"]), TYPES[case["dtype"]]
    s["rows"] = _kept_rows(case)
    M = s["rows"].numel()
    if case["kind"] in ("norm_fwd", "norm_bwd"):
        H = case["H"]
        # residual stream: a mean of its own for each row, a few large channels
        x = normal(n_rows, H, scale=2.0)
        x += normal(n_rows, 1)
        x[:, :: max(1, H // 7)] *= 8.0
        s["x"] = x.to(dt)
        del x
        s["weight"] = normal(H, scale=0.2, shift=1.0, dtype=dt)
        s["bias"] = normal(H, scale=0.1, dtype=dt) if case["bias"] else None
        if case["kind"] == "norm_bwd":
            # what the forward pass left behind, and the derivatives of a token-level mean
            kept = s["x"][s["rows"].long()].float()
            s["mean"] = kept.mean(1)
            s["rstd"] = 1 / torch.sqrt((kept - s["mean"][:, None]).square().mean(1) + EPS_NORM)
            s["grad_y"] = normal(M, H, scale=1.0 / M, dtype=TYPES[case["grad_in"]])
        return s
    # router logits with experts that are liked more than others; the choices are the router's own, some tokens of which found their
    # experts full
    E, k = case["E"], case["k"]
    z = normal(n_rows, E, scale=1.5) + normal(E, scale=0.5)
    if case["dead"]:
        z[:, E - case["dead"]:] = -math.inf
    s["logits"] = z.to(dt)
    s["k"] = k
    choice = z.topk(k, dim=1).indices.to(torch.int32)
    full = torch.rand(n_rows, k, device="cuda", generator=g) < 0.02
    s["experts"] = torch.where(full, torch.full_like(choice, -1), choice).contiguous()
    return s


def _binding():
    from paper_2506_15050_amd import binding
    return binding


def _run_own(s):
    tp, kind, case = _binding(), s["kind"], s["case"]
    kept = s.get("kept")
    if kept is None:
        lib = tp.load()
        if kind == "norm_fwd":
            M, H = s["rows"].numel(), case["H"]
            kept = (torch.empty(M, H, dtype=s["x"].dtype, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, device="cuda"))
        elif kind == "norm_bwd":
            M, H = s["rows"].numel(), case["H"]
            kept = dict(out=torch.empty(M, H, dtype=TYPES[case["grad_out"]], device="cuda"),
                        grad_w=(torch.empty(H, device="cuda"), torch.empty(H, device="cuda") if case["bias"] else None),
                        workspace=tp._workspace(lib.tppo_layer_norm_backward_workspace_bytes(M, H), "cuda"))
        elif kind in ("balance_fwd", "balance_bwd"):
            M, E = s["rows"].numel(), case["E"]
            kept = dict(workspace=tp._workspace(lib.tppo_balance_loss_workspace_bytes(M, E), "cuda"))
        else:
            kept = dict(workspace=tp._workspace(lib.tppo_orthogonalize_workspace_bytes(case["count"], case["rows"], case["cols"]), "cuda"),
                        out=torch.empty(s["g"].shape, dtype=torch.bfloat16, device="cuda"))
        s["kept"] = kept
    if kind == "norm_fwd":
        y, mean, rstd = tp.tppo_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS_NORM, rows=s["rows"], out=kept)
        return dict(y=y, mean=mean, rstd=rstd)
    if kind == "norm_bwd":
        gx, gw, gb = tp.tppo_layer_norm_backward(s["grad_y"], s["x"], s["weight"], s["mean"], s["rstd"], rows=s["rows"],
                                                 want_bias=case["bias"], **kept)
        return dict(grad_x=gx, grad_weight=gw, **(dict(grad_bias=gb) if case["bias"] else {}))
    if kind == "balance_fwd":
        loss, counts, mean_prob = tp.tppo_balance_loss(s["logits"], s["experts"], rows=s["rows"], coefficient=BALANCE_COEFFICIENT, **kept)
        return dict(loss=loss, counts=counts, mean_prob=mean_prob)
    if kind == "balance_bwd":
        grad, loss, counts, mean_prob = tp.tppo_balance_loss_backward(s["logits"], s["experts"], rows=s["rows"],
                                                                      coefficient=BALANCE_COEFFICIENT, **kept)
        return dict(grad_logits=grad, loss=loss, counts=counts, mean_prob=mean_prob)
    return dict(out=tp.tppo_orthogonalize(s["g"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS_ORTHO, **kept))


def _plain_balance(s, with_grad):
    z, rows, E, k = s["logits"], s["rows"].long(), s["case"]["E"], s["k"]
    N = rows.numel()
    zr = z[rows].float()
    top = zr.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)           # a row without any expert: p = 0
    e = torch.exp(zr - top)
    total = e.sum(1, keepdim=True)
    p = e / torch.where(total == 0, torch.ones_like(total), total)
    ids = s["experts"][rows].reshape(-1).long()
    counts = torch.zeros(E + 1, dtype=torch.int64, device="cuda").index_add_(0, ids + 1, torch.ones_like(ids))[1:]
    f = counts.float() / (k * N)
    mean_prob = p.sum(0) / N
    out = dict(loss=(BALANCE_COEFFICIENT * E * (f * mean_prob).sum()).reshape(1), counts=counts, mean_prob=mean_prob)
    if with_grad:
        d = f - f.sum() / E                                                     # the p of a row add up to one
        out["grad_logits"] = ((BALANCE_COEFFICIENT * E / N) * p * (d - (p * d).sum(1, keepdim=True))).to(z.dtype)
    return out


def run(state):
    if own:
        return _run_own(state)
    s, kind = state, state["kind"]
    if kind == "norm_fwd":
        x = s["x"][s["rows"].long()].float()
        mean = x.sum(1) / x.shape[1]
        c = x - mean[:, None]
        rstd = 1 / torch.sqrt((c * c).sum(1) / x.shape[1] + EPS_NORM)
        y = c * rstd[:, None] * s["weight"].float()
        if s["bias"] is not None:
            y = y + s["bias"].float()
        return dict(y=y.to(s["x"].dtype), mean=mean, rstd=rstd)
    if kind == "norm_bwd":
        gy, H = s["grad_y"].float(), s["case"]["H"]
        xh = (s["x"][s["rows"].long()].float() - s["mean"][:, None]) * s["rstd"][:, None]
        gh = gy * s["weight"].float()
        c1, c2 = gh.sum(1, keepdim=True) / H, (gh * xh).sum(1, keepdim=True) / H
        out = dict(grad_x=(s["rstd"][:, None] * (gh - c1 - xh * c2)).to(TYPES[s["case"]["grad_out"]]), grad_weight=(gy * xh).sum(0))
        if s["case"]["bias"]:
            out["grad_bias"] = gy.sum(0)
        return out
    if kind in ("balance_fwd", "balance_bwd"):
        return _plain_balance(s, kind == "balance_bwd")
    x = s["g"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + EPS_ORTHO)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        A = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * A + c * torch.bmm(A, A), x)
    return dict(out=(x.transpose(1, 2).contiguous() if tall else x).to(torch.bfloat16))


def work(case):
    kind = case["kind"]
    size = {"bf16": 2, "f32": 4}
    if kind == "orthogonalize":
        m, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # X X^T and A A are symmetric: half of each
        return dict(bytes=case["count"] * m * n * (size[case["dtype"]] + 2), flops=case["count"] * STEPS * (m * m * n + m * m * m + 2 * m * m * n))
    M, e = case["B"] * case["win"], size[case["dtype"]]
    if kind == "norm_fwd":
        H = case["H"]
        return dict(bytes=M * H * 2 * e + M * 12 + H * e * (2 if case["bias"] else 1), flops=8 * M * H)
    if kind == "norm_bwd":
        H = case["H"]
        return dict(bytes=M * H * (e + size[case["grad_in"]] + size[case["grad_out"]]) + M * 12 + H * (e + (8 if case["bias"] else 4)),
                    flops=14 * M * H)
    E = case["E"]
    return dict(bytes=M * E * e * (2 if kind == "balance_bwd" else 1) + M * (4 * case["k"] + 4) + E * 12, flops=(10 if kind == "balance_bwd" else 5) * M * E)


def exact(case, seed):
    s = prepare(case, seed)
    kind, f64 = case["kind"], torch.float64
    if kind == "orthogonalize":
        G = s["g"].to(f64)
        if case["rows"] > case["cols"]:
            G = G.mT.contiguous()
        X = G / (torch.linalg.vector_norm(G, dim=(1, 2)) + EPS_ORTHO)[:, None, None]
        a, b, c = COEFFICIENTS
        for _ in range(STEPS):
            Y = []
            for M in X:                                                        # one matrix after the other: p(S) M with S = M M^T
                S = M.mm(M.t())
                SM = S.mm(M)
                Y.append(a * M + b * SM + c * S.mm(SM))
            X = torch.stack(Y)
        return dict(out=X.mT.contiguous() if case["rows"] > case["cols"] else X)
    rows = s["rows"].long()
    if kind in ("norm_fwd", "norm_bwd"):
        x = s["x"].index_select(0, rows).to(f64)
        if kind == "norm_fwd":
            var, mean = torch.var_mean(x, dim=1, correction=0)
            y = torch.addcmul(torch.zeros((), dtype=f64, device="cuda") if s["bias"] is None else s["bias"].to(f64),
                              (x - mean[:, None]) * (var + EPS_NORM).rsqrt()[:, None], s["weight"].to(f64))
            return dict(y=y, mean=mean, rstd=(var + EPS_NORM).rsqrt())
        gy = s["grad_y"].to(f64)
        xh = (x - s["mean"].to(f64)[:, None]).mul_(s["rstd"].to(f64)[:, None])
        gh = gy * s["weight"].to(f64)
        gx = (gh - gh.mean(1, keepdim=True) - xh * (gh * xh).mean(1, keepdim=True)) * s["rstd"].to(f64)[:, None]
        out = dict(grad_x=gx, grad_weight=(gy * xh).sum(0))
        return dict(out, grad_bias=gy.sum(0)) if case["bias"] else out
    E, k, N = case["E"], case["k"], rows.numel()
    p = torch.softmax(s["logits"].index_select(0, rows).to(f64), dim=1)
    chosen = s["experts"].index_select(0, rows).flatten()
    counts = torch.bincount(chosen[chosen >= 0].long(), minlength=E)
    f = counts.to(f64) / (k * N)
    mean_prob = p.mean(0)
    out = dict(loss=(BALANCE_COEFFICIENT * E * torch.dot(f, mean_prob)).reshape(1), counts=counts, mean_prob=mean_prob)
    if kind == "balance_bwd":
        out["grad_logits"] = BALANCE_COEFFICIENT * E / N * p * (f - p.mv(f)[:, None])
    return out
