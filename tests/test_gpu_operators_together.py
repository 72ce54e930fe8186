"""The layer norm, the balance loss and the orthogonalisation as a training step uses them, with the calls around them, each result against
the oracle in 64 bits of what the step handed to it; the step captured and replayed; calls side by side on two streams, two captured
calls that share a workspace; addresses whose offsets need more than 32 bits; the longest rows and sides."""
import numpy as np
import pytest
import torch

from oracle import fast as ofast
from oracle import operators as oops
from paper_2506_15050_amd import binding as tp
from paper_2506_15050_amd import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F = torch.bfloat16, torch.float32
# the arithmetic in fp32: sums over a row of H <= 1024 (a thread's 128 terms and 12 steps between lanes) and a handful of roundings, against
# the sizes of the terms: 160 U < 2^-16
ROW = 2.0 ** -16


def _host(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, size, half, what):
    worst = (np.abs(got - want) / (half * np.abs(want) + size + 1e-30)).max()
    assert worst <= 1, (what, worst)


def _batch(seed):
    b = synth.make_batch("tiny", dtype="bf16", H=192, V=1000, seed=seed)
    rng = np.random.default_rng(seed)
    up = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", t)                          # noqa: E731
    bits = lambda a: torch.from_numpy(a.view(np.int16)).view(BF).cuda()                                # noqa: E731
    H, E, k = 192, 40, 4
    ids = rng.integers(0, E, size=(b["n_tok"], k))
    ids[rng.random(ids.shape) < 0.1] = -1
    return dict(b=b, hidden=bits(b["hidden"]), w_head=bits(b["w_head"]), gain=up(1 + 0.2 * rng.normal(size=H), BF),
                shift=up(0.1 * rng.normal(size=H), BF), router=up(rng.normal(size=(b["n_tok"], E)), F), experts=up(ids, torch.int32),
                w_value=up(rng.normal(size=H) / H, BF), v_old=up(b["values"], F), ret=up(rng.normal(size=b["n_resp"]), F),
                adv=up(rng.normal(size=b["n_resp"]), F),
                **{n: up(b[n], torch.int32) for n in ("cu_seqlens", "ctx_len", "done", "resp_off", "input_ids")})


def _select(d):
    return tp.tppo_select(d["cu_seqlens"], d["ctx_len"], d["done"], d["input_ids"], d["b"]["tail_drop"], want_plan=True)


def _step(d, sel, M):
    """One update of the trunk's end: filter's rows -> norm -> heads -> losses and their derivatives -> heads' -> norm's, the router's
    loss on the same rows, the head's gradient made orthogonal."""
    b, r = d["b"], {}
    rows, targets, at = sel["sel_rows"][:M], sel["sel_targets"][:M], sel["sel_resp_idx"][:M]
    compact = torch.arange(M, dtype=torch.int32, device="cuda")
    r["y"], r["mean"], r["rstd"] = tp.tppo_layer_norm(d["hidden"], d["gain"], d["shift"], rows=sel["sel_rows"], m_actual=sel["counts"])
    r["logp"], r["lse"] = tp.tppo_token_logprobs(r["y"], d["w_head"], compact, targets, out_index=at, out_size=b["n_resp"])
    r["v"] = tp.tppo_value_head(r["y"], d["w_value"], 0.1, rows=compact, out_index=at, out_size=b["n_resp"], out=d["v_old"].clone())
    old = r["logp"] - 0.05
    r["g_logp"], r["g_v"], _, _ = tp.tppo_ppo_losses_backward(r["logp"], old, d["adv"], r["v"], d["v_old"], d["ret"], d["resp_off"],
                                                              sel["keep_len"], d["done"], 0.2, 0.28, 0.5, 0.6, plan=sel["plan"])
    r["g_y"], r["g_head"] = tp.tppo_token_logprobs_backward(r["y"], d["w_head"], compact, targets, r["lse"], r["g_logp"], in_index=at)
    r["g_hidden"] = torch.zeros_like(d["hidden"])
    _, r["g_gain"], r["g_shift"] = tp.tppo_layer_norm_backward(r["g_y"], d["hidden"], d["gain"], r["mean"], r["rstd"], rows=rows,
                                                               out=r["g_hidden"], out_index=rows)
    r["g_router"] = torch.zeros_like(d["router"])
    _, r["balance"], r["used"], r["mean_prob"] = tp.tppo_balance_loss_backward(d["router"], d["experts"], rows=rows, coefficient=0.01,
                                                                               grad=r["g_router"], out_index=rows)
    r["update"] = tp.tppo_orthogonalize(r["g_head"], scale=0.2)
    return r


@pytest.mark.parametrize("seed", [0, 5])
def test_update_step(seed):
    d = _batch(seed)
    sel = _select(d)
    M = int(sel["counts"][0])
    r = _step(d, sel, M)
    b, rows = d["b"], sel["sel_rows"][:M].cpu().numpy()
    x, w, sh = _host(d["hidden"]), _host(d["gain"]), _host(d["shift"])
    H = x.shape[1]
    oy, om, os_ = oops.layer_norm(x, w, sh, float(np.float32(1e-5)), rows)
    y, mean, rstd = (_host(r[n])[:M] for n in ("y", "mean", "rstd"))
    xh = np.abs(x[rows] - om[:, None]) * os_[:, None]
    _close(mean, om, ROW * np.abs(x[rows]).mean(1), U, "mean")
    _close(rstd, os_, ROW * os_, U, "rstd")
    _close(y, oy, ROW * ((2 + xh) * np.abs(w) + np.abs(sh)), 2.0 ** -8, "y")
    # the head's derivatives: what dz is rounded to, 2^-9 of each term, and twice that (the log-sum-exp is the device's)
    g = _host(r["g_logp"])[sel["sel_resp_idx"][:M].cpu().numpy()]
    assert np.abs(g).max() > 0
    gy, g_head, a_y, a_head = ofast.token_logprob_grads(y, b["w_head"], np.arange(M), sel["sel_targets"][:M].cpu().numpy(), g,
                                                        return_abs_bounds=True)
    _close(_host(r["g_y"]), gy, 2.0 ** -8 * a_y + 1e-6 * a_y.max(), 0, "g_y")
    _close(_host(r["g_head"]), g_head, 2.0 ** -8 * a_head + 1e-6 * a_head.max(), 0, "g_head")
    # the norm's, from what it was given
    gy = _host(r["g_y"])
    gx, gw, gb = oops.layer_norm_backward(gy, x, w, mean, rstd, rows)
    gyw, xh = np.abs(gy * w), np.abs(x[rows] - mean[:, None]) * rstd[:, None]
    size = rstd[:, None] * (gyw + gyw.mean(1, keepdims=True) + xh * (gyw * xh).mean(1, keepdims=True))
    got = _host(r["g_hidden"])
    _close(got[rows], gx, 2 * ROW * size, 2.0 ** -8, "g_hidden")
    assert not got[np.setdiff1d(np.arange(len(got)), rows)].any()
    _close(_host(r["g_gain"]), gw, (M + 20) * U * (np.abs(gy) * xh).sum(0), U, "g_gain")
    _close(_host(r["g_shift"]), gb, (M + 20) * U * np.abs(gy).sum(0), U, "g_shift")
    # the router's: logits of a few units, exponents rounded at that size, sums of M rows
    z, ids, c = _host(d["router"]), d["experts"].cpu().numpy(), float(np.float32(0.01))
    loss, counts, mean_prob = oops.balance_loss(z, ids, c, rows)
    og = oops.balance_loss_backward(z, ids, c, 1.0, rows)
    p, f = oops.softmax_rows(z[rows]), counts / (4 * M)
    away = np.abs(f - f.mean())
    assert np.array_equal(r["used"].cpu().numpy(), counts)
    _close(_host(r["mean_prob"]), mean_prob, (M + 128) * U * mean_prob, U, "mean_prob")
    assert abs(float(r["balance"]) - loss) <= (M + 132) * U * loss
    got = _host(r["g_router"])
    _close(got[rows], og, 256 * U * c * 40 / M * p * (away + (p * away).sum(1, keepdims=True) + f.mean()), U, "g_router")
    assert not got[np.setdiff1d(np.arange(len(got)), rows)].any()
    # the update: 2^-8 of the norm, rounding to bf16 and the products' operands together
    want = oops.orthogonalize(_host(r["g_head"]), scale=float(np.float32(0.2)))
    got = _host(r["update"])
    assert np.linalg.norm(got - want) <= 2.0 ** -8 * np.linalg.norm(want)


def test_update_step_captured():
    d = _batch(3)
    sel = _select(d)
    M = int(sel["counts"][0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(d, sel, M)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = _step(d, sel, M)
    for k in range(3):
        d["hidden"].normal_()
        d["router"].normal_()
        d["experts"].random_(-1, 40)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in kept.items()}
        for t in kept.values():
            t.fill_(3)
        now = _step(d, sel, M)
        for n, t in now.items():
            a, e = (got[n][:M], t[:M]) if n in ("y", "mean", "rstd") else (got[n], t)
            if n in ("logp", "lse"):                 # (written where a kept token is)
                at = sel["sel_resp_idx"][:M].long()
                a, e = a[at], e[at]
            assert torch.equal(a, e), (k, n)


def _calls(rng, shift):
    """Inputs of one call of each operator, and the calls; sizes that leave room on the chip for others."""
    up = lambda a, t=F: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", t)                        # noqa: E731
    x, w, gy = up(rng.normal(size=(700, 520 + shift))), up(rng.normal(size=520 + shift)), up(rng.normal(size=(700, 520 + shift)))
    z, ids = up(rng.normal(size=(5000, 70 + shift))), up(rng.integers(0, 70, size=(5000, 3)), torch.int32)
    g, large = up(rng.normal(size=(2, 90 + shift, 300))), up(rng.normal(size=(640 + 8 * shift, 700)))

    def run():
        y, mean, rstd = tp.tppo_layer_norm(x, w)
        out = [y, mean, rstd, *tp.tppo_layer_norm_backward(gy, x, w, mean, rstd)]
        out += [*tp.tppo_balance_loss(z, ids), *tp.tppo_balance_loss_backward(z, ids)]
        return out + [tp.tppo_orthogonalize(g), tp.tppo_orthogonalize(large), tp.tppo_orthogonalize(large, steps=7)]
    return run


def test_two_streams_at_once():
    rng = np.random.default_rng(12)
    runs = [_calls(rng, 0), _calls(rng, 3)]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    got = []
    for _ in range(4):
        for s, run in zip(streams, runs):
            with torch.cuda.stream(s):
                got.append(run())
    torch.cuda.synchronize()
    for i, results in enumerate(got):
        assert all(torch.equal(a, e) for a, e in zip(results, want[i % 2])), i


def test_two_graphs_of_one_workspace():
    """Captured one after the other with the same scratch memory, replayed in turn."""
    lib = tp.load()
    z, ids = torch.randn(3000, 50, device="cuda"), torch.randint(0, 50, (3000, 2), dtype=torch.int32, device="cuda")
    x, w = torch.randn(900, 264, device="cuda"), torch.randn(264, device="cuda")
    g = torch.randn(3, 200, 270, device="cuda")
    y, mean, rstd = tp.tppo_layer_norm(x, w)
    ws = tp._workspace(max(lib.tppo_orthogonalize_workspace_bytes(3, 200, 270), lib.tppo_balance_loss_workspace_bytes(3000, 50),
                           lib.tppo_layer_norm_backward_workspace_bytes(900, 264)), "cuda")
    calls = [lambda: tp.tppo_balance_loss_backward(z, ids, workspace=ws),
             lambda: tp.tppo_layer_norm_backward(x, x, w, mean, rstd, workspace=ws),
             lambda: (tp.tppo_orthogonalize(g, workspace=ws),)]
    want = [[t.clone() for t in call()] for call in calls]
    torch.cuda.synchronize()
    graphs, kept = [], []
    for call in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept.append(call())
        graphs.append(graph)
    for order in ((0, 1, 2), (2, 1, 0), (1, 1, 0), (0, 2, 0)):
        for t in (t for out in kept for t in out):
            t.fill_(1)
        for i in order:
            graphs[i].replay()
            calls[i]()
        torch.cuda.synchronize()
        for i in order:
            assert all(torch.equal(a, e) for a, e in zip(kept[i], want[i])), (order, i)


def test_offsets_beyond_32_bits():
    """Rows 1.3e9 elements apart: the last of three begins beyond 2^31 of them, 2^32 bytes."""
    far, H = 1_300_000_000, 200
    flat = torch.empty(2 * far + H, dtype=BF, device="cuda")
    x = flat.as_strided((3, H), (far, 1))
    x.copy_(torch.randn(3, H, device="cuda"))
    near, w = x.contiguous(), torch.randn(H, device="cuda", dtype=BF)
    rows = torch.tensor([2, 0, 2, 1], dtype=torch.int32, device="cuda")
    want = tp.tppo_layer_norm(near, w, rows=rows)
    got = tp.tppo_layer_norm(x, w, rows=rows)
    assert all(torch.equal(a, e) for a, e in zip(got, want))
    gy = torch.randn(4, H, device="cuda", dtype=BF)
    want_b = tp.tppo_layer_norm_backward(gy, near, w, *want[1:], rows=rows)
    got_b = tp.tppo_layer_norm_backward(gy, x, w, *want[1:], rows=rows)
    assert all(torch.equal(a, e) for a, e in zip(got_b, want_b))
    ids = torch.randint(0, H, (3, 4), dtype=torch.int32, device="cuda")
    want_z, got_z = (tp.tppo_balance_loss_backward(t, ids, rows=rows) for t in (near, x))
    assert all(torch.equal(a, e) for a, e in zip(got_z, want_z))
    assert torch.equal(tp.tppo_orthogonalize(x), tp.tppo_orthogonalize(near))
    # and written so far apart
    first, third = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda")
    y = tp.tppo_layer_norm(near, w)
    tp.tppo_layer_norm(near, w, out=(x, None, None))
    assert torch.equal(x, y[0])
    tp.tppo_layer_norm_backward(gy[:3], near, w, *y[1:], out=x, out_index=third, want_w=False)
    assert torch.equal(x[third.long()], tp.tppo_layer_norm_backward(gy[:3], near, w, *y[1:], want_w=False)[0])
    tp.tppo_balance_loss_backward(near, ids, grad=x, out_index=first)
    assert torch.equal(x, tp.tppo_balance_loss_backward(near, ids)[0])
    tp.tppo_orthogonalize(near, out=x)
    assert torch.equal(x, tp.tppo_orthogonalize(near))


def test_only_the_bias_is_wanted():
    x, w, gy = torch.randn(30, 72, device="cuda"), torch.randn(72, device="cuda"), torch.randn(30, 72, device="cuda")
    _, mean, rstd = tp.tppo_layer_norm(x, w)
    full = tp.tppo_layer_norm_backward(gy, x, w, mean, rstd)
    alone = tp.tppo_layer_norm_backward(gy, x, w, mean, rstd, want_x=False, want_w=False, want_bias=True)
    assert alone[0] is None and alone[1] is None and torch.equal(alone[2], full[2])
    kept = (torch.ones(72, device="cuda"), torch.ones(72, device="cuda"))
    some = tp.tppo_layer_norm_backward(gy, x, w, mean, rstd, want_x=False, want_w=False, want_bias=True, grad_w=kept, accumulate_w=True)
    assert some[1] is None and bool((kept[0] == 1).all()) and torch.equal(kept[1], 1 + full[2])
    none = tp.tppo_layer_norm_backward(gy, x, w, mean, rstd, want_x=False, want_w=False, accumulate_w=True)
    assert none == (None, None, None)


@pytest.mark.parametrize("rows,cols", [(1, 65536), (65536, 3), (64, 65536), (65536, 100), (300, 40000), (2100, 20000)])
def test_long_sides(rows, cols):
    """Against the iteration in 64 bits on the device, to 2^-8 of the norm."""
    g = torch.randn(rows, cols, device="cuda")
    out = tp.tppo_orthogonalize(g).double()
    x = g.double()
    x = x.t().contiguous() if rows > cols else x
    x = x / (x.norm() + 1e-7)
    for _ in range(5):
        s = x @ x.t()
        x = 3.4445 * x + (-4.7750 * s + 2.0315 * (s @ s)) @ x
    x = x.t() if rows > cols else x
    assert float((out - x).norm() / x.norm()) <= 2.0 ** -8


@pytest.mark.parametrize("rows,cols", [(2, 3), (17, 40), (90, 64), (100, 333), (300, 200), (600, 700), (1100, 1200)])
def test_singular_values_of_every_size(rows, cols):
    """From 1 down to 1e-6 of the largest, evenly by their logarithms.  Few elements may all be rounded by 2^-8 of themselves; 2^-9 of the
    norm for the arithmetic, whose worst in an emulation on the host was 1.6e-3."""
    rng = np.random.default_rng(rows)
    m = min(rows, cols)
    left, right = np.linalg.qr(rng.normal(size=(rows, m)))[0], np.linalg.qr(rng.normal(size=(cols, m)))[0]
    for low in (1e-2, 1e-6):
        g = torch.from_numpy(left * np.geomspace(1, low, m) @ right.T).float().cuda()
        want = oops.orthogonalize(_host(g))
        got = _host(tp.tppo_orthogonalize(g))
        assert np.linalg.norm(got - want) <= (2.0 ** -8 + 2.0 ** -9) * np.linalg.norm(want), low


def test_the_binding_refuses():
    """What does not fit is a ValueError before anything is launched; what the library refuses, a RuntimeError."""
    x, w, s = torch.zeros(6, 16, device="cuda"), torch.zeros(16, device="cuda"), torch.zeros(6, device="cuda")
    ids, i32 = torch.zeros(6, 2, dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    half = x.half()
    back = lambda *a, **k: tp.tppo_layer_norm_backward(*a, **k)                                        # noqa: E731
    calls = [
        lambda: tp.tppo_layer_norm(half, w), lambda: tp.tppo_layer_norm(x, w.half()), lambda: tp.tppo_layer_norm(x.t(), s),
        lambda: tp.tppo_layer_norm(x[0], w), lambda: tp.tppo_layer_norm(x, w[:15]), lambda: tp.tppo_layer_norm(x[:, ::2], w[:8]),
        lambda: tp.tppo_layer_norm(x[:1].expand(6, 16), w), lambda: tp.tppo_layer_norm(x, w, w.bfloat16()),
        lambda: tp.tppo_layer_norm(x, w.cpu()), lambda: tp.tppo_layer_norm(x, w, rows=i32.long()), lambda: tp.tppo_layer_norm(x, w, M=7),
        lambda: tp.tppo_layer_norm(x, w, M=-1), lambda: tp.tppo_layer_norm(x, w, rows=i32, M=7), lambda: tp.tppo_layer_norm(x, w, m_actual=i32),
        lambda: tp.tppo_layer_norm(x, w, out=x), lambda: tp.tppo_layer_norm(x, w, out=(x[:5], None, None)),
        lambda: tp.tppo_layer_norm(x, w, out=(half, None, None)), lambda: tp.tppo_layer_norm(x, w, out=(x, s[:5], None)),
        lambda: tp.tppo_layer_norm(x, w, status=s),
        lambda: back(x[:5], x, w, s, s), lambda: back(x, x, w, s[:5], s), lambda: back(x, x, w, None, s), lambda: back(half, x, w, s, s),
        lambda: back(x, x, w, s, s, out_index=i32), lambda: back(x, x, w, s, s, out=x[:5]), lambda: back(x, x, w, s, s, out=x, out_index=i32[:5]),
        lambda: back(x, x, w, s, s, grad_dtype=torch.float16), lambda: back(x, x, w, s, s, accumulate_w=True),
        lambda: back(x, x, w, s, s, grad_w=(w, w[:15])), lambda: back(x, x, w, s, s, workspace=x.t()),
        lambda: tp.tppo_balance_loss(half, ids), lambda: tp.tppo_balance_loss(x, ids.long()), lambda: tp.tppo_balance_loss(x, ids[:5]),
        lambda: tp.tppo_balance_loss(x, ids[:, 0]), lambda: tp.tppo_balance_loss(x, ids, out=(s[:1], None)),
        lambda: tp.tppo_balance_loss(x, ids, out=(None, i32, None)), lambda: tp.tppo_balance_loss_backward(x, ids, counts_in=w),
        lambda: tp.tppo_balance_loss_backward(x, ids, out_index=i32), lambda: tp.tppo_balance_loss_backward(x, ids, grad=x.bfloat16()),
        lambda: tp.tppo_balance_loss_backward(x, ids, grad=x[:5]),
        lambda: tp.tppo_orthogonalize(half), lambda: tp.tppo_orthogonalize(x.t()), lambda: tp.tppo_orthogonalize(w),
        lambda: tp.tppo_orthogonalize(x, out=x), lambda: tp.tppo_orthogonalize(x, out=x[:5].bfloat16()),
        lambda: tp.tppo_orthogonalize(x, coefficients=(1.0, 2.0)), lambda: tp.tppo_orthogonalize(x, out=x.bfloat16()[:1].expand(6, 16))]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i}")
    for i, call in enumerate([
            lambda: tp.tppo_layer_norm(x, w, eps=-1.0), lambda: back(x.bfloat16(), x, w, s, s), lambda: back(x, x, w, s, s, workspace=s),
            lambda: tp.tppo_balance_loss(x, ids, coefficient=float("nan")), lambda: tp.tppo_balance_loss(x, ids, workspace=s),
            lambda: tp.tppo_balance_loss_backward(x, ids, token_denominator=-1), lambda: tp.tppo_orthogonalize(x, steps=65),
            lambda: tp.tppo_orthogonalize(x, workspace=s),
            lambda: tp.tppo_orthogonalize(torch.zeros(2, 6, 16, device="cuda"), out=torch.zeros(1, 6, 16, dtype=BF, device="cuda").expand(2, 6, 16))]):
        with pytest.raises(RuntimeError):
            call()
            pytest.fail(f"call {i}")


def test_nothing_to_do():
    x, w = torch.zeros(0, 16, device="cuda"), torch.ones(16, device="cuda")
    ids = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    y, mean, rstd = tp.tppo_layer_norm(x, w)
    assert y.shape == (0, 16) and not bool(tp.tppo_layer_norm_backward(y, x, w, mean, rstd)[1].any())
    grad, loss, counts, mean_prob = tp.tppo_balance_loss_backward(x, ids)
    assert grad.shape == (0, 16) and float(loss) == 0 and not bool(counts.any()) and not bool(mean_prob.any())
    assert tp.tppo_orthogonalize(torch.zeros(0, 6, 16, device="cuda")).shape == (0, 6, 16)
    for shape in ((0, 16), (16, 0), (2, 0, 16)):
        with pytest.raises(RuntimeError):
            tp.tppo_orthogonalize(torch.zeros(shape, device="cuda"))


def test_one_expert_and_one_element():
    """The smallest of everything: E = 1 has a derivative of zero and a loss that is the coefficient."""
    z, ids = torch.randn(300, 1, device="cuda"), torch.zeros(300, 1, dtype=torch.int32, device="cuda")
    grad, loss, counts, mean_prob = tp.tppo_balance_loss_backward(z, ids, coefficient=0.5)
    assert not bool(grad.any()) and float(loss) == 0.5 and counts.tolist() == [300] and mean_prob.tolist() == [1.0]
    y, mean, rstd = tp.tppo_layer_norm(z, torch.ones(1, device="cuda"), torch.full((1,), 2.0, device="cuda"))
    assert bool((y == 2).all()) and torch.equal(mean, z[:, 0])
    for v in (3.0, -1e-3):
        out = tp.tppo_orthogonalize(torch.full((1, 1), v, device="cuda"))
        want = oops.orthogonalize(np.full((1, 1), np.float32(v)))
        assert abs(float(out) - want) <= 2.0 ** -8 * abs(want)


@pytest.mark.parametrize("dtype", [F, BF])
def test_masks_of_the_lowest_value(dtype):
    """Logits masked by their type's lowest value instead of -inf: alone in a row they are alike, beside others nothing."""
    lowest = torch.finfo(dtype).min
    z = torch.randn(6, 24, device="cuda").to(dtype)
    z[0], z[1, 5:], z[2, ::2] = lowest, lowest, lowest
    z[3, 0], z[3, 1:] = torch.finfo(dtype).max, lowest
    ids = torch.tensor([[1, 3, -1]] * 6, dtype=torch.int32, device="cuda")
    grad, loss, counts, mean_prob = tp.tppo_balance_loss_backward(z, ids)
    Z, I = _host(z), ids.cpu().numpy()
    oloss, ocounts, omean = oops.balance_loss(Z, I, 1.0)
    og, p, f = oops.balance_loss_backward(Z, I, 1.0), oops.softmax_rows(Z), ocounts / 18
    # exponents of a few units, rounded twice; sums of 24 and 6 terms
    assert counts.tolist() == ocounts.tolist() and abs(float(loss) - oloss) <= 128 * U * oloss
    _close(_host(mean_prob), omean, 128 * U * omean, U, "mean_prob")
    away = np.abs(f - f.mean())
    half = 2.0 ** -8 if dtype == BF else U
    _close(_host(grad), og, 256 * U * 4 * p * (away + (p * away).sum(1, keepdims=True) + f.mean()), half, "grad")
    assert not bool(grad[2, ::2].any()) and not bool(grad[3, 1:].any())
