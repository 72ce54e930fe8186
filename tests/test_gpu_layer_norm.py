"""The layer norm of listed rows and its derivatives against the oracle in 64 bits: row lengths on either side of every change of
the work division, rows that no vector divides, strides, lists, bad rows, graphs and streams."""
import numpy as np
import pytest
import torch

from oracle import operators as oops
from paper_2506_15050_amd import binding as tp

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                                  # half a step of fp32, relative
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
BF, F = torch.bfloat16, torch.float32


def _host(t):
    return t.detach().double().cpu().numpy()


def _rows(rng, M, n_rows):
    return rng.integers(0, n_rows, size=M).astype(np.int32)


def _terms(H):
    """Roundings on the way of one term into a sum over a row: pieces of a thread (128 elements at most), lanes, wavefronts."""
    return min(H, 128) + 12


def _check_forward(y, mean, rstd, x, w, b, eps, rows, dtype):
    oy, om, os_ = oops.layer_norm(x, w, b, eps, rows)
    xr = x if rows is None else x[rows]
    n, size = _terms(x.shape[1]), np.abs(xr).mean(1)
    # the mean: n roundings of sums of |x|; the variance: n of its own, twice the mean's error against the deviation
    e_mean = n * U * size + U * np.abs(om)
    dev = 1 / os_
    e_rstd = os_ * (U * (n + 8) + 2 * e_mean * np.abs(xr - om[:, None]).mean(1) * os_ ** 2 + (e_mean * os_) ** 2)
    assert np.all(np.abs(mean - om) <= e_mean) and np.all(np.abs(rstd - os_) <= e_rstd)
    xh = np.abs(xr - om[:, None]) * os_[:, None]
    aw, ab = np.abs(w), 0 if b is None else np.abs(b)
    bound = (4 * U + (e_rstd * dev)[:, None]) * xh * aw + ((e_mean + U * np.abs(om)) * os_)[:, None] * aw + 2 * U * ab
    bound = bound * 1.01 + HALF[dtype] * (np.abs(oy) + bound) + 1e-37
    worst = (np.abs(y - oy) / bound).max()
    assert worst <= 1, f"{worst} times the bound"


def _make(rng, n_rows, H, dtype, w_dtype, pad=0, shift=0, bias=True):
    """x [n_rows, H] with a row stride of H + pad elements, from `shift` elements after an aligned address."""
    x = rng.normal(size=(n_rows, H)) * 2 + rng.normal(size=(n_rows, 1))
    x[:, :: max(1, H // 3)] *= 8
    flat = torch.full((n_rows * (H + pad) + shift,), float("nan"), dtype=dtype, device="cuda")
    t = flat[shift:].view(n_rows, H + pad)[:, :H]
    t.copy_(torch.from_numpy(x))
    w = torch.from_numpy(1 + 0.2 * rng.normal(size=H)).to("cuda", w_dtype)
    b = torch.from_numpy(0.1 * rng.normal(size=H)).to("cuda", w_dtype) if bias else None
    return t, w, b


SIZES = [1, 2, 3, 7, 8, 9, 64, 255, 256, 257, 511, 512, 513, 1000, 1024, 1025, 2047, 2048, 2056, 4096, 4100, 5120, 6144, 6152, 8192, 8200,
         12289, 16384]


@pytest.mark.parametrize("H", SIZES)
@pytest.mark.parametrize("dtype,w_dtype", [(BF, BF), (BF, F), (F, F)])
def test_forward(H, dtype, w_dtype):
    rng = np.random.default_rng(H)
    for M, pad, shift, bias in ((1, 0, 0, True), (5, 0, 0, False), (67, 3, 1, True)):
        x, w, b = _make(rng, 70, H, dtype, w_dtype, pad, shift, bias)
        rows = _rows(rng, M, 70)
        st = tp.new_status("cuda")
        y, mean, rstd = tp.tppo_layer_norm(x, w, b, rows=torch.from_numpy(rows).cuda(), status=st)
        assert int(st.item()) == 0 and y.dtype == dtype and y.shape == (M, H)
        _check_forward(_host(y), _host(mean), _host(rstd), _host(x), _host(w), None if b is None else _host(b), np.float64(np.float32(1e-5)),
                       rows, dtype)


TYPES = [(F, F, F), (BF, F, F), (BF, F, BF), (BF, BF, F), (BF, BF, BF)]


def _check_backward(got, gy, x, w, mean, rstd, rows, M, gx_dtype, groups=512):
    gx, gw, gb = got
    ogx, ogw, ogb = oops.layer_norm_backward(gy[:M], x, w, mean[:M], rstd[:M], rows)
    H, n = x.shape[1], _terms(x.shape[1])
    xr = x if rows is None else x[rows]
    xr = xr[:M]
    # x - mean is rounded against its own size (and exact where they are close): 2 roundings of xh
    xh, g, s = np.abs(xr - mean[:M, None]) * rstd[:M, None], np.abs(gy[:M] * w), rstd[:M, None]
    e_xh = 2 * U * xh
    c1, c2 = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    if gx is not None:
        bound = s * (6 * U * g + (n + 4) * U * c1 + ((n + 8) * U * xh + e_xh) * c2) * 1.01
        bound = bound + HALF[gx_dtype] * (np.abs(ogx) + bound) + 1e-37
        worst = (np.abs(gx - ogx) / bound).max()
        assert worst <= 1, f"grad_x: {worst} times the bound"
    # a column's sum: the rows of a thread, then the partial sums of up to `groups` workgroups
    turns = -(-M // groups) + 8 + 64
    if gw is not None:
        assert np.all(np.abs(gw - ogw) <= (turns + 4) * U * (np.abs(gy[:M]) * xh).sum(0) + 1e-37)
    if gb is not None:
        assert np.all(np.abs(gb - ogb) <= turns * U * np.abs(gy[:M]).sum(0) + 1e-37)


@pytest.mark.parametrize("H", SIZES)
@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(str(x).split(".")[1] for x in t))
def test_backward(H, types):
    dtype, gy_dtype, gx_dtype = types
    rng = np.random.default_rng(H + 1)
    for M, pad, shift in ((1, 0, 0), (37, 0, 0), (611, 5, 3)):
        n_rows = 70
        x, w, _ = _make(rng, n_rows, H, dtype, dtype, pad, shift)
        rows = _rows(rng, M, n_rows)
        gy = torch.from_numpy(rng.normal(size=(M, H)) / M).to("cuda", gy_dtype)
        _, mean, rstd = oops.layer_norm(_host(x), _host(w), None, 1e-5, rows)
        mean, rstd = torch.from_numpy(mean).float().cuda(), torch.from_numpy(rstd).float().cuda()
        st = tp.new_status("cuda")
        got = tp.tppo_layer_norm_backward(gy, x, w, mean, rstd, rows=torch.from_numpy(rows).cuda(), grad_dtype=gx_dtype, status=st)
        assert int(st.item()) == 0 and got[0].dtype == gx_dtype
        _check_backward([_host(t) for t in got], _host(gy), _host(x), _host(w), _host(mean), _host(rstd), rows, M, gx_dtype)
        again = tp.tppo_layer_norm_backward(gy, x, w, mean, rstd, rows=torch.from_numpy(rows).cuda(), grad_dtype=gx_dtype)
        assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_gradient_by_differences():
    rng = np.random.default_rng(5)
    M, H = 6, 40
    x, w, b = _make(rng, M, H, F, F)
    gy = torch.from_numpy(rng.normal(size=(M, H))).float().cuda()
    _, mean, rstd = tp.tppo_layer_norm(x, w, b)
    gx, gw, gb = tp.tppo_layer_norm_backward(gy, x, w, mean, rstd)
    X, W, G = _host(x), _host(w), _host(gy)
    f = lambda X, W: float((oops.layer_norm(X, W, None, 1e-5)[0] * G).sum())                          # noqa: E731
    for m, h in ((0, 0), (3, 17), (5, 39)):
        d = np.zeros_like(X)
        d[m, h] = 1e-5
        assert abs((f(X + d, W) - f(X - d, W)) / 2e-5 - float(gx[m, h])) < 1e-4
    for h in (0, 21, 39):
        d = np.zeros_like(W)
        d[h] = 1e-5
        assert abs((f(X, W + d) - f(X, W - d)) / 2e-5 - float(gw[h])) < 1e-4
    assert np.allclose(_host(gb), G.sum(0), atol=1e-5)


@pytest.mark.parametrize("H,dtype", [(64, F), (1001, BF), (5120, BF), (9000, F)])
def test_counts_bad_rows_and_what_is_left_alone(H, dtype):
    rng = np.random.default_rng(H)
    n_rows, M = 50, 45
    x, w, b = _make(rng, n_rows, H, dtype, dtype)
    rows = _rows(rng, M, n_rows)
    rows[[3, 20, 44]] = [-1, n_rows, 2 ** 31 - 1]
    listed = torch.from_numpy(rows).cuda()
    good = (rows >= 0) & (rows < n_rows)
    for m_eff in (0, 1, 30, M, 1000, -5):
        used = max(0, min(M, m_eff))
        count = torch.tensor([m_eff], dtype=torch.int64, device="cuda")
        out = (torch.full((M, H), 7.0, dtype=dtype, device="cuda"), torch.full((M,), 7.0, device="cuda"), torch.full((M,), 7.0, device="cuda"))
        st = tp.new_status("cuda")
        y, mean, rstd = tp.tppo_layer_norm(x, w, b, rows=listed, m_actual=count, out=out, status=st)
        assert (int(st.item()) == tp.STATUS_BAD_ROW) == bool((~good[:used]).any())
        for t in (y, mean[:, None], rstd[:, None]):
            h = _host(t)
            assert np.all(h[used:] == 7) and np.all(np.isnan(h[:used][~good[:used]])) and not np.isnan(h[:used][good[:used]]).any()
        gy = torch.from_numpy(rng.normal(size=(M, H))).to("cuda", dtype)
        m, r = torch.zeros(M, device="cuda"), torch.ones(M, device="cuda")
        to = rng.permutation(M + 9)[:M].astype(np.int32)
        to[7] = M + 9
        gx = torch.full((M + 9, H), 7.0, dtype=dtype, device="cuda")
        gw = (torch.full((H,), 3.0, device="cuda"), torch.full((H,), 5.0, device="cuda"))
        st = tp.new_status("cuda")
        tp.tppo_layer_norm_backward(gy, x, w, m, r, rows=listed, m_actual=count, out=gx, out_index=torch.from_numpy(to).cuda(), grad_w=gw,
                                    accumulate_w=True, status=st)
        keep = good[:used]
        assert (int(st.item()) == tp.STATUS_BAD_ROW) == bool((~keep).any() or used > 7)
        h = _host(gx)
        touched = np.zeros(M + 9, bool)
        touched[[t for i, t in enumerate(to[:used]) if i != 7]] = True
        assert np.all(h[~touched] == 7)
        bad_to = [to[i] for i in range(used) if not keep[i] and i != 7]
        assert np.all(np.isnan(h[bad_to])) and np.isnan(h).sum() == len(bad_to) * H
        idx = np.flatnonzero(keep)
        _, ow, ob = oops.layer_norm_backward(_host(gy)[idx], _host(x), _host(w), np.zeros(len(idx)), np.ones(len(idx)), rows[idx])
        size = np.abs(_host(gy)[idx]).sum(0)
        most = np.abs(_host(x)).max()
        assert np.all(np.abs(_host(gw[0]) - 3 - ow) <= 80 * U * (size * most + 3)) and np.all(np.abs(_host(gw[1]) - 5 - ob) <= 80 * U * (size + 5))


def test_no_rows_and_wanted_parts():
    x, w = torch.randn(4, 96, device="cuda"), torch.ones(96, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    y, mean, rstd = tp.tppo_layer_norm(x, w, rows=none)
    assert y.shape == (0, 96) and mean.numel() == 0
    gx, gw, gb = tp.tppo_layer_norm_backward(x[:0], x, w, mean, rstd, rows=none)
    assert gx.shape == (0, 96) and not bool(gw.any()) and not bool(gb.any())
    kept = torch.ones(96, device="cuda")
    tp.tppo_layer_norm_backward(x[:0], x, w, mean, rstd, rows=none, grad_w=(kept, None), accumulate_w=True)
    assert bool((kept == 1).all())
    y, mean, rstd = tp.tppo_layer_norm(x, w)
    full = tp.tppo_layer_norm_backward(x, x, w, mean, rstd)
    only_x = tp.tppo_layer_norm_backward(x, x, w, mean, rstd, want_w=False)
    only_w = tp.tppo_layer_norm_backward(x, x, w, mean, rstd, want_x=False, want_bias=False)
    assert torch.equal(only_x[0], full[0]) and only_x[1] is None and only_x[2] is None
    assert only_w[0] is None and torch.equal(only_w[1], full[1]) and only_w[2] is None
    bare = tp.tppo_layer_norm(x, w, want_stats=False)
    assert bare[1] is None and torch.equal(bare[0], y)


def test_constant_and_large_rows():
    x = torch.stack([torch.full((512,), 3.0), torch.full((512,), 1e18), torch.zeros(512), torch.linspace(1e4, 1.0001e4, 512)]).cuda()
    w = torch.ones(512, device="cuda")
    y, mean, rstd = tp.tppo_layer_norm(x, w)
    # the mean of equal numbers is off by its sum's roundings; an exact one would give zeros
    assert bool((y[0].abs() <= 20 * U * 3 / 1e-5 ** 0.5).all()) and bool((y[2] == 0).all()) and bool(torch.isfinite(y).all())
    x[1, 3] = float("nan")
    x[2, 5] = float("inf")
    y, mean, rstd = tp.tppo_layer_norm(x, w)
    assert bool(torch.isnan(y[1]).all()) and bool(torch.isnan(y[2]).all()) and bool(torch.isfinite(y[0]).all() and torch.isfinite(y[3]).all())


def test_captured_and_on_another_stream():
    rng = np.random.default_rng(3)
    x, w, b = _make(rng, 90, 1024, BF, BF)
    rows = torch.arange(7, 80, device="cuda", dtype=torch.int32)
    gy = torch.randn(73, 1024, device="cuda")
    ws = tp._workspace(tp.load().tppo_layer_norm_backward_workspace_bytes(73, 1024), "cuda")
    kept = (torch.empty(73, 1024, dtype=BF, device="cuda"), torch.empty(73, device="cuda"), torch.empty(73, device="cuda"))
    gx, gw = torch.empty(73, 1024, dtype=BF, device="cuda"), (torch.empty(1024, device="cuda"), torch.empty(1024, device="cuda"))

    def step():
        tp.tppo_layer_norm(x, w, b, rows=rows, out=kept)
        tp.tppo_layer_norm_backward(gy, x, w, kept[1], kept[2], rows=rows, out=gx, grad_w=gw, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        x.copy_(torch.randn(90, 1024, device="cuda"))
        gy.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*kept, gx, *gw)]
        for t in (*kept, gx, *gw):
            t.fill_(9)
        step()
        assert all(torch.equal(a, t) for a, t in zip(got, (*kept, gx, *gw))), k
