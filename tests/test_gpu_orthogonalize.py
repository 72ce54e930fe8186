"""The orthogonalisation against the oracle in 64 bits: sizes on either side of every tile and kernel, wide and tall, stacks, strides,
low ranks, what is no number, graphs."""
import numpy as np
import pytest
import torch

from oracle import operators as oops
from paper_2506_15050_amd import binding as tp

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
# The result is rounded to bf16: 2^-8 of a value at most, 1.7e-3 of the norm as a rule.  The arithmetic (operands of 11 bits, X in 22,
# diagonals in 24) was off by 1.8e-3 of the norm at most in an emulation on the host (ranks from one to full, 256 .. 3000); twice that and
# the rounding together are 2^-8 of the norm.
NORM = 2.0 ** -8
# an element: its rounding, and eight standard deviations of an error of 3.6e-3 of the elements' root mean square
ELEMENT = 8 * 3.6e-3


def _host(t):
    return t.detach().double().cpu().numpy()


def _check(got, g, **kw):
    want = oops.orthogonalize(_host(g), **kw)
    got = _host(got)
    rms = np.sqrt((want ** 2).mean())
    assert np.linalg.norm(got - want) <= NORM * np.linalg.norm(want), (np.linalg.norm(got - want) / np.linalg.norm(want), g.shape)
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + ELEMENT * rms)


def _matrix(rng, rows, cols, kind):
    small = min(rows, cols)
    if kind == "full":
        return rng.normal(size=(rows, cols))
    if kind == "shared":
        r = max(1, small // 4)
        return rng.normal(size=(rows, r)) @ rng.normal(size=(r, cols)) / np.sqrt(r) * 1e-3 + rng.normal(size=(rows, cols)) * 3e-4
    r = {"rank1": 1, "rank4": 4}[kind]
    return rng.normal(size=(rows, r)) @ rng.normal(size=(r, cols))


SHAPES = [(1, 1), (1, 7), (5, 1), (2, 2), (3, 64), (17, 16), (63, 65), (64, 64), (64, 1024), (65, 129), (127, 128), (128, 128), (129, 127),
          (130, 700), (256, 256), (257, 300), (1000, 333), (384, 1025), (520, 2000)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("kind", ["full", "shared", "rank4", "rank1"])
def test_shapes(shape, kind):
    rng = np.random.default_rng(shape[0] * 7 + shape[1])
    g = torch.from_numpy(_matrix(rng, *shape, kind)).float().cuda()
    out = tp.tppo_orthogonalize(g)
    assert out.dtype == BF and out.shape == g.shape
    _check(out, g)
    assert torch.equal(out, tp.tppo_orthogonalize(g))


@pytest.mark.parametrize("rows,cols", [(33, 70), (70, 33), (200, 200), (600, 150)])
@pytest.mark.parametrize("count", [1, 5])
def test_stacks_strides_and_types(rows, cols, count):
    rng = np.random.default_rng(rows + count)
    for dtype in (F, BF):
        flat = torch.full((count, rows + 3, cols + 5), float("nan"), dtype=dtype, device="cuda")
        g = flat[:, 1:rows + 1, 3:cols + 3]
        g.copy_(torch.from_numpy(np.stack([_matrix(rng, rows, cols, "shared") * 10.0 ** (4 * i) for i in range(count)])))
        room = torch.full((count, rows + 2, cols + 1), 7.0, dtype=BF, device="cuda")
        out = tp.tppo_orthogonalize(g, out=room[:, :rows, 1:], scale=0.25)
        for i in range(count):
            _check(out[i], g[i], scale=0.25)
        assert bool((room[:, rows:] == 7).all()) and bool((room[:, :, 0] == 7).all())
        assert torch.equal(tp.tppo_orthogonalize(g, scale=0.25), out)
        assert torch.equal(tp.tppo_orthogonalize(g[0], scale=0.25), out[0])
        same = g[:1].expand(count, rows, cols)
        assert torch.equal(tp.tppo_orthogonalize(same, scale=0.25)[-1], out[0])


def test_steps_and_coefficients():
    rng = np.random.default_rng(8)
    g = torch.from_numpy(_matrix(rng, 96, 160, "full")).float().cuda()
    for steps in (0, 1, 2, 7):
        _check(tp.tppo_orthogonalize(g, steps=steps), g, steps=steps)
        _check(tp.tppo_orthogonalize(g.t().contiguous(), steps=steps), g.t(), steps=steps)
    cubic = (1.5, -0.5, 0.0)
    _check(tp.tppo_orthogonalize(g, steps=12, coefficients=cubic), g, steps=12, coefficients=cubic)


@pytest.mark.parametrize("shape", [(40, 70), (300, 200)])
def test_sizes_of_values(shape):
    rng = np.random.default_rng(9)
    base = rng.normal(size=shape)
    for scale in (1e-30, 1e-8, 1e18, 3e37):
        g = torch.from_numpy(base * scale / np.abs(base).max()).float().cuda()
        _check(tp.tppo_orthogonalize(g), g)
    assert not bool(tp.tppo_orthogonalize(torch.zeros(shape, device="cuda")).any())
    for bad in (float("nan"), float("inf"), float("-inf")):
        g = torch.from_numpy(base).float().cuda()
        g[shape[0] - 1, 3] = bad
        stack = torch.stack([torch.from_numpy(base).float().cuda(), g])
        out = tp.tppo_orthogonalize(stack)
        assert bool(torch.isnan(out[1]).all())
        _check(out[0], stack[0])


@pytest.mark.parametrize("rows,cols,dtype", [
    (1024, 4096, F), (2056, 1100, BF),          # pairs of 64 x 64 tiles, of more of them than CUs
    (2304, 2304, F), (2049, 2500, F),           # products of X in tiles of 128 x 128, sizes that end inside one
    (5120, 2300, BF), (2304, 5120, F),          # B X in tiles of 192 rows, tall and wide
    (4096, 4096, F), (4000, 4090, BF),          # X X^T in tiles of 160 rows, B X of 256
    (4608, 4608, F), (4610, 4520, F)])          # X X^T in tiles of 192 rows
def test_large(rows, cols, dtype):
    """Against the iteration in 64 bits on the device (the host's takes minutes)."""
    g = torch.randn(rows, cols, device="cuda").to(dtype)
    g[:, : cols // 3] += (torch.randn(rows, 8, device="cuda") @ torch.randn(8, cols // 3, device="cuda")).to(dtype)
    out = tp.tppo_orthogonalize(g).double()
    x = g.double()
    if rows > cols:
        x = x.t().contiguous()
    x = x / (x.norm() + 1e-7)
    for _ in range(5):
        s = x @ x.t()
        x = 3.4445 * x + (-4.7750 * s + 2.0315 * (s @ s)) @ x
    x = x.t() if rows > cols else x
    rms = x.norm() / x.numel() ** 0.5
    assert float((out - x).norm() / x.norm()) <= NORM
    assert bool(((out - x).abs() <= 2.0 ** -8 * x.abs() + ELEMENT * rms).all())


@pytest.mark.parametrize("rows,cols", [(1100, 1030), (700, 1500)])
def test_stacks_of_middling_matrices(rows, cols):
    """A single one goes by pairs, eight by products of X: both against 64 bits."""
    g = torch.randn(8, rows, cols, device="cuda")
    for out, src in ((tp.tppo_orthogonalize(g)[5], g[5]), (tp.tppo_orthogonalize(g[5]), g[5])):
        x = src.double()
        x = x.t().contiguous() if rows > cols else x
        x = x / (x.norm() + 1e-7)
        for _ in range(5):
            s = x @ x.t()
            x = 3.4445 * x + (-4.7750 * s + 2.0315 * (s @ s)) @ x
        x = x.t() if rows > cols else x
        assert float((out.double() - x).norm() / x.norm()) <= NORM


def test_captured():
    g = torch.randn(2, 150, 260, device="cuda")
    out = torch.empty(2, 150, 260, dtype=BF, device="cuda")
    ws = tp._workspace(tp.load().tppo_orthogonalize_workspace_bytes(2, 150, 260), "cuda")
    step = lambda: tp.tppo_orthogonalize(g, workspace=ws, out=out)                                   # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        g.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(9)
        ws.random_(0, 255)
        step()
        assert torch.equal(got, out), k
