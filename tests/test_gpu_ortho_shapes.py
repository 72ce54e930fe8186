"""The orthogonalisation where its products take the other tiles, against the iteration in 64 bits: symmetric products in the largest
tiles, low ranks and wide spectra by products of X, three passes over several tiles.  (Which way a size goes: test_ortho_rules.py.)"""
import numpy as np
import pytest
import torch

from oracle import operators as oops
from paper_2506_15050_amd import binding as tp

pytestmark = pytest.mark.gpu

# as in test_gpu_orthogonalize.py: the norm of the error, and an element's
NORM, ELEMENT = 2.0 ** -8, 8 * 3.6e-3
A = 3.4445


def _iteration(g):
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    x = x / (x.norm() + 1e-7)
    for _ in range(5):
        s = x @ x.t().contiguous()
        x = A * x + (-4.7750 * s + 2.0315 * (s @ s)) @ x
    return x.t() if tall else x


def _spectrum(rng, rows, cols, kind):
    """Rank one or four, or singular values in equal ratios from 1 to 10^-3 or 10^-6."""
    if kind.startswith("rank"):
        r = int(kind[4:])
        return rng.normal(size=(rows, r)) @ rng.normal(size=(r, cols))
    if kind == "full":
        return rng.normal(size=(rows, cols))
    r = min(rows, cols)
    left, right = (np.linalg.qr(rng.normal(size=(n, r)))[0] for n in (rows, cols))
    return left * np.logspace(0, -int(kind[3:]), r) @ right.T


def _check(out, g, elements=True):
    want, out = _iteration(g), out.double()
    worst = float((out - want).norm() / want.norm())
    assert worst <= NORM, worst
    if elements:
        rms = want.norm() / want.numel() ** 0.5
        assert bool(((out - want).abs() <= 2.0 ** -8 * want.abs() + ELEMENT * rms).all())


@pytest.mark.parametrize("rows,cols,dtype", [(5120, 5120, torch.float32), (5121, 5300, torch.bfloat16), (5300, 4900, torch.float32)])
def test_symmetric_products_in_tiles_of_256(rows, cols, dtype):
    g = torch.randn(rows, cols, device="cuda")
    g[:, : cols // 3] += torch.randn(rows, 8, device="cuda") @ torch.randn(8, cols // 3, device="cuda")
    g = g.to(dtype)
    _check(tp.tppo_orthogonalize(g), g)


@pytest.mark.parametrize("count,rows,cols", [(1, 2304, 2304), (8, 1100, 1030), (40, 520, 520), (16, 530, 700)])
@pytest.mark.parametrize("kind", ["rank1", "rank4", "geo3", "geo6"])
def test_spectra_by_products_of_X(count, rows, cols, kind):
    one = torch.from_numpy(_spectrum(np.random.default_rng(rows + len(kind)), rows, cols, kind)).float().cuda()
    g = torch.randn(count, rows, cols, device="cuda")
    g[count // 2] = one
    _check(tp.tppo_orthogonalize(g)[count // 2], one, elements=False)


@pytest.mark.parametrize("rows,cols", [(300, 450), (700, 511), (129, 640)])
@pytest.mark.parametrize("steps", [7, 10])
def test_three_passes_over_several_tiles(rows, cols, steps):
    rng = np.random.default_rng(rows + steps)
    for kind, most in (("rank1", NORM + 5 * 2.0 ** -24 * A ** steps), ("geo6", NORM), ("full", NORM)):
        g = torch.from_numpy(_spectrum(rng, rows, cols, kind)).float().cuda()
        want = oops.orthogonalize(g.double().cpu().numpy(), steps=steps)
        worst = np.linalg.norm(tp.tppo_orthogonalize(g, steps=steps).double().cpu().numpy() - want) / np.linalg.norm(want)
        assert worst <= most, (kind, worst, most)
