"""The oracle of the layer norm, the balance loss and the orthogonalisation against what does not share its formulas:
autograd of library routines, differences, and singular values."""
import numpy as np
import pytest
import torch

from oracle import operators as oops


@pytest.mark.parametrize("M,H", [(1, 1), (3, 7), (5, 64)])
def test_layer_norm_is_the_library_routine_and_its_autograd(M, H):
    rng = np.random.default_rng(M + H)
    x, w, b, gy = rng.normal(size=(M + 2, H)), rng.normal(size=H), rng.normal(size=H), rng.normal(size=(M, H))
    rows = rng.permutation(M + 2)[:M]
    t = torch.from_numpy(x[rows]).requires_grad_()
    tw, tb = torch.from_numpy(w).requires_grad_(), torch.from_numpy(b).requires_grad_()
    y = torch.nn.functional.layer_norm(t, (H,), tw, tb, 1e-5)
    y.backward(torch.from_numpy(gy))
    oy, mean, rstd = oops.layer_norm(x, w, b, 1e-5, rows)
    gx, gw, gb = oops.layer_norm_backward(gy, x, w, mean, rstd, rows)
    for got, want in ((oy, y.detach()), (gx, t.grad), (gw, tw.grad), (gb, tb.grad)):
        assert np.allclose(got, want.numpy(), rtol=1e-9, atol=1e-11)


def test_balance_loss_by_differences_and_in_its_limits():
    rng = np.random.default_rng(0)
    M, E, k = 9, 5, 2
    z, ids = rng.normal(size=(M, E)), rng.integers(-1, E, size=(M, k))
    z[2, 1] = -np.inf
    z[4] = -np.inf
    g = oops.balance_loss_backward(z, ids, 0.3, 1.7)
    for m in range(M):
        for e in range(E):
            if np.isinf(z[m, e]):
                assert g[m, e] == 0.0
                continue
            h = 1e-6
            up, down = z.copy(), z.copy()
            up[m, e] += h
            down[m, e] -= h
            diff = 1.7 * (oops.balance_loss(up, ids, 0.3)[0] - oops.balance_loss(down, ids, 0.3)[0]) / (2 * h)
            assert abs(diff - g[m, e]) <= 1e-9
    # an even use of all experts gives the coefficient; all tokens on one expert with certainty E times it
    even = np.tile(np.arange(E), (3, 1)).repeat(2, 0)
    assert abs(oops.balance_loss(np.zeros((6, E)), even, 0.3)[0] - 0.3) < 1e-12
    one = np.full((6, E), -1e9)
    one[:, 3] = 0.0
    assert abs(oops.balance_loss(one, np.full((6, 1), 3), 0.3)[0] - 0.3 * E) < 1e-12
    # autograd of the library's softmax
    t = torch.from_numpy(np.where(np.isinf(z), -50.0, z)).requires_grad_()
    p = torch.softmax(t, 1)
    counts = torch.bincount(torch.from_numpy(ids[ids >= 0]), minlength=E)
    (0.3 * E * (counts / (k * M) * p.sum(0) / M).sum()).backward()
    assert np.allclose(oops.balance_loss_backward(t.detach().numpy(), ids, 0.3), t.grad.numpy(), atol=1e-12)
    # parts of a batch add up
    whole, counts, _ = oops.balance_loss(z, ids, 0.3)
    halves = [oops.balance_loss(z[s], ids[s], 0.3, counts_in=counts, tokens=M)[0] for s in (slice(0, 4), slice(4, None))]
    assert abs(sum(halves) - whole) < 1e-12
    parts = np.concatenate([oops.balance_loss_backward(z[s], ids[s], 0.3, counts_in=counts, tokens=M) for s in (slice(0, 4), slice(4, None))])
    assert np.allclose(parts, oops.balance_loss_backward(z, ids, 0.3), atol=1e-15)
    assert oops.balance_loss(z[:0], ids[:0], 0.3)[0] == 0.0


@pytest.mark.parametrize("rows,cols", [(1, 9), (9, 1), (6, 6), (5, 12), (12, 5)])
def test_orthogonalize_maps_each_singular_value_by_the_polynomial(rows, cols):
    rng = np.random.default_rng(rows * cols)
    g = rng.normal(size=(rows, cols))
    u, s, vt = np.linalg.svd(g, full_matrices=False)
    s = s / (np.linalg.norm(g) + 1e-7)
    a, b, c = 3.4445, -4.7750, 2.0315
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(oops.orthogonalize(g, scale=0.5), 0.5 * (u * s) @ vt, atol=1e-10)
    assert s.min() > 0.3 and s.max() < 1.3
    assert not np.any(oops.orthogonalize(np.zeros((rows, cols))))
