"""Oracle of the operators around the heads and the losses: numpy fp64, from their definitions.

Test infrastructure only: the product path never imports this module.  The layer norm and its derivatives, the balance loss
of a mixture-of-experts router and its derivative, and the Newton-Schulz iteration; pinned by autograd, differences,
library routines and the singular values of the result (``tests/test_operator_oracle.py``).
"""
import numpy as np

from .fast import decode


def layer_norm(x, weight, bias, eps, rows=None):
    """(y, mean, rstd) of the rows x[rows]."""
    x = decode(x)
    x = x if rows is None else x[rows]
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None] * decode(weight)
    return (y if bias is None else y + decode(bias)), mean, rstd


def layer_norm_backward(grad_y, x, weight, mean, rstd, rows=None):
    """(grad_x, grad_weight, grad_bias) for the given statistics."""
    gy, x = decode(grad_y), decode(x)
    x = x if rows is None else x[rows]
    xh = (x - decode(mean)[:, None]) * decode(rstd)[:, None]
    g = gy * decode(weight)
    gx = decode(rstd)[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return gx, (gy * xh).sum(0), gy.sum(0)


def softmax_rows(z):
    """exp(z) / sum exp(z) by row; a row of -inf has no distribution and gives zeros."""
    z = decode(z)
    with np.errstate(invalid="ignore"):
        top = z.max(1, keepdims=True)
        e = np.exp(z - np.where(top == -np.inf, 0.0, top))
        total = e.sum(1, keepdims=True)
        return e / np.where(total == 0.0, 1.0, total)


def balance_loss(logits, experts, coefficient, rows=None, counts_in=None, tokens=None):
    """(loss, counts, mean_prob): loss = coefficient * E * sum_e counts_e / (k N) * mean_prob_e."""
    p = softmax_rows(logits if rows is None else np.asarray(logits)[rows])
    ids = np.asarray(experts if rows is None else np.asarray(experts)[rows])
    E, k = p.shape[1], ids.shape[1]
    N = p.shape[0] if tokens is None else tokens
    counts = np.bincount(ids[(ids >= 0) & (ids < E)], minlength=E)
    if N == 0:
        return 0.0, counts, np.zeros(E)
    mean_prob = p.sum(0) / N
    f = (counts if counts_in is None else np.asarray(counts_in)) / (k * N)
    return coefficient * E * float((f * mean_prob).sum()), counts, mean_prob


def balance_loss_backward(logits, experts, coefficient, scale=1.0, rows=None, counts_in=None, tokens=None):
    """d (scale * loss) / d logits, the counts being constants."""
    p = softmax_rows(logits if rows is None else np.asarray(logits)[rows])
    ids = np.asarray(experts if rows is None else np.asarray(experts)[rows])
    E, k = p.shape[1], ids.shape[1]
    N = p.shape[0] if tokens is None else tokens
    counts = np.bincount(ids[(ids >= 0) & (ids < E)], minlength=E) if counts_in is None else np.asarray(counts_in)
    f = counts / (k * N)
    return scale * coefficient * E / N * p * (f - (p * f).sum(1, keepdims=True))


def orthogonalize(g, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, scale=1.0):
    """The Newton-Schulz iteration on one matrix."""
    x = decode(g)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    x = x / (np.sqrt((x * x).sum()) + eps)
    a, b, c = coefficients
    for _ in range(steps):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return scale * (x.T if tall else x)
