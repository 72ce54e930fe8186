"""The balance loss's derivative where the counts are many, or nearly alike: counts beyond 32 bits."""
import numpy as np
import pytest
import torch

from oracle import operators as oops
from paper_2506_15050_amd import binding as tp

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("E", [8, 200, 600])
def test_more_choices_of_an_expert_than_32_bits_count(E):
    """One row, listed two million times, with 1023 of its 1024 choices the same: 2.15e9 of one expert, one of another a token."""
    M, k = (1 << 21) + (1 << 12), 1024
    assert M * (k - 1) > 1 << 31
    z = torch.randn(4, E, device="cuda")
    ids = torch.zeros(4, k, dtype=torch.int32, device="cuda")
    ids[3, 77] = 5
    rows = torch.full((M,), 3, dtype=torch.int32, device="cuda")
    grad, loss, counts, _ = tp.tppo_balance_loss_backward(z, ids, rows=rows)
    want = np.zeros(E)
    want[[0, 5]] = M * (k - 1), M
    assert counts.tolist() == want.tolist()
    p, f = oops.softmax_rows(z.double().cpu().numpy()[3:])[0], want / (k * M)
    spread = (p * np.abs(f - f.mean())).sum()
    g = E / M * p * (f - (p * f).sum())
    # the probability: an argument of at most 12 rounded twice, exp2, a sum of 600 over lanes: 64 steps; the sum over the row as many again
    bound = E / M * p * 64 * U * (np.abs(f - f.mean()) + 3 * spread) + U * np.abs(g)
    for got in (grad.amin(0), grad.amax(0)):                        # every token's
        worst = float((np.abs(got.double().cpu().numpy() - g) / bound).max())
        assert worst <= 1, f"{worst} times the bound"
    # a thread adds up to 1028 rows, a workgroup's wavefronts and all workgroups follow
    assert abs(float(loss) - E * (p * f).sum()) <= (64 + 1028 + 16) * U * float(loss)
