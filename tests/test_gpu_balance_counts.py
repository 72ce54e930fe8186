"""The balance loss's derivative where the counts are many, or nearly alike: counts beyond 32 bits, counts one apart in thousands and in
hundreds of millions."""
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


def _nearly_even(E, even, M):
    """Router logits of M tokens, and counts of a batch in which every expert has `even` choices, give or take one."""
    rng = np.random.default_rng(E)
    z = torch.from_numpy(rng.normal(size=(M, E))).float().cuda()
    return z, torch.from_numpy(even + rng.integers(-1, 2, size=E)).cuda()


def _check_nearly_even(grad, z, counts, k, tokens):
    """The same derivative from any f that differs by the same amount everywhere: a row's p add up to one."""
    z, d = z.double().cpu().numpy(), counts.cpu().numpy()
    E = len(d)
    d = (d - int(np.median(d))) / (k * tokens)
    d = d - d.mean()
    p = oops.softmax_rows(z)
    g = E / tokens * p * (d - (p * d).sum(1, keepdims=True))
    spread = (p * np.abs(d)).sum(1, keepdims=True)
    # no term of the size of f itself: d is rounded once, a probability is off by 64 steps (arguments up to 12, rounded twice), the sum over
    # the row by as many, and the steps of the formula
    bound = E / tokens * p * ((64 + 8) * U * (np.abs(d) + spread) + (64 + 64) * U * spread) + U * np.abs(g) + 1e-37
    worst = float((np.abs(grad.double().cpu().numpy() - g) / bound).max())
    assert worst <= 1, f"{worst} times the bound"


@pytest.mark.parametrize("E,k", [(128, 8), (67, 3), (500, 7)])
def test_counts_one_apart(E, k):
    """An update's tokens, spread over the experts as evenly as they go: counts that are no powers of two, one apart."""
    M = 77536
    ids = torch.arange(M * k, dtype=torch.int32).remainder(E).view(M, k).cuda()
    ids[17, 2] = -1
    z = torch.randn(M, E, device="cuda")
    grad, _, counts, _ = tp.tppo_balance_loss_backward(z, ids)
    assert int(counts.max() - counts.min()) in (1, 2)
    _check_nearly_even(grad[:3000], z[:3000], counts, k, M)


@pytest.mark.parametrize("M", [40, 5000])                          # one workgroup; many
@pytest.mark.parametrize("E,k,tokens", [(256, 8, 10 ** 7), (256, 8, 10 ** 9), (60, 2, 123_456_789)])
def test_counts_of_a_large_batch_one_apart(M, E, k, tokens):
    z, counts = _nearly_even(E, tokens * k // E, M)
    ids = torch.zeros(M, k, dtype=torch.int32, device="cuda")
    grad, _, own, _ = tp.tppo_balance_loss_backward(z, ids, counts_in=counts, token_denominator=tokens)
    assert own.tolist() == [M * k] + [0] * (E - 1)
    _check_nearly_even(grad, z, counts, k, tokens)


@pytest.mark.parametrize("E,M", [(8, 500_000), (100, 77_536), (600, 60_000)])
def test_means_over_many_rows_keep_their_digits(E, M):
    """A workgroup adds up its rows in fp32: eight of a thread for 500 000 of 8 experts, 10 of 100 (32 rows at a time in each of 512), 15 of
    600 (8 rows); its lanes, wavefronts and the probability itself are the other roundings."""
    z = torch.randn(M // 4, E, device="cuda")
    rows = torch.randint(0, M // 4, (M,), dtype=torch.int32, device="cuda")
    ids = torch.zeros(M // 4, 1, dtype=torch.int32, device="cuda")
    loss, _, mean_prob = tp.tppo_balance_loss(z, ids, rows=rows)
    p = torch.softmax(z.double(), 1)[rows.long()].mean(0).cpu().numpy()
    worst = float((np.abs(mean_prob.double().cpu().numpy() - p) / p).max() / U)
    assert worst <= 64 + 15 + 16, worst
    assert abs(float(loss) - E * p[0]) <= (64 + 15 + 20) * U * E * p[0]
