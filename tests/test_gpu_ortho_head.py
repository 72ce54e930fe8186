"""The orthogonalisation of a matrix with a vocabulary's rows: the LM head's gradient, against the iteration in 64 bits on the device."""
import pytest
import torch

from paper_2506_15050_amd import binding as tp

pytestmark = pytest.mark.gpu

# the result's rounding to bf16, 1.7e-3 of its norm as a rule, and as much again for the arithmetic; an element: its rounding and eight
# standard deviations of an error of 3.6e-3 of the elements' root mean square
NORM, ELEMENT = 2.0 ** -8, 8 * 3.6e-3


def _iteration(g):
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    x = x / (x.norm() + 1e-7)
    for _ in range(5):
        s = x @ x.t().contiguous()
        x = 3.4445 * x + (-4.7750 * s + 2.0315 * (s @ s)) @ x
    return x.t() if tall else x


# X X^T alone, all steps in one workgroup or by pairs, and products of X, wide and tall
@pytest.mark.parametrize("rows,cols,dtype", [(262144, 1, torch.float32), (3, 262143, torch.float32), (152064, 64, torch.float32), (90, 262144, torch.bfloat16), (152064, 192, torch.float32),
                                             (152065, 1027, torch.bfloat16), (152064, 2112, torch.float32), (2049, 152063, torch.float32)])
def test_a_vocabulary_of_rows(rows, cols, dtype):
    g = torch.randn(rows, cols, device="cuda")
    few = torch.randn(rows, 4, device="cuda") @ torch.randn(4, cols, device="cuda")      # tokens that come often
    g = (g + few).to(dtype)
    del few
    out = tp.tppo_orthogonalize(g).double()
    want = _iteration(g)
    rms = want.norm() / want.numel() ** 0.5
    assert float((out - want).norm() / want.norm()) <= NORM
    out.sub_(want).abs_()
    assert bool((out <= 2.0 ** -8 * want.abs() + ELEMENT * rms).all())
