"""GPU tests of the vocabulary losses at the largest vocabularies that 32 bits count."""
import math

import pytest
import torch

import paper_2103_00959_amd as cg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [2 ** 31 - 60, 2 ** 31 - 1])
@pytest.mark.parametrize("k", [1, 2])
def test_no_logit_behind_the_last_answer(V, k):
    """Every logit is -64: lse = log V - 64, where one logit of 0 behind the last answer, in the last 64 columns, would
    make it about 0.  Bounds (u = 2^-24): exponents 8 u (2 x 64 + 2), sums 2^8 u, the logarithm's 8 u x 43: 1e-4.
    dW is -8 g / V, in bf16, but of the targets' rows."""
    W = torch.zeros((V, k), dtype=torch.bfloat16, device="cuda")
    W[:, 0] = 8.0
    X = torch.zeros((2, k), dtype=torch.bfloat16, device="cuda")
    X[:, 0] = -8.0
    t = torch.tensor([V - 1, 5], dtype=torch.int32, device="cuda")
    loss, lse = cg.linear_cross_entropy(X, W, t)
    assert (lse.double().cpu() - (math.log(V) - 64)).abs().max() <= 1e-4
    assert (loss.double().cpu() - math.log(V)).abs().max() <= 1e-4
    g = torch.full((2,), 0.5, device="cuda")
    dW = cg.linear_cross_entropy_backward(g, X, W, t, loss, lse, out={"dX": None})["dW"]
    # half a step of bf16 in dz and one in dW (2^-8 each), and p: its exponent by the bound above and the forward's 1e-4
    want = -8.0 / V
    off = (dW[:, 0].double() - want).abs() > (2.0 ** -7 + 2.0 ** -16 + 2.1e-4) * abs(want)
    assert int(off.sum()) == 2 and off[V - 1] and off[5]
    assert dW[V - 1, 0] == 4.0 and dW[5, 0] == 4.0
    assert k == 1 or not dW[:, 1].any()
