"""GPU tests of the vocabulary losses' gradients under weights whose dz fp16 could not hold by itself."""
import pytest
import torch

import paper_2103_00959_amd as cg
import vocab_exact as ex

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which,x,w", [("dX", 2.0 ** -11, 2.0 ** 11), ("dW", 2.0 ** 12, 2.0 ** -12)])
@pytest.mark.parametrize("distill", [False, True])
def test_small_weights_in_fp16(which, x, w, distill):
    """Weights under 2^-25: every dz, unscaled, would round to zero in fp16.  Large features (or a large table) bring
    the gradient back into its range: most of it lies far above the bound, which all zeros would not pass."""
    g = torch.Generator().manual_seed(6)
    n, V, k = 150, 300, 48
    X = (torch.randn((n, k), generator=g) * x).half()
    W = (torch.randn((V, k), generator=g) * w * k ** -0.5).half()
    b = torch.randn(V, generator=g)
    weights = (torch.rand(n, generator=g) + 1) * 2.0 ** -27
    t = torch.randint(0, 40, (n, 1), generator=g, dtype=torch.int32)
    t[::9] = -1
    d = [v.cuda() for v in (X, W, t, b, weights)]
    held = t >= 0
    if distill:
        teacher = torch.zeros((n, 1), device="cuda")
        loss, lse, logp = cg.linear_distill(d[0], d[1], d[2], teacher, d[3])
        out = cg.linear_distill_backward(d[4], d[0], d[1], d[2], teacher, lse, logp, d[3])
    else:
        loss, lse = cg.linear_cross_entropy(d[0], d[1], d[2][:, 0].contiguous(), d[3])
        out = cg.linear_cross_entropy_backward(d[4], d[0], d[1], d[2][:, 0].contiguous(), loss, lse, d[3])
    want = ex.gradients(X, W, t, held.double(), held, held[:, 0], weights, b)
    value, bound = want[which]
    rows = held[:, 0] if which == "dX" else torch.arange(V) < 40          # (the answers that are targets)
    # (dX: about one term of weight 2^-26.4 times a normal W of deviation 296, 3.3e-6, over a bound of at least 2^-24:
    # four of them are 0.073 deviations, and 94% of normal values lie past that)
    assert float((value[rows].abs() > 4 * bound[rows]).double().mean()) > 0.9
    for name in ("dX", "dW", "db"):
        ex.close(name, out[name], *want[name])


@pytest.mark.parametrize("n", [150, 20_000])
@pytest.mark.parametrize("wrong", [float("inf"), -float("inf"), float("nan")])
def test_small_weights_beside_one_that_is_not_finite(wrong, n):
    """dX of the other rows is what it is without that row."""
    g = torch.Generator().manual_seed(7)
    V, k = 300, 48
    X = (torch.randn((n, k), generator=g) * 2.0 ** -11).half()
    W = (torch.randn((V, k), generator=g) * 2.0 ** 11 * k ** -0.5).half()
    weights = (torch.rand(n, generator=g) + 1) * 2.0 ** -27
    t = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    held = t[:, None] >= 0
    want, bound = (v[torch.arange(n) != 5] for v in ex.gradients(X, W, t[:, None], held.double(), held, held[:, 0], weights)["dX"])
    weights[5] = wrong
    d = [v.cuda() for v in (X, W, t)]
    loss, lse = cg.linear_cross_entropy(*d)
    dX = cg.linear_cross_entropy_backward(weights.cuda(), *d, loss, lse)["dX"].cpu()
    assert not torch.isfinite(dX[5]).any()
    ex.close("dX", dX[torch.arange(n) != 5], want, bound)
    one = torch.ones((n, 1))
    loss, lse, logp = cg.linear_distill(d[0], d[1], d[2][:, None].contiguous(), one.cuda())
    dX = cg.linear_distill_backward(weights.cuda(), d[0], d[1], d[2][:, None].contiguous(), one.cuda(), lse, logp)["dX"].cpu()
    assert not torch.isfinite(dX[5]).any()
    ex.close("dX", dX[torch.arange(n) != 5], want, bound)
