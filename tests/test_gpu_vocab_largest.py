"""GPU tests of the vocabulary losses at their largest sizes: vocabularies that 32 bits just count, the most rows,
features past 4 GiB."""
import math

import pytest
import torch

import paper_2103_00959_amd as cg
import vocab_exact as ex

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


def one_hot(t, V):
    held = ((t >= 0) & (t < V))[:, None]
    return t[:, None], held.double(), held, held[:, 0]


@pytest.mark.parametrize("K", [0, 3])
def test_the_most_rows(K):
    """2^24 rows over 3 answers."""
    n, V, k = 2 ** 24, 3, 8
    g = torch.Generator(device="cuda").manual_seed(K)
    X = torch.randn((n, k), generator=g, device="cuda").half()
    W = torch.randn((V, k), generator=g, device="cuda").half()
    b = torch.randn(V, generator=g, device="cuda")
    w = torch.rand(n, generator=g, device="cuda") / n
    index = torch.randint(-1, V + 1, (n, max(K, 1)), generator=g, device="cuda", dtype=torch.int32)
    if K:
        teacher = torch.randn((n, K), generator=g, device="cuda")
        share = ex.teacher_share(index, teacher, V, 1.0)
        loss, lse, logp = cg.linear_distill(X, W, index, teacher, b)
        out = cg.linear_distill_backward(w, X, W, index, teacher, lse, logp, b)
    else:
        t = index[:, 0].contiguous()
        share = one_hot(t, V)[1:]
        loss, lse = cg.linear_cross_entropy(X, W, t, b)
        out = cg.linear_cross_entropy_backward(w, X, W, t, loss, lse, b)
    f = ex.loss(X, W, index, *share, b)
    ex.close("loss", loss, *f["loss"])
    ex.close("lse", lse, *f["lse"])
    del f
    want = ex.gradients(X, W, index, *share, w, b)
    for name in ("dX", "dW", "db"):
        ex.close(name, out[name], *want[name])


def test_features_past_4_gib():
    """X and dX behind the 4 GiB that 32-bit offsets reach.  Only some rows weigh anything, so that dW is theirs."""
    n, V, k = 3_700_000, 40, 640
    g = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randn((n, k), generator=g, device="cuda", dtype=torch.bfloat16)
    W = (torch.randn((V, k), generator=g, device="cuda") * 2 * k ** -0.5).bfloat16()
    b = torch.randn(V, generator=g, device="cuda")
    t = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    at = torch.cat([torch.arange(40), torch.arange(3_355_400, 3_355_480), torch.arange(n - 50, n)]).cuda()
    w = torch.zeros(n, device="cuda")
    w[at] = 0.01
    loss, lse = cg.linear_cross_entropy(X, W, t, b)
    out = cg.linear_cross_entropy_backward(w, X, W, t, loss, lse, b)
    f = ex.loss(X[at], W, *one_hot(t[at], V), b)
    ex.close("loss", loss[at], *f["loss"])
    ex.close("lse", lse[at], *f["lse"])
    want = ex.gradients(X[at], W, *one_hot(t[at], V), w[at], b)
    ex.close("dX", out["dX"][at], *want["dX"])
    ex.close("dW", out["dW"], *want["dW"])
    assert int((out["dX"] != 0).any(1).sum()) == len(at)
