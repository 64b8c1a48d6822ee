"""GPU tests of the distillation's gradients where a row is not finite, against their definition in 64 bits with the
bounds of vocab_exact."""
import pytest
import torch

import paper_2103_00959_amd as cg
import vocab_exact as ex

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def close(name, got, value, bound):
    """Within the bound where the definition is finite, and the same infinity or NaN elsewhere."""
    got, value, bound = got.double().cpu(), value.cpu(), bound.cpu()
    fin = torch.isfinite(value)
    for what in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(what(got), what(value)), f"{name}: {what.__name__} {int(what(got).sum())}, expected {int(what(value).sum())}"
    ex.close(name, got[fin], value[fin], bound[fin])


def problem(n, V, k, K, dt, seed):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn((n, k), generator=g).to(dt)
    W = (torch.randn((V, k), generator=g) * k ** -0.5).to(dt)
    index = torch.randint(0, V, (n, K), generator=g, dtype=torch.int32)
    index[:, 1] = index[:, 0]                                  # the same answer twice
    index[::4, 2] = -1
    # shares far above a probability of the student (about 1 / V): the sign of p - q is sure
    teacher = torch.rand((n, K), generator=g)
    return X, W, index, teacher, torch.randn(V, generator=g), torch.rand(n, generator=g) + 0.1


def run(X, W, index, teacher, b, g, T, **out):
    d = [v.cuda() for v in (X, W, index, teacher, b)]
    loss, lse, logp = cg.linear_distill(*d, temperature=T)
    return loss, cg.linear_distill_backward(g.cuda(), *d[:4], lse, logp, d[4], temperature=T, out=out or None)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("wrong", [NAN, INF])
@pytest.mark.parametrize("n,V,K", [(40, 700, 5), (300, 1000, 70)])
def test_db_beside_a_teacher_gone_wrong(n, V, K, wrong, dt):
    """A teacher's row that holds NaN or +inf has no shares: its loss, its dX, and its entries' rows of dW and values of
    db are NaN, and nothing else is."""
    T = 2.0
    X, W, index, teacher, b, g = problem(n, V, 32, K, dt, n + K)
    teacher[9, 3] = wrong
    teacher[17, 0] = wrong
    teacher[8, 2] = wrong                                      # (an entry that does not count: nothing)
    q, held, live = ex.teacher_share(index, teacher, V, T)
    want = ex.gradients(X, W, index, q, held, live, g, b, T)
    loss, got = run(X, W, index, teacher, b, g, T)
    bad = torch.zeros(n, dtype=torch.bool)
    bad[9] = bad[17] = True
    assert torch.equal(torch.isnan(loss).cpu(), bad) and 0 < int(torch.isnan(want["db"][0]).sum()) <= 2 * K
    for name in ("dX", "dW", "db"):
        close(name, got[name], *want[name])
    alone = run(X, W, index, teacher, b, g, T, dX=None, dW=None)[1]["db"]
    close("db", alone, *want["db"])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("weights", [{3: INF}, {3: -INF}, {3: INF, 20: INF}, {3: INF, 20: -INF}, {3: NAN}, {3: INF, 20: NAN}])
@pytest.mark.parametrize("n,V,K", [(40, 700, 5), (200, 300, 6)])
def test_db_of_infinite_weights(n, V, K, weights, dt):
    """dloss = +-inf: db is an infinity of the sign of p - q, NaN where two rows' signs differ."""
    X, W, index, teacher, b, g = problem(n, V, 32, K, dt, n + 1)
    for i, w in weights.items():
        g[i] = w
    q, held, live = ex.teacher_share(index, teacher, V, 1.0)
    value, bound = ex.gradients(X, W, index, q, held, live, g, b)["db"]
    assert not torch.isfinite(value).any()
    close("db", run(X, W, index, teacher, b, g, 1.0, dX=None, dW=None)[1]["db"], value, bound)


def test_db_of_a_student_gone_wrong():
    """NaN in a row of X: all of dW and db; a row that is left out: nothing."""
    X, W, index, teacher, b, g = problem(60, 400, 32, 5, torch.float16, 3)
    index[11] = -1
    X[11, 4] = NAN
    g[11] = INF
    q, held, live = ex.teacher_share(index, teacher, 400, 1.0)
    _, got = run(X, W, index, teacher, b, g, 1.0)
    for name, t in got.items():
        assert torch.isfinite(t).all(), name
    X[12, 4] = NAN
    loss, got = run(X, W, index, teacher, b, g, 1.0)
    assert torch.isnan(loss[12]) and torch.isnan(got["dX"][12]).all() and int(torch.isnan(got["dX"]).any(1).sum()) == 1
    assert torch.isnan(got["dW"]).all() and torch.isnan(got["db"]).all()


def test_db_beside_a_teacher_gone_wrong_in_several_pieces():
    """Entries of one row in every piece of the vocabulary, at their borders."""
    n, V, K = 8192, 70001, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    X = torch.randn((n, 16), generator=g, device="cuda").bfloat16()
    W = torch.randn((V, 16), generator=g, device="cuda").mul_(0.25).bfloat16()
    index = torch.randint(0, V, (n, K), generator=g, device="cuda", dtype=torch.int32)
    teacher = torch.rand((n, K), generator=g, device="cuda")
    b, w = torch.zeros(V, device="cuda"), torch.full((n,), 1.0 / n, device="cuda")
    at = torch.tensor([0, 23551, 23552, 23553, 47103, 47104, 60000, V - 1], dtype=torch.int32, device="cuda")
    index[4000] = at
    teacher[4000, 5] = NAN
    loss, lse, logp = cg.linear_distill(X, W, index, teacher, b)
    db = cg.linear_distill_backward(w, X, W, index, teacher, lse, logp, b, out={"dX": None, "dW": None})["db"]
    assert torch.equal(torch.isnan(db).nonzero()[:, 0].int(), at)
