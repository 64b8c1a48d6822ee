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


def layer(n, V, k, K, dt, seed):
    """Rows on the device, some without an entry; answers twice in a row, outside the vocabulary, taken out by a
    teacher's -inf; and entries at the columns around multiples of 256, where pieces and tiles meet."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn((n, k), generator=g, device="cuda").to(dt)
    W = (torch.randn((V, k), generator=g, device="cuda") * 2 * k ** -0.5).to(dt)
    index = torch.randint(0, V, (n, K), generator=g, device="cuda", dtype=torch.int32)
    border = torch.randint(0, (V + 255) // 256, (n,), generator=g, device="cuda", dtype=torch.int32) * 256
    for e, off in enumerate((-1, 0, 1)[:K]):
        index[e::3, e] = (border + off)[e::3].clamp(0, V - 1)
    index[::5, K - 1] = V - 1
    if K > 3:
        index[1::7, 3] = index[1::7, 0]
        index[2::7, 1] = V + 3
    index[3::11] = -1
    teacher = torch.randn((n, K), generator=g, device="cuda") * 2 + 1
    teacher[4::9, 0] = -INF
    return X, W, index, teacher, torch.randn(V, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda") / n


@pytest.mark.parametrize("n,V,k,K,T,dt", [(8192, 70001, 24, 8, 1.0, torch.bfloat16), (8100, 66000, 18, 3, 2.0, torch.float16),
                                          (2560, 4096, 264, 5, 1.0, torch.bfloat16), (1024, 20000, 1024, 7, 2.0, torch.float16),
                                          (16, 1000, 264, 4, 1.0, torch.float16), (1, 3000, 64, 2, 3.0, torch.bfloat16),
                                          (40, 3000, 32, 1024, 2.0, torch.bfloat16), (20, 500, 33, 1024, 1.0, torch.float16)])
def test_several_pieces_wide_tiles_and_many_entries(n, V, k, K, T, dt):
    """Entries in every piece of the vocabulary, at the pieces' and the tiles' borders; tiles of 256 x 256; up to the most
    entries of a row."""
    X, W, index, teacher, b, g = layer(n, V, k, K, dt, n + K)
    q, held, live = ex.teacher_share(index, teacher, V, T)
    for bias in (b, None):
        loss, lse, logp = cg.linear_distill(X, W, index, teacher, bias, temperature=T)
        f = ex.loss(X, W, index, q, held, live, bias, T)
        for name, got in (("loss", loss), ("lse", lse), ("logp", logp)):
            ex.close(name, got, *f[name])
        del f
        out = cg.linear_distill_backward(g, X, W, index, teacher, lse, logp, bias, temperature=T)
        want = ex.gradients(X, W, index, q, held, live, g, bias, T)
        for name in ("dX", "dW") + (("db",) if bias is not None else ()):
            ex.close(name, out[name], *want[name])
        del out, want


def by_autograd(X, W, index, teacher, b, g, T):
    """dX, dW and db of sum g T^2 KL(q || softmax(z / T)) in 64 bits by autograd."""
    X, W, b = (v.double().requires_grad_() for v in (X, W, b))
    V = W.shape[0]
    held = (index >= 0) & (index < V)
    t = (teacher.double() / T).masked_fill(~held, -INF)
    live = (t > -INF).any(1)
    q = torch.softmax(t[live], 1)
    logp = torch.log_softmax((X[live] @ W.t() + b) / T, 1).gather(1, index[live].clamp(0, V - 1).long())
    kl = torch.where(q > 0, q * (torch.where(q > 0, q, 1.0).log() - logp), 0.0).sum(1)
    (T * T * (kl * g.double()[live])).sum().backward()
    return {"dX": X.grad, "dW": W.grad, "db": b.grad}


@pytest.mark.parametrize("T", [1.0, 0.5, 4.0])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_gradients_are_autograds(dt, T):
    X, W, index, teacher, b, g = layer(150, 600, 40, 9, dt, 21)
    loss, lse, logp = cg.linear_distill(X, W, index, teacher, b, temperature=T)
    out = cg.linear_distill_backward(g, X, W, index, teacher, lse, logp, b, temperature=T)
    value = by_autograd(*(v.cpu() for v in (X, W, index, teacher, b, g)), T)
    bounds = ex.gradients(X, W, index, *ex.teacher_share(index, teacher, 600, T), g, b, T)
    for name in ("dX", "dW", "db"):
        ex.close(name, out[name].cpu(), value[name], bounds[name][1].cpu())


@pytest.mark.parametrize("T", [1.0, 2.0])
def test_gradients_are_slopes_of_the_loss(T):
    """Differences of the fp16 losses along a direction that table and features hold exactly (steps of 2^-6 on values
    of few bits), against the gradients.  A logit moves by |d| <= 16 h (|x| |D| over 32 terms of up to 1/2) or h (the
    bias).  The loss is T^2 (log sum exp(z / T) - ...), its third derivative at most T^2 |d / (h T)|^3 a row, so the
    difference is off by h^2 / 6 of w times that; the gradients by their roundings (2^-11 of dz and of the sums); the
    losses' fp32 by 2^-20 a row (values up to 16 T^2, of 2^-24), over h."""
    g = torch.Generator().manual_seed(4)
    n, V, k, K, h = 60, 200, 32, 6, 2.0 ** -6
    X = torch.randint(-8, 9, (n, k), generator=g) / 16.0
    W = torch.randint(-8, 9, (V, k), generator=g) / 16.0
    index = torch.randint(-1, V, (n, K), generator=g, dtype=torch.int32).cuda()
    teacher = torch.randn((n, K), generator=g).cuda()
    b, w = torch.randn(V, generator=g).cuda(), torch.rand(n, generator=g).cuda()
    for which in ("dX", "dW", "db"):
        D = torch.randint(-1, 2, {"dX": (n, k), "dW": (V, k), "db": (V,)}[which], generator=g).double()

        def at(s):
            x = (X + s * D if which == "dX" else X).half().cuda()
            y = (W + s * D if which == "dW" else W).half().cuda()
            z = b + s * D.float().cuda() if which == "db" else b
            r = cg.linear_distill(x, y, index, teacher, z, temperature=T)
            return float((r[0].double() * w.double()).sum()), r

        _, (loss, lse, logp) = at(0.0)
        assert float(loss.abs().max()) <= 16 * T * T
        got = cg.linear_distill_backward(w, X.half().cuda(), W.half().cuda(), index, teacher, lse, logp, b, temperature=T)
        got = got[which].double().cpu()
        slope = (at(h)[0] - at(-h)[0]) / (2 * h)
        third = n * (16.0 if which != "db" else 1.0) ** 3 / T
        fp32 = n * T * T * 2.0 ** -20 / h
        size = float((got.abs() * D.abs()).sum())
        assert abs(slope - float((got * D).sum())) <= h * h * third / 6 + 2.0 ** -11 * 2 * size + fp32


def test_a_loss_below_zero():
    """The same answer twice, each entry with half the teacher's weight, and a student that is sure of it: log 1/2, T^2
    times."""
    W = torch.zeros((50, 8), dtype=torch.bfloat16, device="cuda")
    W[7, 0] = 64.0
    X = torch.ones((3, 8), dtype=torch.bfloat16, device="cuda")
    index = torch.full((3, 2), 7, dtype=torch.int32, device="cuda")
    for T in (1.0, 2.0):
        loss, _, logp = cg.linear_distill(X, W, index, torch.zeros((3, 2), device="cuda"), temperature=T)
        assert (logp.abs() <= 1e-5).all()
        assert ((loss.double() + T * T * 0.6931471805599453).abs() <= 2e-5 * T * T).all()
