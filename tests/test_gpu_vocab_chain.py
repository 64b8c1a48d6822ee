"""GPU tests of the embedding lookup and the vocabulary losses as a program uses them: a model over a tied table, its
gradients against differences, captured graphs, streams, workspaces, and sizes that go through several pieces."""
import pytest
import torch

import paper_2103_00959_amd as cg
import vocab_exact as ex

pytestmark = pytest.mark.gpu


class Tied:
    """Rows of a table, a typed layer over them, and the table again as the vocabulary: loss and gradients."""

    def __init__(self, n=300, V=900, k=64, dt=torch.bfloat16, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.table = (torch.randn((V, k), generator=g) * k ** -0.5).to(dt).cuda()
        self.W = (torch.randn((3, k, k), generator=g) * k ** -0.5).to(dt).cuda()
        self.offsets = torch.tensor([0, n // 3, n // 2, n], dtype=torch.int32).cuda()
        self.index = torch.randint(-1, V, (n,), generator=g, dtype=torch.int32).cuda()
        self.target = torch.randint(-1, V, (n,), generator=g, dtype=torch.int32).cuda()
        self.dloss = torch.full((n,), 1.0 / n).cuda()
        self.scale, self.V = float(k) ** 0.5, V

    def step(self):
        H = cg.embedding(self.table, self.index, scale=self.scale)
        Y = cg.grouped_linear(H, self.W, self.offsets, act="relu")
        loss, lse = cg.linear_cross_entropy(Y, self.table, self.target)
        head = cg.linear_cross_entropy_backward(self.dloss, Y, self.table, self.target, loss, lse)
        layer = cg.grouped_linear_backward(head["dX"], self.W, self.offsets, X=H, Y=Y, act="relu")
        dtable = cg.embedding_backward(layer["dX"], self.index, self.V, scale=self.scale, out=head["dW"], accumulate=True)
        return loss, dtable, layer["dW"]


def reference(m):
    """The same step in 64 bits by autograd, on the CPU."""
    T, W = (t.double().cpu().requires_grad_() for t in (m.table, m.W))
    index, target = m.index.long().cpu(), m.target.long().cpu()
    H = T[index.clamp(min=0)] * m.scale * (index >= 0)[:, None]
    o = m.offsets.tolist()
    Y = torch.cat([torch.relu(H[a:b] @ W[g].t()) for g, (a, b) in enumerate(zip(o, o[1:]))])
    logp = torch.log_softmax(Y @ T.t(), 1)
    loss = -logp.gather(1, target.clamp(min=0)[:, None])[:, 0] * (target >= 0)
    (loss * m.dloss.double().cpu()).sum().backward()
    return loss.detach(), T.grad, W.grad


def rel(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("dt,step", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
def test_a_model_over_a_tied_table(dt, step):
    """Tolerance: a value of the chain is rounded to 16 bits at most 7 times on its way (H, Y, dz, dX, dZ, dH, and the
    gradient itself), each by half a step at most; errors of the forward reach the gradients through exp(z), whose
    logits (|z| up to about 8 here, of Y rounded twice) are off by 2 half steps of 8: 16 more."""
    m = Tied(dt=dt)
    loss, dT, dW = m.step()
    want = reference(m)
    assert float((loss.double().cpu() - want[0]).abs().max()) <= 2 * 16 * step
    assert rel(dT, want[1]) <= 23 * step and rel(dW, want[2]) <= 23 * step


def test_gradients_are_slopes_of_the_loss():
    """Differences of the fp16 losses along a direction that table and features hold exactly (steps of 2^-6 on values
    of few bits), against the gradients: (L(+h) - L(-h)) / 2h is off by h^2 |L'''| / 6, and by the rounding of loss
    and gradients (2^-11 of each term)."""
    g = torch.Generator().manual_seed(3)
    n, V, k, h = 60, 200, 32, 2.0 ** -6
    X = (torch.randint(-8, 9, (n, k), generator=g) / 16.0)
    W = (torch.randint(-8, 9, (V, k), generator=g) / 16.0)
    t = torch.randint(0, V, (n,), generator=g, dtype=torch.int32).cuda()
    b = torch.randn(V, generator=g).cuda()
    w = torch.rand(n, generator=g).cuda()
    for which in ("dX", "dW", "db"):
        D = torch.randint(-1, 2, {"dX": (n, k), "dW": (V, k), "db": (V,)}[which], generator=g).double()

        def total(s):
            x = (X + s * D if which == "dX" else X).half().cuda()
            y = (W + s * D if which == "dW" else W).half().cuda()
            loss, lse = cg.linear_cross_entropy(x, y, t, b + s * D.float().cuda() if which == "db" else b)
            return float((loss.double() * w.double()).sum()), loss, lse

        _, loss, lse = total(0.0)
        got = cg.linear_cross_entropy_backward(w, X.half().cuda(), W.half().cuda(), t, loss, lse, b)[which]
        slope = (total(h)[0] - total(-h)[0]) / (2 * h)
        size = float((got.double().cpu().abs() * D.abs()).sum())
        # along the direction a logit moves by |d| <= 16 h (|x| |D| over 32 terms of up to 1/2) or h (the bias); the
        # third derivative of log sum exp is at most |d / h|^3, and w sums to n
        third = n * (16.0 if which != "db" else 1.0) ** 3
        fp32 = n * 2.0 ** -20 / h
        assert abs(slope - float((got.double().cpu() * D).sum())) <= h * h * third / 6 + 2.0 ** -11 * 2 * size + fp32


def step_of(m, K=0):
    if K == 0:
        return list(m.step())
    X = cg.embedding(m.table, m.index, scale=m.scale)
    loss, lse, logp = cg.linear_distill(X, m.table, m.entries, m.teacher, temperature=2.0)
    o = cg.linear_distill_backward(m.dloss, X, m.table, m.entries, m.teacher, lse, logp, m.bias0, temperature=2.0)
    return [loss, lse, logp, o["dX"], o["dW"], o["db"]]


def fresh(m, seed):
    """New contents in place."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    m.table.copy_((torch.randn(m.table.shape, generator=g, device="cuda") * 0.2).to(m.table.dtype))
    m.index.copy_(torch.randint(-1, m.V, m.index.shape, generator=g, device="cuda", dtype=torch.int32))
    m.target.copy_(torch.randint(-1, m.V, m.target.shape, generator=g, device="cuda", dtype=torch.int32))
    m.dloss.copy_(torch.rand(m.dloss.shape, generator=g, device="cuda"))
    if hasattr(m, "entries"):
        m.entries.copy_(torch.randint(-1, m.V, m.entries.shape, generator=g, device="cuda", dtype=torch.int32))
        m.teacher.copy_(torch.randn(m.teacher.shape, generator=g, device="cuda"))


def model(K, seed=0, n=300):
    m = Tied(n=n, seed=seed)
    if K:
        m.entries = torch.zeros((n, K), dtype=torch.int32, device="cuda")
        m.teacher = torch.zeros((n, K), device="cuda")
        m.bias0 = torch.zeros(m.V, device="cuda")
    return m


@pytest.mark.parametrize("K", [0, 6])
@pytest.mark.parametrize("n", [16, 40, 300, 9000, 40_000])
def test_captured_steps_replay(n, K):
    """A whole step captured into a graph: every replay, with eager work and new contents between, equals the eager
    one (the number of rows that count changes from replay to replay)."""
    m = model(K, n=n)
    fresh(m, 99)
    step_of(m, K)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step_of(m, K)
    for seed in range(4):
        fresh(m, seed)
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step_of(m, K)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_two_captured_graphs_with_workspaces_of_their_own():
    ms = [model(0, seed=1), model(6, seed=2)]
    for i, m in enumerate(ms):
        fresh(m, i)
    wanted = [step_of(ms[0], 0), step_of(ms[1], 6)]
    torch.cuda.synchronize()
    graphs, held = [], []
    for m, K in zip(ms, (0, 6)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(step_of(m, K))
    for order in ((0, 1), (1, 0), (0, 0, 1), (1, 1, 0)):
        for i in order:
            graphs[i].replay()
        step_of(ms[0], 0)
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(held[i], wanted[i])), (order, i)


def test_steps_on_two_streams_at_once():
    ms = [model(0, seed=3, n=2000), model(0, seed=4, n=2000)]
    want = [step_of(m) for m in ms]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(step_of(ms[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        for o in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(o, want[i]))


def test_given_workspaces_and_outputs():
    """Workspaces that hold anything, of any type, larger than asked for; outputs that hold NaN; the same bits."""
    m = model(0, seed=5, n=700)
    n, V, k = 700, m.V, m.table.shape[1]
    X = cg.embedding(m.table, m.index)
    loss, lse = cg.linear_cross_entropy(X, m.table, m.target)
    ws = torch.full((cg.linear_loss_workspace(n, V, k) // 4 + 5,), float("nan"), device="cuda")
    l2, s2 = torch.full_like(loss, float("nan")), torch.full_like(lse, float("nan"))
    r = cg.linear_cross_entropy(X, m.table, m.target, loss=l2, lse=s2, workspace=ws)
    assert r[0] is l2 and r[1] is s2 and torch.equal(l2, loss) and torch.equal(s2, lse)
    zeros = torch.zeros(V, device="cuda")
    whole = cg.linear_cross_entropy_backward(m.dloss, X, m.table, m.target, loss, lse, zeros)
    ws = torch.full((cg.linear_loss_backward_workspace(n, V, k) // 4 + 5,), float("nan"), device="cuda")
    out = {name: torch.full_like(t, float("nan")) for name, t in whole.items()}
    again = cg.linear_cross_entropy_backward(m.dloss, X, m.table, m.target, loss, lse, zeros, out=out, workspace=ws)
    assert all(again[name] is out[name] and torch.equal(out[name], whole[name]) for name in whole)
    dT = cg.embedding_backward(X, m.index, V)
    ws = torch.full((cg.embedding_backward_workspace(n, V, k) // 4 + 5,), float("nan"), device="cuda")
    assert torch.equal(cg.embedding_backward(X, m.index, V, out=torch.full_like(dT, float("nan")), workspace=ws), dT)
    with pytest.raises(cg.CogdlError, match="contiguous"):
        cg.linear_cross_entropy(X.t().contiguous().t(), m.table, m.target)
    with pytest.raises(cg.CogdlError, match="workspace has"):
        cg.embedding_backward(X, m.index, V, workspace=ws[:8])


def random_layer(n, V, k, dt, seed, pad=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn((n, k), generator=g, device="cuda").to(dt)
    W = (torch.randn((V, k), generator=g, device="cuda") * 2 * k ** -0.5).to(dt)
    t = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    t[torch.rand(n, generator=g, device="cuda") < pad] = -1
    return X, W, t, torch.randn(V, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda") / n


def one_hot(t, V):
    held = ((t >= 0) & (t < V))[:, None]
    return t[:, None], held.double(), held, held[:, 0]


@pytest.mark.parametrize("n,V,k,dt", [(8192, 70001, 24, torch.bfloat16), (8100, 66000, 18, torch.float16),
                                      (2560, 4096, 264, torch.bfloat16), (1024, 20000, 1024, torch.float16),
                                      (3000, 9000, 515, torch.bfloat16), (30000, 41, 48, torch.bfloat16),
                                      (150_000, 3, 130, torch.float16), (70_000, 200, 260, torch.bfloat16)])
def test_several_pieces_and_wide_tiles(n, V, k, dt):
    """Vocabularies in pieces with a short last one, tiles of 256 x 256 and of 128 x 128, odd widths, many rows over a
    few classes (dW in parts of the rows, dX without slices); with and without the bias and its gradient (kernels of
    their own)."""
    X, W, t, b, g = random_layer(n, V, k, dt, n + V)
    for bias in (b, None):
        loss, lse = cg.linear_cross_entropy(X, W, t, bias)
        f = ex.loss(X, W, *one_hot(t, V), bias)
        ex.close("loss", loss, *f["loss"])
        ex.close("lse", lse, *f["lse"])
        del f
        out = cg.linear_cross_entropy_backward(g, X, W, t, loss, lse, bias)
        want = ex.gradients(X, W, *one_hot(t, V), g, bias)
        for name in ("dX", "dW") + (("db",) if bias is not None else ()):
            ex.close(name, out[name], *want[name])
        del out, want


def test_statistics_in_blocks_of_rows():
    """A vocabulary whose statistics of all rows would pass 256 MB: by blocks of rows.  (The same rows given apart join
    their slots in other groups, so they are held to the bound, not to the same bits.)"""
    n, V, k = 2300, 1_050_000, 16
    X, W, t, b, _ = random_layer(n, V, k, torch.bfloat16, 5)
    loss, lse = cg.linear_cross_entropy(X, W, t, b)
    for rows in (slice(0, 50), slice(2020, 2070), slice(2250, 2300)):
        part, part_lse = cg.linear_cross_entropy(X[rows].contiguous(), W, t[rows].contiguous(), b)
        f = ex.loss(X[rows], W, *one_hot(t[rows], V), b)
        for got, got_lse in ((loss[rows], lse[rows]), (part, part_lse)):
            ex.close("loss", got, *f["loss"])
            ex.close("lse", got_lse, *f["lse"])


def test_a_table_past_4_gib():
    """W behind the 4 GiB that 32-bit offsets reach: targets, logits and dW at both ends."""
    V, k, n = 2_200_000, 1024, 130
    W = torch.zeros((V, k), dtype=torch.bfloat16, device="cuda")
    X = torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    X[:, 0] = 1.0
    W[V - 1, 0], W[1, 0] = 8.0, 4.0
    t = torch.full((n,), V - 1, dtype=torch.int32, device="cuda")
    t[::2] = 1
    z = torch.tensor([4.0, 8.0], dtype=torch.float64)
    lse = torch.log(z.exp().sum() + (V - 2))
    loss, got = cg.linear_cross_entropy(X, W, t)
    assert torch.allclose(got.double().cpu(), lse.expand(n), rtol=1e-6)
    assert torch.allclose(loss.double().cpu(), lse - torch.where(t.cpu() == 1, z[0], z[1]), rtol=1e-6)
    g = torch.full((n,), 1.0 / n, device="cuda")
    o = cg.linear_cross_entropy_backward(g, X, W, t, loss, got)
    want = torch.exp(z - lse) - 0.5
    dW = o["dW"][[1, V - 1], 0].double().cpu()
    # half the rows' terms near p, half near p - 1, each rounded, and the sum
    assert ((dW - want).abs() <= 2.0 ** -8 * (0.5 + want.abs())).all()
    other = o["dW"][[0, 2, V - 2], 0].double().cpu()
    assert ((other - torch.exp(-lse)).abs() <= 2.0 ** -7 * torch.exp(-lse)).all()
    assert not o["dW"][:, 1:8].any()
