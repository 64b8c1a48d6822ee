"""GPU tests of the softmax cross entropy and the distillation over a vocabulary, against their definition in 64
bits with the bounds of vocab_exact."""
import pytest
import torch

import paper_2103_00959_amd as cg
import vocab_exact as ex

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def layer(n, V, k, dt, seed, bias):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn((n, k), generator=g)
    W = torch.randn((V, k), generator=g) * 2.0 / max(1, k) ** 0.5
    b = torch.randn(V, generator=g) if bias else None
    t = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    if n > 3:
        t[::5] = -1
        t[n // 2] = V
        X = X + (torch.arange(n) % 3)[:, None] * W[t.clamp(0, V - 1).long()]       # some rows are sure
    return X.to(DT[dt]), W.to(DT[dt]), t, b, torch.rand(n, generator=g) + 0.1, g


def dev(t):
    return None if t is None else t.cuda()


def one_hot(t, V):
    held = ((t >= 0) & (t < V))[:, None]
    return t[:, None], held.double(), held, held[:, 0]


def check_cross_entropy(X, W, t, b, g):
    V = W.shape[0]
    d = [dev(v) for v in (X, W, t, b)]
    loss, lse = cg.linear_cross_entropy(*d)
    f = ex.loss(X, W, *one_hot(t, V), b)
    ex.close("loss", loss, *f["loss"])
    ex.close("lse", lse, *f["lse"])
    out = cg.linear_cross_entropy_backward(dev(g), d[0], d[1], d[2], loss, lse, d[3])
    want = ex.gradients(X, W, *one_hot(t, V), g, b)
    for name in ("dX", "dW") + (("db",) if b is not None else ()):
        ex.close(name, out[name], *want[name])
    assert (out["db"] is None) == (b is None)
    return loss, lse, out


SIZES = [(1, 1, 1), (1, 2, 8), (1, 500, 64), (1, 70, 40), (16, 1000, 264), (17, 15, 31), (3, 3000, 4102),
         (33, 4097, 520), (48, 300, 1030), (64, 17, 9), (2, 3, 7), (5, 129, 65), (33, 64, 16), (64, 1000, 128), (130, 257, 100),
         (257, 1433, 33), (300, 700, 602), (1000, 41, 256), (128, 5000, 24), (33000, 41, 16)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("n,V,k", SIZES)
def test_cross_entropy(n, V, k, dt):
    X, W, t, b, g, _ = layer(n, V, k, dt, 11 * n + V + k, (n + V + k) % 2 == 0)
    check_cross_entropy(X, W, t, b, g)


def teacher_rows(n, V, K, g):
    index = torch.randint(0, V, (n, K), generator=g, dtype=torch.int32)
    teacher = torch.randn((n, K), generator=g) * 3 + 5
    if K > 2:
        index[::3, -1] = -1
        index[1::3, 1] = index[1::3, 0]             # the same answer twice
        teacher[2::4, 0] = -torch.inf
    if n > 4:
        index[4] = -1                                # no entry
        teacher[3] = -torch.inf                      # none that weighs anything
        index[2, 0] = V + 7
    return index, teacher


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("n,V,k,K,T", [(1, 1, 1, 1, 1.0), (1, 300, 40, 5, 2.0), (7, 90, 33, 3, 1.0), (65, 1000, 64, 10, 4.0),
                                       (200, 513, 130, 70, 0.5), (20000, 60, 24, 3, 1.0), (300, 2000, 256, 128, 2.0), (40, 700, 16, 300, 1.5)])
def test_distill(n, V, k, K, T, dt):
    X, W, _, b, g, gen = layer(n, V, k, dt, n + V + k + K, K % 2 == 0)
    index, teacher = teacher_rows(n, V, K, gen)
    q, held, live = ex.teacher_share(index, teacher, V, T)
    d = [dev(v) for v in (X, W, index, teacher, b)]
    loss, lse, logp = cg.linear_distill(*d, temperature=T)
    f = ex.loss(X, W, index, q, held, live, b, T)
    for name, got in (("loss", loss), ("lse", lse), ("logp", logp)):
        ex.close(name, got, *f[name])
    out = cg.linear_distill_backward(dev(g), *d[:4], lse, logp, d[4], temperature=T)
    want = ex.gradients(X, W, index, q, held, live, g, b, T)
    for name in ("dX", "dW") + (("db",) if b is not None else ()):
        ex.close(name, out[name], *want[name])


def test_distill_of_one_sure_entry_is_cross_entropy():
    X, W, t, b, g, _ = layer(100, 600, 96, "bf16", 5, True)
    d = [dev(v) for v in (X, W, t, b)]
    loss, lse = cg.linear_cross_entropy(*d)
    dl, dlse, logp = cg.linear_distill(d[0], d[1], d[2][:, None].contiguous(), torch.zeros(100, 1, device="cuda"), d[3])
    assert torch.equal(dlse, lse)
    assert torch.allclose(dl, loss, rtol=0, atol=1e-5) and torch.allclose(-logp[:, 0], loss, rtol=0, atol=1e-5)


def test_rows_left_out_may_hold_anything():
    """NaN and infinities in rows without a target reach no output of another row, and no gradient of W."""
    X, W, t, b, g, _ = layer(200, 300, 72, "f16", 8, True)
    out_rows = (t < 0) | (t >= 300)
    X[out_rows] = float("nan")
    g[out_rows] = float("inf")
    loss, lse, out = check_cross_entropy(X, W, t, b, g)
    assert (loss.cpu()[out_rows] == 0).all() and (lse.cpu()[out_rows] == 0).all()
    assert (out["dX"].cpu()[out_rows] == 0).all()
    # and all of them left out
    t[:] = -1
    loss, lse, out = check_cross_entropy(X, W, t, b, g)
    assert all((out[name] == 0).all() for name in ("dX", "dW", "db"))


def test_answers_taken_out_by_the_bias():
    """-inf in the bias: no probability, no gradient; a target taken out costs an infinite loss."""
    X, W, t, b, g, _ = layer(90, 400, 64, "bf16", 9, True)
    t[t < 0] = 1
    b[::3] = -torch.inf
    t[t % 3 == 0] += 1
    loss, lse, out = check_cross_entropy(X, W, t, b, g)
    assert (out["dW"][::3] == 0).all() and (out["db"][::3] == 0).all()
    t[5] = 3
    loss, _ = cg.linear_cross_entropy(dev(X), dev(W), dev(t), dev(b))
    assert torch.isposinf(loss[5]) and torch.isfinite(loss[:5]).all() and torch.isfinite(loss[6:]).all()


def test_a_row_gone_wrong_stays_visible():
    X, W, t, b, g, _ = layer(70, 150, 32, "bf16", 10, False)
    t[t < 0] = 0
    X[9, 3] = float("nan")
    X[11, 0] = float("inf")
    loss, lse = cg.linear_cross_entropy(dev(X), dev(W), dev(t))
    bad = torch.zeros(70, dtype=torch.bool)
    bad[9] = bad[11] = True
    assert torch.equal(torch.isnan(loss).cpu(), bad) and torch.equal(torch.isfinite(lse).cpu(), ~bad)
    out = cg.linear_cross_entropy_backward(dev(g), dev(X), dev(W), dev(t), loss, lse)
    assert torch.equal(torch.isnan(out["dX"]).all(1).cpu(), bad) and torch.isnan(out["dW"]).all()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_large_and_small_gradients_of_the_loss(dt):
    """fp16's dz is brought near its top by a power of two: means over many rows and scaled losses alike."""
    for factor in (2.0 ** -30, 1e-6, 1.0, 2.0 ** 20):
        X, W, t, b, g, _ = layer(150, 900, 48, dt, 12, True)
        X, W = X / 64, W
        g *= factor
        if dt == "f16" and factor > 1:
            continue                                 # (the gradients themselves pass its range)
        check_cross_entropy(X, W, t, b, g)


def test_no_rows_and_no_features():
    W = torch.randn(50, 16, dtype=torch.bfloat16, device="cuda")
    X, t = W.new_empty(0, 16), torch.empty(0, dtype=torch.int32, device="cuda")
    loss, lse = cg.linear_cross_entropy(X, W, t)
    assert loss.shape == (0,) and lse.shape == (0,)
    out = cg.linear_cross_entropy_backward(loss, X, W, t, loss, lse, torch.zeros(50, device="cuda"))
    assert out["dX"].shape == (0, 16) and (out["dW"] == 0).all() and (out["db"] == 0).all()
    b = torch.randn(50)
    X, t = torch.empty(3, 0, dtype=torch.bfloat16), torch.tensor([4, -1, 49], dtype=torch.int32)
    check_cross_entropy(X, torch.empty(50, 0, dtype=torch.bfloat16), t, b, torch.ones(3))


def test_any_alignment():
    """X, W, dX and dW off the 4-byte grid."""
    X, W, t, b, g, _ = layer(77, 333, 45, "bf16", 13, True)
    bx, bw = (torch.zeros(v.numel() + 1, dtype=v.dtype, device="cuda") for v in (X, W))
    bx[1:], bw[1:] = X.flatten().cuda(), W.flatten().cuda()
    Xo, Wo = bx[1:].view(X.shape), bw[1:].view(W.shape)
    loss, lse = cg.linear_cross_entropy(Xo, Wo, dev(t), dev(b))
    ex.close("loss", loss, *ex.loss(X, W, *one_hot(t, 333), b)["loss"])
    ox, ow = torch.full_like(bx, 3.0), torch.full_like(bw, 3.0)
    out = cg.linear_cross_entropy_backward(dev(g), Xo, Wo, dev(t), loss, lse, dev(b),
                                           out={"dX": ox[1:].view(X.shape), "dW": ow[1:].view(W.shape)})
    want = ex.gradients(X, W, *one_hot(t, 333), g, b)
    for name in ("dX", "dW", "db"):
        ex.close(name, out[name], *want[name])
    assert ox[0] == 3 and ow[0] == 3


@pytest.mark.parametrize("x,w", [(1, 0), (0, 1), (2, 4), (1, 1)])
@pytest.mark.parametrize("n", [1, 5, 16])
def test_few_rows_at_any_alignment(n, x, w):
    """Up to 16 rows, X or W some elements off the grid, between NaN."""
    X, W, t, b, g, _ = layer(n, 333, 46, "f16", 30 + n, True)
    bx, bw = (torch.full((v.numel() + 8,), float("nan"), dtype=v.dtype, device="cuda") for v in (X, W))
    bx[x:x + X.numel()], bw[w:w + W.numel()] = X.flatten().cuda(), W.flatten().cuda()
    Xo, Wo = bx[x:x + X.numel()].view(X.shape), bw[w:w + W.numel()].view(W.shape)
    loss, lse = cg.linear_cross_entropy(Xo, Wo, dev(t), dev(b))
    f = ex.loss(X, W, *one_hot(t, 333), b)
    ex.close("loss", loss, *f["loss"])
    ex.close("lse", lse, *f["lse"])


def test_db_of_many_rows_alone():
    """More row tiles than one launch joins: db without the other gradients, with rows left out at the end."""
    X, W, t, b, g, _ = layer(40_000, 70, 24, "bf16", 15, True)
    t[-9000:] = -1
    d = [dev(v) for v in (X, W, t, b)]
    loss, lse = cg.linear_cross_entropy(*d)
    out = cg.linear_cross_entropy_backward(dev(g), d[0], d[1], d[2], loss, lse, d[3], out={"dX": None, "dW": None})
    ex.close("db", out["db"], *ex.gradients(X, W, *one_hot(t, 70), g, b)["db"])


def test_each_gradient_alone_and_the_same_bits_again():
    X, W, t, b, g, _ = layer(300, 2000, 136, "bf16", 14, True)
    d = [dev(v) for v in (X, W, t, b)]
    loss, lse = cg.linear_cross_entropy(*d)
    args = (dev(g), d[0], d[1], d[2], loss, lse, d[3])
    whole = cg.linear_cross_entropy_backward(*args)
    again = cg.linear_cross_entropy_backward(*args)
    for name in ("dX", "dW", "db"):
        assert torch.equal(whole[name], again[name])
        others = {o: None for o in ("dX", "dW", "db") if o != name}
        alone = cg.linear_cross_entropy_backward(*args, out=others)
        assert torch.equal(alone[name], whole[name]) and all(alone[o] is None for o in others)
    assert all(torch.equal(a, b) for a, b in zip((loss, lse), cg.linear_cross_entropy(*d)))
