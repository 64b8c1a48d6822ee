"""GPU tests of the grouped products and the 8-bit activation checkpoints against the formulas in 64 bits.

Tolerances.  Products of two 16-bit numbers are exact in fp32; a sum of t of them in fp32, in any
order, is off by at most t 2^-23 of the sum of their magnitudes (2^-23, not 2^-24: an addition of the
matrix cores may truncate).  A stored output is rounded once more, by half a step of its type (and half
of the smallest fp16 subnormal).  Checkpoints are exact by definition: powers of two."""
import numpy as np
import pytest
import torch

import paper_2103_00959_amd as cg

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STEP = 2.0 ** -23


# ------------------------------------------------------------ checkpoints

def checkpoint_ref(A):
    """Codes and exponent bytes of a CPU tensor from the definition, by frexp in 64 bits."""
    n, F = A.shape
    nb = -(-F // 32)
    lo, hi = (-24, 9) if A.dtype == torch.float16 else (-126, 121)
    x = np.zeros((n, nb * 32))
    x[:, :F] = A.double().numpy()
    x = x.reshape(n, nb, 32)
    bad = ~np.isfinite(x).all(-1)
    x[bad] = 0.0
    top = np.abs(x).max(-1)
    mant, e = np.frexp(top)                       # top = mant 2^e, mant in [0.5, 1)
    e = np.where(mant * 128 >= 127.5, e - 6, e - 7)
    e = np.where(top == 0, lo, np.clip(e, lo, hi))
    q = np.clip(np.rint(np.ldexp(x, -e[..., None])), -127, 127)
    b = np.where(bad, 255, e + 127)
    return q.reshape(n, nb * 32)[:, :F].astype(np.int8), b.astype(np.uint8)


def decode_ref(codes, exps):
    n, F = codes.shape
    s = np.where(exps == 255, np.nan, np.ldexp(1.0, exps.astype(np.int64) - 127))
    return codes.astype(np.float64) * np.repeat(s, 32, axis=1)[:, :F]


def awkward(n, F, dt, seed):
    """Activations with blocks of zeros, of the smallest and largest values, of ties and near 127.5 steps."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, F), generator=g) * torch.exp(2 * torch.randn((n, 1), generator=g))
    info = torch.finfo(DT[dt])
    kind = torch.randint(0, 12, (n, -(-F // 32)), generator=g).repeat_interleave(32, 1)[:, :F]
    x = torch.where(kind == 0, torch.zeros(()), x)
    x = torch.where(kind == 1, torch.sign(x) * info.smallest_normal * torch.rand((n, F), generator=g), x)
    x = torch.where(kind == 2, torch.sign(x) * info.max * (1 - torch.rand((n, F), generator=g) ** 8), x)
    x = torch.where(kind == 3, torch.round(x * 4) / 2 + 0.25, x)
    x = torch.where(kind == 4, torch.tensor([127.5, 0.5, 1.5, 2.5])[torch.randint(0, 4, (n, F), generator=g)], x)
    x = torch.where(kind == 5, -x.relu(), x)
    return x.to(DT[dt])


SHAPES = [(1, 1), (1, 8), (3, 31), (5, 32), (7, 33), (2, 1433), (64, 256), (300, 8), (1000, 47), (129, 300), (0, 16)]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,F", SHAPES)
def test_checkpoint_is_the_definition(n, F, dt):
    A = awkward(n, F, dt, 100 + n + F)
    codes, exps = cg.act_checkpoint(A.cuda())
    q, b = checkpoint_ref(A)
    assert codes.shape == (n, F) and exps.shape == (n, -(-F // 32))
    assert np.array_equal(exps.cpu().numpy(), b)
    assert np.array_equal(codes.cpu().numpy(), q)
    v = decode_ref(q, b)
    # back in the activations' own type: no rounding (bf16 and fp32 hold 7 bits, fp16 by its bounds)
    back = cg.act_restore(codes, exps, out_dtype=DT[dt])
    assert np.array_equal(back.double().cpu().numpy(), v)
    # within half a step, one step where the block saturates
    step = np.repeat(np.ldexp(1.0, b.astype(np.int64) - 127), 32, axis=1)[:, :F]
    off = np.abs(v - A.double().numpy())
    assert np.all(off <= np.where(np.abs(q) == 127, 1.0, 0.5) * step)


def test_checkpoint_at_any_alignment():
    """Rows that start off the 4-byte grid, in storage that goes on behind them."""
    for dt, F in (("bf16", 33), ("f16", 41), ("f32", 35)):
        A = awkward(50, F, dt, 7)
        d = A.cuda()[3:]
        q, b = checkpoint_ref(A[3:])
        buf = torch.full((47 * F + 7,), 77, dtype=torch.int8, device="cuda")
        codes = buf[3:3 + 47 * F].view(47, F)
        codes, exps = cg.act_checkpoint(d, codes=codes)
        assert np.array_equal(codes.cpu().numpy(), q) and np.array_equal(exps.cpu().numpy(), b)
        assert (buf[:3] == 77).all() and (buf[3 + 47 * F:] == 77).all()
        out = torch.full((47 * F + 2,), 5.0, dtype=DT[dt], device="cuda")
        cg.act_restore(codes, exps, out=out[1:1 + 47 * F].view(47, F))
        assert np.array_equal(out[1:-1].double().cpu().numpy(), decode_ref(q, b).ravel())
        assert out[0] == 5.0 and out[-1] == 5.0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_checkpoint_of_values_that_are_not_finite(dt):
    """A block with an infinity or NaN decodes to NaN; the blocks beside it are as ever."""
    A = torch.randn(6, 100, generator=torch.Generator().manual_seed(3)).to(DT[dt])
    A[1, 5], A[2, 40], A[4, 99], A[5, 0] = float("inf"), float("nan"), -float("inf"), float("nan")
    codes, exps = cg.act_checkpoint(A.cuda())
    q, b = checkpoint_ref(A)
    assert np.array_equal(codes.cpu().numpy(), q) and np.array_equal(exps.cpu().numpy(), b)
    for out in DT.values():
        back = cg.act_restore(codes, exps, out_dtype=out).double().cpu().numpy()
        assert np.array_equal(np.isnan(back), np.isnan(decode_ref(q, b)))


def test_restore_rounds_to_narrower_types():
    """fp32 activations restored in fp16: the decoded values rounded once (infinite past its range)."""
    A = awkward(200, 96, "f32", 5)
    codes, exps = cg.act_checkpoint(A.cuda())
    v = decode_ref(codes.cpu().numpy(), exps.cpu().numpy())
    got = cg.act_restore(codes, exps, out_dtype=torch.float16).cpu()
    assert torch.equal(got, torch.from_numpy(v).float().half())     # v is exact in fp32


# ---------------------------------------------------------- grouped products

def offsets_of(sizes, first=0):
    return torch.tensor([first] + [first + int(s) for s in np.cumsum(sizes)], dtype=torch.int32)


def act_ref(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "elu":
        return torch.where(v > 0, v, torch.expm1(v))
    return v


def slope_ref(y, act):
    if act == "relu":
        return (y > 0).double()
    if act == "elu":
        return torch.where(y > 0, 1.0, y + 1.0)
    return torch.ones_like(y)


def close(got, ref, bound, what):
    """|got - ref| <= bound + the rounding of got's type."""
    got, t = got.detach().cpu(), got.dtype
    u = torch.finfo(t).eps / 2
    tiny = 2.0 ** -25 if t == torch.float16 else 2.0 ** -134 if t == torch.bfloat16 else 2.0 ** -150
    room = bound + u * (ref.abs() + bound) + tiny
    worst = ((got.double() - ref).abs() / room).max().item() if ref.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst} of what its arithmetic allows"


class Problem:
    """Inputs on both sides for groups of the given sizes, `before` and `behind` rows of no group."""

    def __init__(self, sizes, k, m, dt="bf16", act="none", bias=True, before=0, behind=0, seed=0, codes=False):
        g = torch.Generator().manual_seed(seed + 31 * k + m)
        self.sizes, self.k, self.m, self.act, self.dt = list(sizes), k, m, act, DT[dt]
        self.E, self.n = len(self.sizes), before + sum(self.sizes) + behind
        r = lambda *s, scale=1.0: (torch.randn(s, generator=g) * scale)
        self.X = r(self.n, k).to(self.dt)
        self.W = r(self.E, m, k, scale=max(k, 1) ** -0.5).to(self.dt)
        self.bias = r(self.E, m) if bias else None
        self.dY = r(self.n, m).to(self.dt)
        self.Y = act_ref(r(self.n, m), act).to(self.dt)
        self.offsets = offsets_of(self.sizes, before)
        self.codes = self.exps = None
        if codes:
            q, b = checkpoint_ref(self.X)
            self.codes, self.exps = torch.from_numpy(q), torch.from_numpy(b)
            self.Xk = torch.from_numpy(decode_ref(q, b))
        else:
            self.Xk = self.X.double()

    def spans(self):
        o = self.offsets.tolist()
        return [(g, o[g], o[g + 1]) for g in range(self.E)]

    def dev(self, t):
        return None if t is None else t.cuda()

    def forward(self, **kw):
        return cg.grouped_linear(self.dev(self.X), self.dev(self.W), self.dev(self.offsets), self.dev(self.bias),
                                 self.act, **kw)

    def backward(self, **kw):
        kept = {"codes": self.dev(self.codes), "exps": self.dev(self.exps)} if self.codes is not None else {
            "X": self.dev(self.X)}
        return cg.grouped_linear_backward(self.dev(self.dY), self.dev(self.W), self.dev(self.offsets), **kept,
                                          Y=self.dev(self.Y) if self.act != "none" else None, act=self.act, **kw)

    def check_forward(self, Y):
        for g, a, b in self.spans():
            X, W = self.X[a:b].double(), self.W[g].double()
            v, mag = X @ W.t(), X.abs() @ W.abs().t()
            if self.bias is not None:
                v, mag = v + self.bias[g].double(), mag + self.bias[g].double().abs()
            # every activation moves by no more than its argument; expm1 is off by under 4 steps of itself
            bound = (self.k + 1) * STEP * mag + (4 * STEP * act_ref(v, "elu").abs() if self.act == "elu" else 0)
            close(Y[a:b], act_ref(v, self.act), bound, f"Y of group {g}")

    def check_backward(self, o):
        for g, a, b in self.spans():
            d = self.dY[a:b].double() * slope_ref(self.Y[a:b].double(), self.act)
            W, X = self.W[g].double(), self.Xk[a:b]
            # ELU: y + 1 and the product round in fp32, dZ to its type for the products
            z = 2 * STEP if self.act == "elu" else 0.0
            z16 = z + torch.finfo(self.dt).eps / 2 if self.act == "elu" else 0.0
            # 16-bit subnormals of dZ: half the smallest, absolute
            tiny = 2.0 ** -25 if self.act == "elu" and self.dt == torch.float16 else 0.0
            mag = d.abs() @ W.abs()
            if o.get("dX") is not None:
                close(o["dX"][a:b], d @ W, (self.m * STEP * 1.01 + z16) * mag + tiny * W.abs().sum(0), f"dX of group {g}")
            t = b - a
            if o.get("dW") is not None:
                mag = d.abs().t() @ X.abs()
                close(o["dW"][g], d.t() @ X, (t * STEP * 1.01 + z16) * mag + tiny * X.abs().sum(0), f"dW of group {g}")
            if o.get("db") is not None:
                close(o["db"][g], d.sum(0), (t * STEP + z) * d.abs().sum(0), f"db of group {g}")


GROUPS = {
    "one": [300],
    "single rows": [1, 1, 1, 1, 1],
    "with empty ones": [0, 130, 0, 0, 1, 127, 0, 64, 0],
    "tile edges": [128, 256, 127, 129, 1],
    "many": [(7 * i) % 5 for i in range(150)],
    "none": [0, 0, 0],
}
WIDTHS = [(1, 1), (7, 5), (8, 8), (16, 33), (33, 16), (64, 64), (65, 127), (128, 128), (130, 129), (300, 47),
          (47, 300), (602, 128), (256, 520)]


@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("k,m", WIDTHS)
def test_forward_sizes(k, m, groups):
    p = Problem(GROUPS[groups], k, m, "bf16", "relu")
    p.check_forward(p.forward())


@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("k,m", WIDTHS)
@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
def test_backward_sizes(k, m, groups, codes):
    p = Problem(GROUPS[groups], k, m, "bf16", codes=codes)
    p.check_backward(p.backward(dw_dtype=torch.float32))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("act", ["none", "relu", "elu"])
@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
def test_forward_types(dt, act, out):
    for k, m in ((96, 72), (45, 31)):
        for bias in (True, False):
            p = Problem([40, 0, 200, 3], k, m, dt, act, bias, seed=5)
            Y = p.forward(out_dtype=DT[out])
            assert Y.dtype == DT[out]
            p.check_forward(Y)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("act", ["none", "relu", "elu"])
@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
def test_backward_types(dt, act, codes):
    for k, m in ((96, 72), (45, 31), (130, 200)):
        p = Problem([40, 0, 200, 3], k, m, dt, act, codes=codes, seed=6)
        for dw in (None, torch.float32):
            o = p.backward(dw_dtype=dw)
            assert o["dW"].dtype == (dw or p.dt)
            p.check_backward(o)


@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
@pytest.mark.parametrize("k,m", [(24, 40), (100, 70), (136, 264), (33, 129)])
def test_backward_over_many_rows(k, m, codes):
    """Groups of several chunks (partial sums), of one and of none, beside each other."""
    p = Problem([6000, 0, 1, 1500, 1024, 1025, 0, 20000], k, m, "bf16", "relu", codes=codes)
    o = p.backward(dw_dtype=torch.float32)
    p.check_backward(o)
    again = p.backward(dw_dtype=torch.float32)
    for name in o:
        assert torch.equal(o[name], again[name]), f"{name} differs from run to run"


def test_single_tokens():
    """One row, a few rows among many groups, and the most groups there can be."""
    for sizes in ([1], [0] * 63 + [1], [1 if i % 9 == 0 else 0 for i in range(64)], [0] * 4095 + [2],
                  [i % 2 for i in range(4096)]):
        for k, m in ((512, 264), (33, 41)) if len(sizes) < 100 else ((24, 10),):
            p = Problem(sizes, k, m, "bf16", "none", bias=False, seed=2)
            p.check_forward(p.forward())
            p.check_backward(p.backward())


def test_rows_of_no_group_keep_their_place():
    p = Problem([50, 0, 90], 72, 40, "bf16", "relu", before=3, behind=140)
    Y = torch.full((p.n, p.m), 7.0, dtype=p.dt, device="cuda")
    dX = torch.full((p.n, p.k), 9.0, dtype=p.dt, device="cuda")
    p.check_forward(p.forward(out=Y))
    o = p.backward(out={"dX": dX}, dw_dtype=torch.float32)
    p.check_backward(o)
    assert o["dX"] is dX
    for t, v in ((Y, 7.0), (dX, 9.0)):
        assert (t[:3] == v).all() and (t[143:] == v).all()


def test_what_is_not_finite_stays_in_its_row_and_group():
    """NaN in one row: the row's outputs and its group's dW and db are NaN, nothing else is touched."""
    for codes in (False, True):
        p = Problem([70, 60, 0, 33], 45, 37, "bf16", codes=False)
        q = Problem([70, 60, 0, 33], 45, 37, "bf16", codes=False)
        q.X[75], q.dY[76] = float("nan"), float("inf")
        if codes:
            for t in (p, q):
                c, e = checkpoint_ref(t.X)
                t.codes, t.exps = torch.from_numpy(c), torch.from_numpy(e)
        a, b = p.forward(), q.forward()
        assert torch.isnan(b[75]).all()
        keep = torch.arange(p.n) != 75
        assert torch.equal(a[keep.cuda()], b[keep.cuda()])
        a, b = p.backward(), q.backward()
        keep = torch.arange(p.n) != 76
        assert torch.equal(a["dX"][keep.cuda()], b["dX"][keep.cuda()])
        assert not torch.isfinite(b["dX"][76]).any()
        assert torch.isnan(b["dW"][1]).all() and not torch.isfinite(b["db"][1]).any()
        for g in (0, 2, 3):
            assert torch.equal(a["dW"][g], b["dW"][g]) and torch.equal(a["db"][g], b["db"][g])


def test_save_writes_the_checkpoint():
    for dt, k, m in (("bf16", 96, 72), ("f16", 45, 300), ("bf16", 300, 47), ("f16", 33, 1), ("bf16", 128, 256)):
        p = Problem([200, 0, 77], k, m, dt, "relu")
        p.X = awkward(p.n, k, dt, 11)
        plain = p.forward()
        Y, codes, exps = p.forward(save=True)
        q, b = checkpoint_ref(p.X)
        assert np.array_equal(codes.cpu().numpy(), q) and np.array_equal(exps.cpu().numpy(), b)
        assert torch.equal(Y.view(torch.int16), plain.view(torch.int16))
        mine = torch.empty_like(codes), torch.empty_like(exps)
        got = p.forward(codes=mine[0], exps=mine[1])
        assert got[1] is mine[0] and torch.equal(mine[0], codes) and torch.equal(mine[1], exps)


def test_outputs_left_out():
    p = Problem([1500, 0, 2000], 40, 56, "bf16", "elu")
    whole = p.backward()
    for names in (("dX",), ("dW",), ("db",), ("dW", "db"), ("dX", "db")):
        o = p.backward(out={n: None for n in whole if n not in names})
        for n in whole:
            assert (o[n] is None) if n not in names else torch.equal(o[n], whole[n])
    d = [p.dev(t) for t in (p.dY, p.W, p.offsets, p.Y)]
    o = cg.grouped_linear_backward(d[0], d[1], d[2], Y=d[3], act="elu", out={"dW": None})
    assert torch.equal(o["dX"], whole["dX"]) and torch.equal(o["db"], whole["db"])


def test_one_group_is_the_dense_layer():
    """With one group the forward is linear()'s product (another order of the sums), and its gradients follow."""
    p = Problem([3000], 136, 88, "bf16", "elu", seed=9)
    Y = cg.linear(p.dev(p.X), p.dev(p.W)[0], p.dev(p.bias)[0], "elu")
    p.check_forward(Y)
    p.check_forward(p.forward())


def test_gradients_against_differences():
    """The loss sum(c * act(X W^T + b)) of the operator itself, moved along a direction: bf16 inputs, fp32
    outputs.  The loss is linear in W for act none, so a difference is exact up to the sums' roundings."""
    p = Problem([60, 0, 45], 40, 24, "bf16", "none", seed=3)
    c = p.dY.float().cuda()
    o = p.backward(dw_dtype=torch.float32)

    def loss(X, W, b):
        Y = cg.grouped_linear(X, W, p.dev(p.offsets), b, out_dtype=torch.float32)
        return (c.double() * Y.double()).sum().item()

    X, W, b = p.dev(p.X), p.dev(p.W), p.dev(p.bias)
    base = loss(X, W, b)
    g = torch.Generator().manual_seed(1)
    for name, t, grad in (("X", X, o["dX"]), ("W", W, o["dW"]), ("b", b, o["db"])):
        moved = (t.float() + torch.randn(t.shape, generator=g).cuda()).to(t.dtype)
        step = moved.double() - t.double()                       # what the move became in 16 bits
        args = {"X": X, "W": W, "b": b, name: moved}
        got = loss(args["X"], args["W"], args["b"]) - base
        want = (grad.double() * step).sum().item()
        # each output is off by (k + 1) 2^-23 of its magnitudes, twice; dX is rounded to bf16
        mag = (c.double().abs() @ torch.ones(p.m, 1, dtype=torch.float64, device="cuda")).sum().item()
        top = X.double().abs().max().item() * W.double().abs().sum(-1).max().item() + b.abs().max().item()
        allow = 4 * (p.k + 1) * STEP * mag * 4 * top + 2.0 ** -8 * (grad.double() * step).abs().sum().item()
        assert abs(got - want) <= allow, (name, got, want, allow)


def test_two_layers_forward_and_backward():
    """A run of them together: two typed layers with the first one's input and output kept in 8 bits, then the
    gradients from the checkpoints, against the same steps from the formulas on the kernels' own intermediates."""
    sizes, k, h, m = [700, 0, 1300, 41], 100, 72, 19
    one = Problem(sizes, k, h, "bf16", "relu", seed=21)
    two = Problem(sizes, h, m, "bf16", "none", seed=22)
    H, c1, e1 = one.forward(save=True)
    one.check_forward(H)
    two.X = H.cpu()
    Y, c2, e2 = two.forward(save=True)
    two.check_forward(Y)
    two.codes, two.exps = c2.cpu(), e2.cpu()
    two.Xk = torch.from_numpy(decode_ref(two.codes.numpy(), two.exps.numpy()))
    o2 = two.backward(dw_dtype=torch.float32)
    two.check_backward(o2)
    one.dY, one.Y = o2["dX"].cpu(), H.cpu()
    one.codes, one.exps = c1.cpu(), e1.cpu()
    one.Xk = torch.from_numpy(decode_ref(one.codes.numpy(), one.exps.numpy()))
    one.check_backward(one.backward(dw_dtype=torch.float32))


def test_captured_step_replays():
    """Forward with its checkpoint and backward captured into a graph: every replay, with eager work and new
    contents between, equals the eager call."""
    p = Problem([500, 0, 2500, 9], 96, 80, "bf16", seed=4)
    X, W, off, dY = (p.dev(t) for t in (p.X, p.W, p.offsets, p.dY))

    def step():
        Y, c, e = cg.grouped_linear(X, W, off, save=True)
        o = cg.grouped_linear_backward(dY, W, off, codes=c, exps=e, dw_dtype=torch.float32)
        return [Y, c, e, o["dX"], o["dW"], o["db"]]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        X.copy_(torch.randn(p.X.shape, generator=g).to(p.dt))
        dY.copy_(torch.randn(p.dY.shape, generator=g).to(p.dt))
        sizes = torch.randint(0, 750, (4,), generator=g).tolist()
        off.copy_(offsets_of(sizes))
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step()
        rows = sum(sizes)
        for i, (a, b) in enumerate(zip(got, want)):
            if i in (0, 3):
                a, b = a[:rows], b[:rows]
            elif i in (1, 2):
                a, b = a[:rows], b[:rows]
            assert torch.equal(a, b), (seed, i)


def test_calls_on_other_streams():
    """Two calls at once, each on a stream and with a workspace of its own."""
    ps = [Problem([3000, 0, 900], 72, 64, "bf16", seed=s) for s in (1, 2)]
    ins = [[p.dev(t) for t in (p.dY, p.W, p.offsets, p.X)] for p in ps]
    need = cg.grouped_linear_backward_workspace(ps[0].n, 3, 72, 64)
    work = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    got = []
    for (dY, W, off, X), w, s in zip(ins, work, streams):
        with torch.cuda.stream(s):
            got.append((cg.grouped_linear(X, W, off),
                        cg.grouped_linear_backward(dY, W, off, X=X, dw_dtype=torch.float32, workspace=w)))
    torch.cuda.synchronize()
    for p, (Y, o) in zip(ps, got):
        p.bias = None
        p.check_forward(Y)
        p.check_backward(o)


def test_offsets_past_the_ends_count_as_the_ends():
    p = Problem([100, 60], 40, 24, "bf16", bias=False)
    want, wanted = p.forward(), p.backward(dw_dtype=torch.float32)
    p.offsets = torch.tensor([-5, 100, 2 ** 31 - 1], dtype=torch.int32)
    got, o = p.forward(), p.backward(dw_dtype=torch.float32)
    assert torch.equal(want, got)
    for name in o:
        assert torch.equal(o[name], wanted[name])


def test_elements_past_32_bits():
    """More than 2^31 elements in X, dX and the codes: the last rows against the formulas."""
    n, k, m, tail = 2_200_000, 1024, 16, 300
    assert n * k > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randn((n, k), generator=g, device="cuda", dtype=torch.bfloat16)
    dY = torch.randn((n, m), generator=g, device="cuda", dtype=torch.bfloat16)
    W = (torch.randn((2, m, k), generator=g, device="cuda") * k ** -0.5).to(torch.bfloat16)
    off = torch.tensor([0, n - tail, n], dtype=torch.int32, device="cuda")
    Y, codes, exps = cg.grouped_linear(X, W, off, save=True)
    o = cg.grouped_linear_backward(dY, W, off, codes=codes, exps=exps, dw_dtype=torch.float32)
    p = Problem([tail], k, m, "bf16", bias=False)
    p.X, p.W, p.dY = X[-tail:].cpu(), W[1:].cpu(), dY[-tail:].cpu()
    q, b = checkpoint_ref(p.X)
    assert np.array_equal(codes[-tail:].cpu().numpy(), q) and np.array_equal(exps[-tail:].cpu().numpy(), b)
    p.Xk = torch.from_numpy(decode_ref(q, b))
    p.check_forward(Y[-tail:])
    p.check_backward({"dX": o["dX"][-tail:], "dW": o["dW"][1:], "db": o["db"][1:]})
    back = cg.act_restore(codes, exps, out_dtype=torch.bfloat16)
    assert torch.equal(back[-tail:].cpu().double(), p.Xk)


@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
@pytest.mark.parametrize("seed", range(4))
def test_groups_across_slices(seed, codes):
    """Uneven groups over several windows of 64, empty ones anywhere, rows of no group at both ends: groups that
    lie inside a slice of rows, reach over one border or over many."""
    g = torch.Generator().manual_seed(seed)
    E = (150, 64, 65, 9)[seed]
    sizes = (torch.rand(E, generator=g) ** 6 * 2500).int()
    sizes[torch.rand(E, generator=g) < 0.3] = 0
    sizes[-1 if seed % 2 else 0] = 0
    k, m = ((24, 40), (33, 17), (130, 72), (264, 300))[seed]
    p = Problem(sizes.tolist(), k, m, ("bf16", "f16")[seed % 2], ("relu", "none")[seed % 2], before=7 * seed,
                behind=300 * seed, codes=codes, seed=seed)
    p.check_forward(p.forward())
    o = p.backward(dw_dtype=torch.float32)
    p.check_backward(o)
    again = p.backward(dw_dtype=torch.float32)
    rows = slice(int(p.offsets[0]), int(p.offsets[-1]))
    assert torch.equal(o["dX"][rows], again["dX"][rows])
    assert torch.equal(o["dW"], again["dW"]) and torch.equal(o["db"], again["db"])


@pytest.mark.parametrize("act", ["none", "relu", "elu"])
@pytest.mark.parametrize("k,m", [(3, 2), (2, 5), (7, 64), (6, 200), (64, 7), (300, 3), (5, 6)])
def test_narrow_rows(k, m, act):
    """Rows of under 8 elements in either operand, through both forms of the input."""
    for codes in (False, True):
        for dt in ("bf16", "f16"):
            p = Problem([700, 0, 90, 1], k, m, dt, act, codes=codes, seed=k)
            p.check_forward(p.forward())
            p.check_backward(p.backward(dw_dtype=torch.float32))


@pytest.mark.parametrize("shift", [1, 2, 4])
@pytest.mark.parametrize("k,m", [(64, 72), (130, 300), (47, 33), (256, 264)])
def test_operands_at_any_alignment(k, m, shift):
    """Operands that start off the 16-byte, the 4-byte grid, with other values around them."""
    def off(t):
        buf = torch.full((t.numel() + 16,), float("nan"), dtype=t.dtype, device="cuda") if t.is_floating_point() else \
            torch.full((t.numel() + 16,), 99, dtype=t.dtype, device="cuda")
        v = buf[shift:shift + t.numel()].view(t.shape)
        v.copy_(t)
        return v

    for codes in (False, True):
        p = Problem([400, 3, 0, 300], k, m, "bf16", "none", codes=codes)
        p.dev = lambda t: None if t is None else off(t) if t.dtype in (torch.bfloat16, torch.int8, torch.uint8) else t.cuda()
        p.check_forward(p.forward())
        p.check_backward(p.backward(dw_dtype=torch.float32))


def test_no_rows_at_all():
    W = torch.randn(3, 40, 24, device="cuda").bfloat16()
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    X, dY = W.new_empty((0, 24)), W.new_empty((0, 40))
    Y, codes, exps = cg.grouped_linear(X, W, off, save=True)
    assert Y.shape == (0, 40) and codes.shape == (0, 24) and exps.shape == (0, 1)
    o = cg.grouped_linear_backward(dY, W, off, X=X, out={"dW": torch.full_like(W, 3.0)})
    assert o["dX"].shape == (0, 24) and (o["dW"] == 0).all() and (o["db"] == 0).all()
    # rows, but none of a group: the gradients are zero too
    X, dY = torch.randn(500, 24, device="cuda").bfloat16(), torch.randn(500, 40, device="cuda").bfloat16()
    o = cg.grouped_linear_backward(dY, W, off, X=X, out={"dW": torch.full_like(W, 3.0), "dX": torch.full_like(X, 2.0)})
    assert (o["dW"] == 0).all() and (o["db"] == 0).all() and (o["dX"] == 2.0).all()


def test_no_features_or_no_outputs():
    """k = 0: the activation of the bias, and db; m = 0: a gradient of zeros."""
    off = offsets_of([3, 0, 5]).cuda()
    bias = torch.randn(3, 20, device="cuda")
    Y = cg.grouped_linear(torch.empty(8, 0, dtype=torch.bfloat16, device="cuda"),
                          torch.empty(3, 20, 0, dtype=torch.bfloat16, device="cuda"), off, bias, "relu", out_dtype=torch.float32)
    assert torch.equal(Y, bias[[0, 0, 0, 2, 2, 2, 2, 2]].relu())
    dY = torch.randn(8, 20, device="cuda").bfloat16()
    o = cg.grouped_linear_backward(dY, torch.empty(3, 20, 0, dtype=torch.bfloat16, device="cuda"), off,
                                   X=torch.empty(8, 0, dtype=torch.bfloat16, device="cuda"))
    d = dY.cpu().double()
    for g, (a, b) in enumerate(((0, 3), (3, 3), (3, 8))):
        close(o["db"][g], d[a:b].sum(0), (b - a) * STEP * d[a:b].abs().sum(0), f"db of group {g}")
    o = cg.grouped_linear_backward(dY[:, :0].contiguous(), torch.empty(3, 0, 16, dtype=torch.bfloat16, device="cuda"), off,
                                   X=torch.empty(8, 16, dtype=torch.bfloat16, device="cuda"))
    assert (o["dX"] == 0).all()


def test_two_captured_graphs_with_workspaces_of_their_own():
    """Two captured backward passes replayed one after another and interleaved, eager work between."""
    ps = [Problem([4000, 0, 2500], 72, 64, "bf16", seed=s, codes=True) for s in (5, 6)]
    ins = [[p.dev(t) for t in (p.dY, p.W, p.offsets, p.codes, p.exps)] for p in ps]

    def call(i):
        dY, W, off, c, e = ins[i]
        return cg.grouped_linear_backward(dY, W, off, codes=c, exps=e, dw_dtype=torch.float32)

    wanted = [call(0), call(1)]
    torch.cuda.synchronize()
    graphs, held = [], []
    for i in (0, 1):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            held.append(call(i))
    for order in ((0, 1), (1, 0), (0, 0, 1), (1, 1, 0)):
        for i in order:
            graphs[i].replay()
        call(0)
        torch.cuda.synchronize()
        for i in (0, 1):
            for name in wanted[i]:
                assert torch.equal(held[i][name], wanted[i][name]), (order, i, name)


@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
def test_the_widest_rows(codes):
    """2^22 features: byte offsets inside a tile reach 2^31.  Whole numbers, so that every sum is exact."""
    n, k, m = 300, 2 ** 22, 136
    g = torch.Generator(device="cuda").manual_seed(2)

    def digits(*s):
        return torch.randint(-1, 2, s, generator=g, device="cuda", dtype=torch.int8).to(torch.bfloat16)

    X, W, off = digits(n, k), digits(1, m, k), offsets_of([n]).cuda()
    kept = {"X": X}
    if codes:
        Y, c, e = cg.grouped_linear(X, W, off, out_dtype=torch.float32, save=True)
        kept = {"codes": c, "exps": e}
    else:
        Y = cg.grouped_linear(X, W, off, out_dtype=torch.float32)
    ref = torch.zeros(n, m, device="cuda")
    for a in range(0, k, 2 ** 18):
        ref += X[:, a:a + 2 ** 18].float() @ W[0, :, a:a + 2 ** 18].float().t()
    assert torch.equal(Y, ref)
    dY = digits(n, m)
    o = cg.grouped_linear_backward(dY, W, off, **kept, dw_dtype=torch.float32)
    for a in range(0, k, 2 ** 18):
        assert torch.equal(o["dX"][:, a:a + 2 ** 18].float(), dY.float() @ W[0, :, a:a + 2 ** 18].float())
        assert torch.equal(o["dW"][0, :, a:a + 2 ** 18], dY.float().t() @ X[:, a:a + 2 ** 18].float())
    # and as outputs: 2^22 of them a row
    V = W.view(1, k, m)
    Z = cg.grouped_linear(dY, V, off)
    for a in range(0, k, 2 ** 18):
        assert torch.equal(Z[:, a:a + 2 ** 18].float(), dY.float() @ V[0, a:a + 2 ** 18].float().t())
    o = cg.grouped_linear_backward(X, V, off, X=dY, dw_dtype=torch.float32)
    ref = torch.zeros(n, m, device="cuda")
    for a in range(0, k, 2 ** 18):
        ref += X[:, a:a + 2 ** 18].float() @ V[0, a:a + 2 ** 18].float()
        assert torch.equal(o["dW"][0, a:a + 2 ** 18], X[:, a:a + 2 ** 18].float().t() @ dY.float())
    assert torch.equal(o["dX"].float(), ref.to(torch.bfloat16).float())
    assert torch.equal(o["db"][0], X.float().sum(0))


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("k,m", [(64, 72), (130, 300), (47, 33), (260, 4), (4, 264)])
def test_outputs_at_any_alignment(k, m, shift):
    """Outputs off the 16-byte grid, in storage that holds other values before and behind them."""
    p = Problem([400, 3, 0, 300, 5000], k, m, "bf16", "none")
    held = {}

    def off(name, shape, dt):
        size = int(np.prod(shape))
        buf = held[name] = torch.full((size + 8,), 77.0, dtype=dt, device="cuda")
        return buf[shift:shift + size].view(shape)

    for y in ("bf16", "f16", "f32"):
        out = off("Y", (p.n, m), DT[y])
        p.check_forward(p.forward(out=out))
        few = Problem([20, 0, 1], k, m, "bf16", "none")
        few.check_forward(few.forward(out=off("few", (few.n, m), DT[y])))
        for name in ("Y", "few"):
            assert (held[name][:shift] == 77).all() and (held[name][shift - 8:] == 77).all()
    for dt in (torch.bfloat16, torch.float32):
        o = {"dX": off("dX", (p.n, k), torch.bfloat16), "dW": off("dW", (p.E, m, k), dt),
             "db": off("db", (p.E, m), torch.float32)}
        p.check_backward(p.backward(out=o))
        for name in o:
            assert (held[name][:shift] == 77).all() and (held[name][shift - 8:] == 77).all()


@pytest.mark.parametrize("act", ["none", "relu", "elu"])
@pytest.mark.parametrize("k,m", [(40, 264), (264, 40), (130, 300), (520, 258), (33, 1000)])
def test_many_rows_of_wide_outputs(k, m, act):
    """Enough rows for the widest tiles, in groups that fill them, miss them by one, or have none."""
    sizes = [300, 0, 1, 255, 257, 33500, 0, 128, 129]
    for dt in ("bf16", "f16"):
        p = Problem(sizes, k, m, dt, act, before=3, behind=5)
        p.check_forward(p.forward())
        o = p.backward(dw_dtype=torch.float32)
        p.check_backward(o)
        again = p.backward(dw_dtype=torch.float32)
        rows = slice(3, 3 + sum(sizes))
        assert torch.equal(o["dX"][rows], again["dX"][rows]) and torch.equal(o["dW"], again["dW"])


@pytest.mark.parametrize("E,rows", [(1, 255), (1, 256), (1, 257), (30, 8), (30, 9), (3, 20000)])
def test_borders_of_the_kernels_for_few_and_many_rows(E, rows):
    for k, m in ((64, 520), (520, 64), (7, 300), (8, 300)):
        p = Problem([rows] * E, k, m, "bf16", "none")
        p.check_forward(p.forward(out_dtype=torch.float32))
        p.check_backward(p.backward())


@pytest.mark.parametrize("n,E,k,m", [(46, 253, 104, 28), (40, 47, 664, 888), (1, 5, 144, 280), (9, 4096, 8, 8),
                                     (5000, 4096, 24, 16), (141671, 1, 19, 19), (141671, 3, 20, 20)])
def test_slices_of_few_rows_and_of_many(n, E, k, m):
    """More groups than rows, so that most have none; and sums over a thousand slices."""
    g = torch.Generator().manual_seed(n)
    sizes = torch.bincount(torch.randint(0, E, (n,), generator=g) ** 2 // E, minlength=E)
    for codes in (False, True):
        p = Problem(sizes.tolist(), k, m, "bf16", "none", codes=codes)
        dW = torch.full((E, m, k), float("nan"), device="cuda")
        o = p.backward(out={"dW": dW})
        p.check_backward(o)
        assert torch.equal(o["dW"], p.backward(dw_dtype=torch.float32)["dW"])
