"""GPU tests of the grouped products on values that an epilogue or a number format could lose.  No tolerances: an
output is compared bit for bit."""
import pytest
import torch

import paper_2103_00959_amd as cg
from grouped_exact import Whole, agree
from test_gpu_grouped import Problem

pytestmark = pytest.mark.gpu

NAN = float("nan")

# (group sizes, k, m): the kernel for few rows; tiles of 64 and 128 columns, loaded directly and through registers;
# rows of under 8 features; tiles of 256 x 256
FORWARDS = [([9, 0, 30], 64, 40), ([300, 0, 41], 64, 40), ([300, 0, 41], 72, 200), ([300, 0, 41], 45, 130),
            ([300, 0, 41], 5, 33), ([17000, 0, 16500], 64, 264)]


def same(a, b):
    """Equal bit for bit, any NaN like any other."""
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[~torch.isnan(a)], b[~torch.isnan(b)])


@pytest.mark.parametrize("act", ["none", "relu", "elu"])
@pytest.mark.parametrize("sizes,k,m", FORWARDS)
def test_nan_stays_under_an_activation(sizes, k, m, act):
    """A NaN feature makes its row of Y NaN, a NaN weight or bias its column of the group's rows; the others keep
    their bits."""
    for dt, out in (("bf16", torch.float32), ("f16", torch.float16)):
        p = Problem(sizes, k, m, dt, act)
        want = p.forward(out_dtype=out)
        last, r, c = p.E - 1, sizes[0] - 1, m // 2
        first = int(p.offsets[last])
        p.X[r, k - 1] = NAN
        want[r] = NAN
        p.W[last, c, 0] = NAN
        want[first:, c] = NAN
        p.bias[last, m - 1] = NAN
        want[first:, m - 1] = NAN
        assert same(p.forward(out_dtype=out), want)


@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
@pytest.mark.parametrize("sizes,k,m", FORWARDS)
def test_slope_of_nan(sizes, k, m, codes):
    """ReLU's slope is 0 where Y <= 0 and 1 elsewhere: a NaN of Y lets dY through, a NaN of dY stays where Y > 0 or
    is NaN, and goes where Y <= 0.  ELU's slope of NaN is NaN."""
    for dt in ("bf16", "f16"):
        p = Problem(sizes, k, m, dt, "relu", codes=codes)
        g, r = p.E - 1, int(p.offsets[p.E - 1]) + 7
        cols = torch.tensor([0, m // 2, m - 1])
        p.Y[r, cols] = 1.0
        want = p.backward(dw_dtype=torch.float32)
        p.Y[r, cols] = NAN
        got = p.backward(dw_dtype=torch.float32)
        for name in want:
            assert same(got[name], want[name]), name
        p.dY[r, cols] = NAN
        got = p.backward(dw_dtype=torch.float32)
        want["dX"][r] = NAN
        want["dW"][g, cols] = NAN
        want["db"][g, cols] = NAN
        for name in want:
            assert same(got[name], want[name]), name
        p.Y[r, cols] = 0.0
        gone = p.backward(dw_dtype=torch.float32)
        p.dY[r, cols] = 5.0
        for name, t in p.backward(dw_dtype=torch.float32).items():
            assert same(gone[name], t), name
        p.act = "elu"
        want = p.backward(dw_dtype=torch.float32)
        p.Y[r, cols] = NAN
        want["dX"][r] = NAN
        want["dW"][g, cols] = NAN
        want["db"][g, cols] = NAN
        for name, t in p.backward(dw_dtype=torch.float32).items():
            assert same(t, want[name]), name


# the smallest subnormals; the codes of a checkpoint have steps of 2^-24 (fp16) and 2^-126 (bf16) at least
TINY = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133}


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "elu"])
@pytest.mark.parametrize("sizes,k,m", FORWARDS)
def test_subnormal_gradients(sizes, k, m, act, dt):
    """dY of two subnormal steps, of which ELU's slope of 1/2 leaves one: dW and db are whole numbers of steps, dX and
    a narrow dW the same rounded once."""
    p = Whole(sizes, k, m, dt, act)
    p.dY = (2 * p.dY.double() * TINY[dt]).to(p.dt)
    for codes in (False, True):
        X = p.X.cuda()
        kept = dict(zip(("codes", "exps"), cg.act_checkpoint(X))) if codes else {"X": X}
        for dw in (torch.float32, p.dt):
            o = cg.grouped_linear_backward(p.dY.cuda(), p.W.cuda(), p.offsets.cuda(), **kept, act=act,
                                           Y=p.Y.cuda() if act != "none" else None, dw_dtype=dw)
            want = p.sums("cuda")
            assert want["dW"].abs().max() > 0 and (p.dY != 0).any()
            for name in o:
                assert agree(o[name], want[name]), (name, codes, dw)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("sizes,k,m", FORWARDS)
def test_subnormal_features(sizes, k, m, dt):
    """X of one subnormal step through the forward and dW; fp16 checkpoints hold it as it is."""
    p = Whole(sizes, k, m, dt)
    p.X = (p.X.double() * TINY[dt]).to(p.dt)
    for out in (torch.float32, p.dt):
        Y = cg.grouped_linear(p.X.cuda(), p.W.cuda(), p.offsets.cuda(), out_dtype=out)
        assert agree(Y, p.outputs("cuda"))
    want = p.sums("cuda")
    for codes in (False, True) if dt == "f16" else (False,):
        X = p.X.cuda()
        kept = dict(zip(("codes", "exps"), cg.act_checkpoint(X))) if codes else {"X": X}
        o = cg.grouped_linear_backward(p.dY.cuda(), p.W.cuda(), p.offsets.cuda(), **kept, dw_dtype=torch.float32)
        for name in o:
            assert agree(o[name], want[name]), (name, codes)
