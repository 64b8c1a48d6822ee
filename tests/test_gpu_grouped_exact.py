"""GPU tests of the grouped products where sums run over many rows: whole numbers, compared by equality."""
import pytest
import torch

import paper_2103_00959_amd as cg
from grouped_exact import MANY, Whole, agree, digits

pytestmark = pytest.mark.gpu


def kept_of(p, codes):
    X = p.X.cuda()
    if not codes:
        return {"X": X}
    c, e = cg.act_checkpoint(X)
    return {"codes": c, "exps": e}          # (digits come back as they were)


def check(p, codes):
    rows = slice(int(p.offsets[0]), int(p.offsets[-1]))
    if p.act != "elu":
        Y = cg.grouped_linear(p.X.cuda(), p.W.cuda(), p.offsets.cuda(), act=p.act, out_dtype=torch.float32)
        assert agree(Y[rows], p.outputs("cuda")[rows])
    want = p.sums("cuda")
    for dw in (torch.float32, p.dt):
        o = cg.grouped_linear_backward(p.dY.cuda(), p.W.cuda(), p.offsets.cuda(), **kept_of(p, codes), act=p.act,
                                       Y=p.Y.cuda() if p.act != "none" else None, dw_dtype=dw)
        assert agree(o["dX"][rows], want["dX"][rows]), "dX"
        assert o["dW"].dtype == dw and agree(o["dW"], want["dW"]), "dW"
        assert agree(o["db"], want["db"]), "db"


@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
@pytest.mark.parametrize("act", ["none", "relu", "elu"])
@pytest.mark.parametrize("sizes,k,m", MANY)
def test_every_row_counts(sizes, k, m, act, codes):
    for dt in ("bf16", "f16"):
        check(Whole(sizes, k, m, dt, act, before=3, behind=5), codes)


@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
@pytest.mark.parametrize("E,rows,k,m", [(1, 1, 64, 64), (64, 40, 136, 72), (150, 90, 33, 48), (9, 2500, 260, 4),
                                        (3, 20000, 8, 7), (3, 20000, 3, 130), (2, 40000, 256, 256)])
def test_every_row_counts_in_uneven_groups(E, rows, k, m, codes):
    """Groups of 0 to twice the mean, whose borders lie anywhere in the slices."""
    g = torch.Generator().manual_seed(E)
    sizes = torch.randint(0, 2 * rows + 1, (E,), generator=g).tolist()
    for act in ("none", "relu", "elu"):
        check(Whole(sizes, k, m, "bf16", act), codes)


@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
def test_every_row_counts_past_32_bits(codes):
    """More than 2^31 elements in X, dX and the codes: all rows of both groups."""
    n, k, m, tail, part = 2_200_000, 1024, 16, 300, 100_000
    assert n * k > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(3)
    X = torch.empty((n, k), dtype=torch.bfloat16, device="cuda")
    for a in range(0, n, part):
        X[a:a + part] = digits(g, part, k, device="cuda")
    dY = digits(g, n, m, device="cuda").to(torch.bfloat16)
    W = digits(g, 2, m, k, device="cuda").to(torch.bfloat16)
    off = torch.tensor([0, n - tail, n], dtype=torch.int32, device="cuda")
    kept = {"X": X}
    if codes:
        Y, c, e = cg.grouped_linear(X, W, off, out_dtype=torch.float32, save=True)
        kept = {"codes": c, "exps": e}
    else:
        Y = cg.grouped_linear(X, W, off, out_dtype=torch.float32)
    o = cg.grouped_linear_backward(dY, W, off, **kept, dw_dtype=torch.float32)
    dW = torch.zeros((2, m, k), dtype=torch.float64, device="cuda")
    db = torch.zeros((2, m), dtype=torch.float64, device="cuda")
    cuts = list(range(0, n - tail, part)) + [n - tail, n]
    for a, b in zip(cuts, cuts[1:]):
        t = int(a == n - tail)
        x, d, w = X[a:b].double(), dY[a:b].double(), W[t].double()
        assert agree(Y[a:b], torch.mm(x, w.t().contiguous())), (a, b)
        assert agree(o["dX"][a:b], torch.mm(d, w)), (a, b)
        dW[t] += torch.mm(d.t().contiguous(), x)
        db[t] += d.sum(0)
    assert agree(o["dW"], dW) and agree(o["db"], db)
    if codes:
        for a in range(0, n, part):
            assert torch.equal(cg.act_restore(c[a:a + part], e[a:a + part], out_dtype=torch.bfloat16), X[a:a + part])
