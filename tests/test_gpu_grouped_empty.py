"""GPU tests of the gradients of groups without rows: zeros wherever they lie, in a time that does not depend on it."""
import pytest
import torch

import paper_2103_00959_amd as cg
from grouped_exact import Whole, agree

pytestmark = pytest.mark.gpu


def places(E, live, rows):
    """`rows` rows in each of `live` groups of E: the first ones, the last ones, and spread out."""
    every = E // live
    return {"first": [rows] * live + [0] * (E - live), "last": [0] * (E - live) + [rows] * live,
            "spread": [rows if g % every == 0 and g // every < live else 0 for g in range(E)]}


# (groups, those with rows, rows of each, k, m): single tokens, one row, many groups, wide tiles, matrices of several
# pieces and of an odd size, slices with and without partial sums, no group with rows
CASES = [(64, 8, 1, 512, 264), (253, 1, 46, 104, 28), (4096, 2, 100, 24, 8), (33, 1, 1, 1024, 264), (9, 3, 3000, 264, 130),
         (70, 5, 500, 131, 129), (130, 130, 1, 40, 7), (66, 1, 0, 200, 90)]


@pytest.mark.parametrize("place", ["first", "last", "spread"])
@pytest.mark.parametrize("codes", [False, True], ids=["input", "8bit"])
@pytest.mark.parametrize("E,live,rows,k,m", CASES)
def test_zeros_wherever_groups_have_no_rows(E, live, rows, k, m, codes, place):
    p = Whole(places(E, live, rows)[place], k, m, act="relu", before=2, behind=3)
    want = p.sums("cuda")
    X = p.X.cuda()
    kept = dict(zip(("codes", "exps"), cg.act_checkpoint(X))) if codes else {"X": X}
    for dw in (torch.float32, p.dt):
        # off the 16-byte grid, with other values around
        held = [torch.full((E * s + 9,), 77.0, dtype=t, device="cuda") for s, t in ((m * k, dw), (m, torch.float32))]
        dW, db = held[0][3:-6].view(E, m, k), held[1][1:-8].view(E, m)
        for out in ({"dW": dW, "db": db}, {"dW": dW, "db": None}, {"dW": None, "db": db}):
            dW.fill_(float("nan"))
            db.fill_(float("nan"))
            cg.grouped_linear_backward(p.dY.cuda(), p.W.cuda(), p.offsets.cuda(), **kept, act="relu", Y=p.Y.cuda(),
                                       out=dict(out, dX=None))
            for name, t in (("dW", dW), ("db", db)):
                assert agree(t, want[name]) if out[name] is not None else torch.isnan(t).all(), (name, dw)
            for t, a, b in ((held[0], 3, -6), (held[1], 1, -8)):
                assert (t[:a] == 77).all() and (t[b:] == 77).all()


def test_replays_with_other_groups_empty():
    """A captured backward pass replayed while the groups with rows move."""
    E, k, m = 70, 72, 40
    sets = [Whole(s, k, m, seed=i) for i, s in enumerate(places(E, 7, 100).values())]
    X, W, dY, off = (t.cuda() for t in (sets[0].X, sets[0].W, sets[0].dY, sets[0].offsets))

    def call():
        return cg.grouped_linear_backward(dY, W, off, X=X, dw_dtype=torch.float32)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for p in sets + sets:
        for t, s in ((X, p.X), (W, p.W), (dY, p.dY), (off, p.offsets)):
            t.copy_(s)
        graph.replay()
        got = {name: t.clone() for name, t in held.items()}
        eager, want = call(), p.sums("cuda")
        torch.cuda.synchronize()
        for name in want:
            assert agree(got[name], want[name]) and torch.equal(got[name], eager[name]), name


def kernel_time(sizes, k, m):
    """Microseconds of the kernel of dW, the median of 20 calls."""
    p = Whole(sizes, k, m)
    X, W, dY, off = (t.cuda() for t in (p.X, p.W, p.dY, p.offsets))
    out = {"dX": None, "dW": torch.empty((p.E, m, k), device="cuda")}
    for _ in range(5):
        cg.grouped_linear_backward(dY, W, off, X=X, out=out)
    torch.cuda.synchronize()
    cg.trace_enable(256)
    for _ in range(20):
        cg.grouped_linear_backward(dY, W, off, X=X, out=out)
    torch.cuda.synchronize()
    times = sorted(1e3 * ms for name, ms in cg.trace_read() if name == "grouped_linear_dw")
    cg.trace_enable(0)
    return times[len(times) // 2]


@pytest.mark.parametrize("E,live,rows,k,m", [(64, 8, 1, 1024, 1024), (256, 2, 23, 104, 28), (4096, 2, 100, 24, 16)])
def test_groups_without_rows_do_not_queue(E, live, rows, k, m):
    """Runs of empty groups take no more time than as many groups of one row (while one workgroup zeroed a run, one
    group after another, several times as much)."""
    most = 1.5 * kernel_time([1] * E, k, m) + 10
    for place, sizes in places(E, live, rows).items():
        t = kernel_time(sizes, k, m)
        assert t <= most, (place, t, most)
