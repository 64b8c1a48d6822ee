"""Grouped products of small whole numbers: every sum of them is exact in fp32, whatever its order, so that outputs
are compared with 64-bit sums by equality, and a row that was left out shows however many there are."""
import torch

from test_gpu_grouped import Problem


def digits(g, *shape, device="cpu"):
    return torch.randint(-1, 2, shape, generator=g, device=device, dtype=torch.int8)


class Whole(Problem):
    """A Problem of digits -1, 0 and 1; ELU's outputs are 1, 0 and -1/2, slopes 1, 1 and 1/2."""

    def __init__(self, sizes, k, m, dt="bf16", act="none", before=0, behind=0, seed=0):
        super().__init__(sizes, 1, 1, dt, act, bias=False, before=before, behind=behind)
        g = torch.Generator().manual_seed(seed + 31 * k + m)
        self.k, self.m = k, m
        self.X, self.W, self.dY = (digits(g, *s).to(self.dt) for s in ((self.n, k), (self.E, m, k), (self.n, m)))
        self.Xk = None
        y = digits(g, self.n, m).to(self.dt)
        self.Y = torch.where(y < 0, -0.5, y) if act == "elu" else y.relu() if act == "relu" else y
        # sums of halves up to so many are exact in fp32
        assert 2 * max(max(self.sizes, default=0), k, m) <= 2 ** 24

    def slopes(self, device):
        """dZ in 64 bits."""
        dY, Y = self.dY.to(device).double(), self.Y.to(device).double()
        if self.act == "relu":
            return torch.where(Y > 0, dY, 0.0)
        return torch.where(Y > 0, dY, dY * (Y + 1.0)) if self.act == "elu" else dY

    def sums(self, device="cpu", leave_out=None):
        """dX (rows of a group), dW and db in 64 bits; leave_out: without these rows."""
        d, X, W = self.slopes(device), self.X.to(device).double(), self.W.to(device).double()
        if leave_out is not None:
            d[leave_out] = 0.0
        dX = torch.zeros((self.n, self.k), dtype=torch.float64, device=device)
        dW = torch.zeros((self.E, self.m, self.k), dtype=torch.float64, device=device)
        db = torch.zeros((self.E, self.m), dtype=torch.float64, device=device)
        for g, a, b in self.spans():
            dX[a:b] = torch.mm(d[a:b], W[g])
            dW[g] = torch.mm(d[a:b].t().contiguous(), X[a:b])
            db[g] = d[a:b].sum(0)
        return {"dX": dX, "dW": dW, "db": db}

    def outputs(self, device="cpu"):
        X, W = self.X.to(device).double(), self.W.to(device).double()
        Y = torch.zeros((self.n, self.m), dtype=torch.float64, device=device)
        for g, a, b in self.spans():
            Y[a:b] = torch.mm(X[a:b], W[g].t().contiguous())
        return Y.relu() if self.act == "relu" else Y


def agree(got, want):
    """got is the exact sum, rounded once to got's type."""
    return torch.equal(got, want.float().to(got.dtype))


# (sizes, k, m): one and three groups over a thousand slices of rows; groups that fill the widest tiles, miss them by
# one, or have no rows, beside one over many slices
WIDE = [300, 0, 1, 255, 257, 33500, 0, 128, 129]
MANY = [([141671], 19, 19), ([70000, 1, 71670], 20, 20)] + [
    (WIDE, k, m) for k, m in ((40, 264), (264, 40), (130, 300), (520, 258), (33, 1000))]
