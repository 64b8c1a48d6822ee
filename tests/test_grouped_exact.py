"""The comparison of grouped sums with 64-bit ones (no GPU): it accepts them and rejects any slice of rows left out."""
import pytest
import torch

from grouped_exact import MANY, Whole, agree


@pytest.mark.parametrize("sizes,k,m", MANY)
@pytest.mark.parametrize("act", ["none", "relu", "elu"])
def test_a_slice_left_out_shows(sizes, k, m, act):
    p = Whole(sizes, k, m, act=act)
    want = p.sums()
    assert agree(want["dW"].float(), want["dW"]) and agree(want["db"].float(), want["db"])
    big = max(range(p.E), key=lambda g: sizes[g])
    lo = int(p.offsets[big])
    d, X = p.slopes("cpu")[lo:lo + sizes[big]].float(), p.X[lo:lo + sizes[big]].float()
    # slices as the kernels cut them have 16 rows and more, here 129 and more
    for per in (16, 129, 139):
        for a in range(0, sizes[big] - per, sizes[big] // 61):
            part, bias = d[a:a + per].t() @ X[a:a + per], d[a:a + per].sum(0)
            assert not agree((want["dW"][big] - part).float(), want["dW"][big])
            assert not agree((want["db"][big] - bias).float(), want["db"][big])
    short = p.sums(leave_out=slice(lo + sizes[big] // 2, lo + sizes[big] // 2 + 129))
    assert not agree(short["dW"].float(), want["dW"]) and not agree(short["db"].float(), want["db"])
    assert not agree(torch.zeros_like(want["dW"]).float(), want["dW"])
