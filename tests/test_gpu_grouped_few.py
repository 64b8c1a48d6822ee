"""GPU tests of the choice between the kernel for few rows and tiles, where the weights are large."""
import pytest
import torch

import paper_2103_00959_amd as cg
from grouped_exact import Whole, agree

pytestmark = pytest.mark.gpu


# (groups, rows of each, k, m): both sides of the choice, by the rows, the outputs and the groups
@pytest.mark.parametrize("E,rows,k,m", [(1, 128, 1024, 2048), (1, 256, 1024, 2048), (1, 64, 264, 7710), (1, 64, 264, 7711),
                                        (64, 4, 40, 4095), (64, 4, 40, 4096), (129, 3, 33, 2033), (1, 1, 72, 262143),
                                        (1, 1, 72, 262144), (3, 17, 48, 9000), (3, 17, 47, 9003)])
def test_either_kernel_at_wide_outputs(E, rows, k, m):
    p = Whole([rows] * E, k, m, act="relu", before=1, behind=2)
    rows = slice(1, p.n - 2)
    Y = torch.full((p.n, m), 7.0, dtype=torch.float32, device="cuda")
    cg.grouped_linear(p.X.cuda(), p.W.cuda(), p.offsets.cuda(), act="relu", out=Y)
    assert agree(Y[rows], p.outputs("cuda")[rows])
    assert (Y[0] == 7).all() and (Y[-2:] == 7).all()


def kernel_time(n, k, m):
    """Microseconds of the kernel, the median of 20 calls."""
    X, W = torch.ones((n, k), device="cuda").bfloat16(), torch.ones((1, m, k), device="cuda").bfloat16()
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out = torch.empty((n, m), dtype=torch.bfloat16, device="cuda")
    for _ in range(5):
        cg.grouped_linear(X, W, off, out=out)
    torch.cuda.synchronize()
    cg.trace_enable(64)
    for _ in range(20):
        cg.grouped_linear(X, W, off, out=out)
    torch.cuda.synchronize()
    times = sorted(1e3 * ms for _, ms in cg.trace_read())
    cg.trace_enable(0)
    return times[len(times) // 2]


@pytest.mark.parametrize("k,m", [(4096, 4096), (8192, 8192)])
def test_rows_that_fill_tiles_take_no_longer_than_one_more(k, m):
    """256 rows, which the kernel for few rows took with any weights: 121 and 453 us, where 257 took 56 and 105."""
    one_more = kernel_time(257, k, m)
    assert kernel_time(256, k, m) <= 1.5 * one_more + 5
