"""GPU tests of the embedding lookup's gradient over tables and lists that the one launch for small ones does not take
(lists up to 8192 over at most 2048 tokens times chunks of columns), with the bounds of test_gpu_embedding."""
import pytest
import torch

import paper_2103_00959_amd as cg
from test_gpu_embedding import DT, check_gradient, gradient_ref, half, tiny, tokens

pytestmark = pytest.mark.gpu

PAIRS = [(a, b) for a in DT for b in DT]


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dt,out", PAIRS)
@pytest.mark.parametrize("k", [1, 3, 4, 5, 7, 8, 33, 300])
def test_longer_lists_over_small_tables(k, dt, out, add):
    """Tokens over many pieces (9000 places of 3 tokens: over 100 pieces of 16 to 64), single columns, a last vector
    moved back to the row's end, sums added to each type."""
    for i, (n, V, skew) in enumerate(((9000, 90, 2.0), (9000, 3, 1.5), (20_000, 1, 1.0))):
        check_gradient(n, V, k, dt, out, skew, add, 57 * k + i)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dt,out", PAIRS)
@pytest.mark.parametrize("k", [1, 4, 7, 12, 130, 1030])
def test_short_lists_over_larger_tables(k, dt, out, add):
    """Sorted by one workgroup: one place, a few, as many as it takes; a token that has half of them."""
    for i, (n, V, skew) in enumerate(((1, 5000, 1.0), (70, 2049, 1.0), (8192, 2600, 12.0))):
        check_gradient(n, V, k, dt, out, skew, add, 91 * k + i)


@pytest.mark.parametrize("n,V", [(200, 5000), (9000, 20), (9000, 5000)])
@pytest.mark.parametrize("dt,k", [("bf16", 33), ("f32", 7), ("f16", 64), ("f16", 3), ("f32", 2)])
def test_any_alignment(dt, k, n, V):
    """Gradients an element off the grid, between values that have to stay."""
    g = torch.Generator().manual_seed(n + k)
    dY = torch.randn((n, k), generator=g).to(DT[dt])
    index = tokens(n, V, g, 1.5)
    buf = torch.zeros(n * k + 1, dtype=DT[dt], device="cuda")
    buf[1:] = dY.flatten().cuda()
    base = torch.randn((V, k), generator=g).to(DT[dt])
    for add in (False, True):
        out = torch.full((V * k + 2,), 5.0, dtype=DT[dt], device="cuda")
        if add:
            out[1:-1] = base.flatten().cuda()
        cg.embedding_backward(buf[1:].view(n, k), index.cuda(), V, out=out[1:-1].view(V, k), accumulate=add)
        value, bound = gradient_ref(dY, index, V, 1.0, base if add else None)
        got = out[1:-1].view(V, k).double().cpu()
        assert (got - value).abs().le(bound + half(DT[dt]) * (value.abs() + bound) + tiny(DT[dt])).all()
        assert out[0] == 5 and out[-1] == 5


@pytest.mark.parametrize("n", [15, 9000])
def test_sums_in_the_order_of_the_batch(n):
    """15 rows of one token that only add up right in order (2^24 + 1 + 1 ... stays 2^24 in fp32, 1 + 1 + ... + 2^24 does
    not), in one piece of the sorted list, whatever stands around them."""
    V, k = 6000, 4
    big = torch.ones((n, k), device="cuda")
    index = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(15, device="cuda") * (n // 15)
    index[at] = 0                                              # (the first of the sorted list)
    for first, want in ((0, 2.0 ** 24), (14, 2.0 ** 24 + 14)):
        big[:] = 1.0
        big[at[first]] = 2.0 ** 24
        got = cg.embedding_backward(big, index, V)
        assert (got[0] == want).all() and not got[1:].any()
