"""GPU tests of the embedding lookup and its gradient on the longest list and the largest table that the library
takes."""
import pytest
import torch

import paper_2103_00959_amd as cg

pytestmark = pytest.mark.gpu


def test_the_longest_list():
    """2^31 - 4097 places of 5 tokens, their rows 1 each: the sums are the tokens' numbers of places.  In fp32 they are
    exact up to 2^24, and past that each of up to 10 joins in a tree and the last rounding adds 2^-24 of the sum."""
    n, V = cg.MAX_NNZ, 5
    index = torch.arange(n, dtype=torch.int32, device="cuda").remainder_(V + 1)          # (5: a padded place)
    table = torch.arange(1, V + 1, dtype=torch.bfloat16, device="cuda")[:, None].contiguous()
    rows = cg.embedding(table, index)
    for at in (0, 2 ** 30, n - V - 1):
        part = index[at:at + V + 1].long()
        want = torch.where(part < V, part + 1, 0).to(torch.bfloat16)
        assert torch.equal(rows[at:at + V + 1, 0], want)
    rows.fill_(1.0)
    got = cg.embedding_backward(rows, index, V, out_dtype=torch.float32)[:, 0].double().cpu()
    want = torch.tensor([(n - v + V) // (V + 1) for v in range(V)], dtype=torch.float64)
    assert ((got - want).abs() <= 11 * 2.0 ** -24 * want).all()


@pytest.mark.parametrize("n", [100, 9000, 2 ** 23 + 1])
def test_the_largest_table(n):
    """2^31 - 2 rows of one value: tokens of 31 bits through each sort.  Small whole numbers, so every sum is exact."""
    V = 2 ** 31 - 2
    g = torch.Generator(device="cuda").manual_seed(n)
    index = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    index[1::3] = V - 1 - index[1::3] % 50                      # many places of few tokens, at the table's end
    index[::7] = torch.tensor([-1, V, 0], dtype=torch.int32, device="cuda")[torch.arange(len(index[::7]), device="cuda") % 3]
    dY = torch.randint(-2, 3, (n, 1), generator=g, device="cuda").half()
    inside = (index >= 0) & (index < V)
    token, at = index[inside].long().unique(return_inverse=True)
    sums = torch.zeros(len(token), dtype=torch.float64, device="cuda").index_add_(0, at, dY[inside, 0].double())
    out = torch.full((V, 1), 3.0, device="cuda")
    assert cg.embedding_backward(dY, index, V, out=out) is out
    assert torch.equal(out[token, 0].double(), sums) and int(out.count_nonzero()) == int(sums.count_nonzero())
    out.fill_(3.0)
    cg.embedding_backward(dY, index, V, out=out, accumulate=True)
    assert torch.equal(out[token, 0].double(), sums + 3) and int((out != 3.0).sum()) == int(sums.count_nonzero())
    rows = cg.embedding(out, index)
    want = torch.where(inside, out[index.clamp(0, V - 1).long(), 0], 0.0)
    assert torch.equal(rows[:, 0], want)
