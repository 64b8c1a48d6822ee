"""GPU test of the embedding lookup and its gradient on the longest list that the library takes."""
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
