"""Results of more than 2^32 work items' launches, to the last element."""
import pytest
import torch

import paper_2501_04266_amd as zq
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [600, 40])
def test_gradient_of_many_short_rows(T):
    """A wave a row: more than 2^26 rows.  Whole numbers, so sums are exact; T tokens with
    a row of more than 64 of them among the last rows."""
    V, D = 70_000_003, 1
    g = torch.Generator(device=DEV).manual_seed(T)
    ids = torch.randint(0, V, (T,), device=DEV, generator=g)
    ids[::5] = V - 1
    ids[1::5] = 3
    dy = torch.randint(-8, 9, (T, D), device=DEV, generator=g).float()
    got = zq.embedding_grad(ids, dy, V)
    want = torch.zeros(V, D, device=DEV).index_add_(0, ids, dy)
    assert torch.equal(got, want)
    zq.embedding_grad(ids, dy, V, out=got, accumulate=True)
    assert torch.equal(got, 2 * want)


def test_lookup_of_many_tokens():
    T, D = (1 << 32) // 7 + 100_003, 7
    table = torch.arange(1, 3 * D + 1, device=DEV).view(3, D).bfloat16()
    ids = torch.zeros(T, dtype=torch.int32, device=DEV)
    ids[1::2], ids[-1], ids[-2] = 1, 2, -1
    y = zq.embedding(ids, table)
    assert torch.equal(y[-2:], torch.stack([torch.zeros_like(table[0]), table[2]]))
    for r in (0, 1):
        assert bool((y[r:T - 2:2] == table[r]).all())
