"""Selection of pages whose scores are equal, or sums that float64 rounds."""

import pytest
import torch

import _decoding as ref
from paper_2603_06492_amd import decoding as nd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per,rows", [(40, 1), (600, 1), (600, 60), (3000, 1), (3000, 200)])
@pytest.mark.parametrize("D,dt", [(128, torch.float32), (64, torch.float32), (40, torch.float32), (128, torch.bfloat16), (72, torch.bfloat16)])
def test_equal_means_of_any_sums_rank_by_their_place(per, rows, D, dt):
    """Products of exponents so far apart that every sum is rounded, differently in every order: pages of equal means, far from
    each other, have equal scores all the same, in each of the kernels that form them, and the first of them are taken."""
    page, count = 8, 12
    g = torch.Generator(device="cuda").manual_seed(D + per)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda") * 2.0 ** torch.randint(-40, 40, s, generator=g, device="cuda")  # noqa: E731
    means = rand(per, 2, D).to(dt)
    table = torch.randperm(per, generator=g, device="cuda").to(torch.int32).repeat(rows, 1)
    q = rand(1, 4, D).to(dt).repeat(rows, 1, 1)   # two heads to a key head
    # the sum of the queries times 2^30 has the largest product with itself by far
    top = (q[0].view(2, 2, D).double().sum(1) * 2.0 ** 30).to(dt)
    equal = list(range(3, per - 1, 2))
    means[table[0, equal].long()] = top
    lengths = torch.full((rows,), per * page, dtype=torch.int32, device="cuda")
    got = nd.noble_block_select(q, means, table, lengths, count, page=page, sink=1, local=1)
    expect = [0, *equal[:count - 2], per - 1]
    assert bool((got == torch.tensor(expect, dtype=torch.int32, device="cuda")).all()), got[0].tolist()
    if rows == 1:
        assert ref.select(q.cpu(), means.cpu(), table[0].tolist(), per * page, 1, count, page, 1, 1)[0].tolist() == [expect] * 2
