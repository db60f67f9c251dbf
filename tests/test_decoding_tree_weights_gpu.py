"""Drafts in a cache that keeps attention weights: what a tree's step, its acceptance and the steps after it do to them."""

import pytest
import torch

from paper_2603_06492_amd.attention import NobleSelfAttention, PagedCache

pytestmark = pytest.mark.gpu


def test_weights_of_drafted_tokens():
    """A tree's step adds nothing to any token; accepted tokens begin with nothing, and receive from the next step on."""
    block = NobleSelfAttention(128, 4, 16, kv_heads=2, longest=256)
    rows = lambda n, seed: torch.randn(n, 128, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()  # noqa: E731
    c = PagedCache(2, 64, 20, kv_heads=2, head_dim=32, page=8, weights=True)
    block.step(rows(2 * 19, 1), c, *c.extend(19))
    before = c.weights[0].clone()
    torch.testing.assert_close(before.sum(2), torch.full((2, 2), 19.0 * 2, device="cuda"), rtol=1e-4, atol=0)
    parents = torch.tensor([[-1, 0, 0, 1], [-1, -1, 1, -2]], device="cuda", dtype=torch.int32)
    positions, slots, tree = c.draft(parents)
    c.weights[0][:, :, 19:] = 7.0   # whatever an earlier draft's place holds
    block.step(rows(8, 2), c, positions, slots, tree=tree)
    assert bool((c.weights[0][:, :, :19] == before[:, :, :19]).all())
    parents.fill_(-1)               # acceptance goes by the tree as it was drafted
    with pytest.raises(ValueError, match="branch"):
        c.accept([[0, 3], []])
    c.accept([[0, 1, 3], [1]])
    w = c.weights[0]
    assert bool((w[:, :, :19] == before[:, :, :19]).all())
    assert bool((w[0, :, 19:22] == 0).all()) and bool((w[1, :, 19:20] == 0).all())
    block.step(rows(2, 3), c, *c.extend(1))
    for b, held in enumerate((23, 21)):
        added = (w[b, :, :held] - torch.nn.functional.pad(before[b, :, :19], (0, held - 19)))
        assert bool((added > 0).all())
        # one row of two heads to a key head: their probabilities; the sums before are rounded to 2^-24 of about 1 per token
        torch.testing.assert_close(added.sum(1), torch.full((2,), 2.0, device="cuda"), rtol=1e-4, atol=0)
