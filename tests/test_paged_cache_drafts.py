"""Drafts in PagedCache: which lists of nodes may be accepted, on the CPU, with the kernels' calls replaced by their names."""

import pytest
import torch

from paper_2603_06492_amd import decoding as nd
from paper_2603_06492_amd.attention import PagedCache


@pytest.fixture
def calls(monkeypatch):
    made = []

    def tree_rows(parents, lengths):
        made.append("tree_rows")
        n = parents.shape[1]
        return torch.zeros(*parents.shape, (n + 31) // 32), torch.zeros(parents.shape), torch.zeros(parents.shape, dtype=torch.int32)

    monkeypatch.setattr(nd, "noble_tree_rows", tree_rows)
    monkeypatch.setattr(nd, "noble_cache_keep", lambda *a: made.append("keep"))
    monkeypatch.setattr(nd, "noble_page_means", lambda *a: made.append("means"))
    return made


def _cache(**kw):
    c = PagedCache(2, 64, 20, kv_heads=1, head_dim=8, page=8, device="cpu", means=True, weights=True, **kw)
    c.extend(9)
    return c


def _state(c):
    return (c.lengths.tolist(), c.page_table.tolist(), list(c._held), list(c._seen), [list(t) for t in c._table], list(c._free),
            c._drafted)


PARENTS = [[-1, 0, 0, 1, -1, 4, -2], [-1, -1, 1, 2, 9, 4, 3]]


@pytest.mark.parametrize("first,what", [
    ([0, 4], "two roots"), ([1, 3], "not from the root"), ([0, 3], "a parent left out"), ([1], "no root"), ([6], "no node"),
    ([0, 1, 2], "a sibling"), ([0, 6], "no node below one"), ([4, 5, 6], "no node at the end")], ids=str)
def test_what_is_no_branch_is_refused(calls, first, what):
    """Such nodes' keys were rotated for other places than they would be moved to."""
    c = _cache()
    c.draft(torch.tensor(PARENTS))
    before, n = _state(c), len(calls)
    for kept in ([first, []], [[0], [4]], [[], [5]], [[0, 2], [1, 2, 6]]):   # in the second tree, 4 and 5 are no nodes
        with pytest.raises(ValueError, match="branch"):
            c.accept(kept)
        assert _state(c) == before and len(calls) == n   # nothing has changed, another list may follow
    c.accept([[0, 1, 3], [1, 2, 3, 6]])
    assert c._held == c._seen == [12, 13] and not c._drafted


@pytest.mark.parametrize("kept", [[[], []], [[0], [0]], [[4, 5], [1]], [[0, 2], [1, 2, 3, 6]]], ids=str)
@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_branches_are_accepted(calls, kept, dtype):
    """By the parents as they were drafted, whatever becomes of the tensor that gave them."""
    c = _cache()
    parents = torch.tensor(PARENTS, dtype=dtype)
    c.draft(parents)
    parents.fill_(-1)
    c.accept(kept)
    assert c._held == c._seen == [9 + len(k) for k in kept]
    assert sorted(c._free + sum(c._table, [])) == list(range(20))
    c.draft(torch.tensor([[-1, 0], [-1, -1]]))   # and the next draft goes by its own
    with pytest.raises(ValueError, match="branch"):
        c.accept([[0, 1], [0, 1]])
    c.accept([[0, 1], [1]])
