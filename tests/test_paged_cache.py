"""The page bookkeeping of PagedCache, on the CPU."""

import pytest
import torch

from paper_2603_06492_amd.attention import PagedCache


def _state(c):
    return c.lengths.tolist(), c.page_table.tolist(), list(c._held), [list(t) for t in c._table], list(c._free)


def test_extend_refuses_fewer_than_no_tokens():
    c = PagedCache(2, 40, 12, kv_heads=1, head_dim=8, page=8, device="cpu")
    c.extend(9)
    before = _state(c)
    with pytest.raises(ValueError):
        c.extend(-3)
    assert _state(c) == before
    positions, slots = c.extend(0)
    assert positions.shape == slots.shape == (0,) and (positions.dtype, slots.dtype) == (torch.int32, torch.int64)
    assert _state(c) == before
    positions, _ = c.extend(2)
    assert positions.tolist() == [9, 10] * 2
