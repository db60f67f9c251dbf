"""Limits of the decoding calls' numbers, on the CPU: what the kernels count in 32 bits is refused past them.  Every call here
has exactly one defect, so nothing reaches a device."""

import ctypes

import pytest

from paper_2603_06492_amd import attention as na
from paper_2603_06492_amd import decoding as nd

SHAPE = 2
FAKE = [0x100000 + 0x1000 * i for i in range(4)]   # aligned, never dereferenced
MOST = 2 ** 31 - 4096


@pytest.mark.parametrize("keep,sink,recent", [(MOST + 1, 0, 0), (2 ** 31 - 1024, 1, 2), (2 ** 31 - 1, 0, 0),
                                              (2 ** 31 - 1, 2 ** 30, 2 ** 30 - 1)])
@pytest.mark.parametrize("B,row", [(2, 100), (1, MOST), (1, 0)])
def test_evict_select_keeps_no_more_than_its_counters_hold(keep, sink, recent, B, row):
    """The entries behind the last token are filled 1024 at a time, by a number that would pass 2^31 and come back negative:
    kept[i] lay gigabytes before the list."""
    d = nd.noble_evict_desc(B, row, 4, keep, sink, recent)
    assert nd.lib().noble_evict_select(ctypes.byref(d), *FAKE, None) == SHAPE


def test_python_refuses_it_before_the_lists_are_made(monkeypatch):
    """Their 17 GB for each head are not asked for."""
    import torch
    monkeypatch.setattr(nd, "_gpu", lambda t, name: t.device)
    monkeypatch.setattr(nd, "_native", lambda: type("Native", (), {"evict_select": staticmethod(lambda *a: None)}))
    monkeypatch.setattr(nd, "_tensor", lambda *a: FAKE[0])
    w, lengths = torch.zeros(1, 1, 8), torch.zeros(1, dtype=torch.int32)
    for keep in (MOST + 1, 2 ** 31 - 1, 2 ** 31):
        with pytest.raises(ValueError, match="keep"):
            nd.noble_evict_select(w, lengths, keep)


@pytest.mark.parametrize("B,new,heads,tokens", [(8, 512, 32, 32768), (1, 1, 4, 1 << 20), (64, 1, 16, 32768), (3, 5, 8, 96)])
def test_the_weights_scratch_goes_by_the_page_table(B, new, heads, tokens):
    """Four bytes for each row, query head and token of the table, and little else."""
    d = na.noble_paged_desc(B, tokens // 16, 100, 16, new, 0, heads, 4, 64, 0, 0.125, 0.0, 0)
    n = ctypes.c_size_t(0)
    assert nd.lib().noble_attn_weigh_scratch_size(ctypes.byref(d), ctypes.byref(n)) == 0
    scores = B * new * heads * -(-tokens // 64) * 64 * 4
    # maxima and sums of every row, and parts of 16 to 256 rows of 64 + 4 floats for up to some thousand workgroups
    assert scores <= n.value <= scores + B * new * heads * 8 + 4096 * 256 * 68 * 4
