"""Limits of the decoding calls' numbers, on the CPU: what the kernels count in 32 bits is refused past them.  Every call here
has exactly one defect, so nothing reaches a device."""

import ctypes

import pytest

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
