"""The C ABI of the decoding side on the CPU: the library exports what include/noble_decode.h declares, the header is plain C,
and bad arguments are refused before any HIP call.  Every call here has exactly one defect, so nothing reaches a device."""

import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2603_06492_amd import attention as na
from paper_2603_06492_amd import decoding as nd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "noble_decode.h")
NULL, SHAPE, DTYPE, MISAL, WS = 1, 2, 3, 4, 5
FAKE = [0x100000 + 0x1000 * i for i in range(32)]   # aligned, never dereferenced
REF = ctypes.byref
BIG = 1 << 50


def test_library_exports_every_declared_function():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(noble_[a-z_0-9]+)\s*\(", src))
    assert names == set(nd._SIGNATURES)
    for n in names:
        assert hasattr(nd.lib(), n), n


@pytest.mark.parametrize("lang,compiler", [("c99", "gcc"), ("c++17", "g++")])
def test_header_compiles_and_structures_match(lang, compiler, tmp_path):
    cc = shutil.which(compiler)
    if cc is None:
        pytest.skip(f"{compiler} not found")
    names = ["noble_keep_desc", "noble_select_desc", "noble_evict_desc"]
    checks = "\n".join(f"    if (sizeof({n}) != {ctypes.sizeof(getattr(nd, n))}) return {i + 1};" for i, n in enumerate(names))
    checks += f"\n    if (NOBLE_TREE_MOST != {nd.TREE_MOST}) return 9;"
    src = tmp_path / ("h.c" if lang == "c99" else "h.cpp")
    src.write_text(f'#include "noble_decode.h"\nint main(void) {{\n{checks}\n    return 0;\n}}\n')
    exe = tmp_path / "h"
    res = subprocess.run([cc, f"-std={lang}", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I",
                          os.path.join(ROOT, "include"), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    assert subprocess.run([str(exe)]).returncode == 0


def _desc(**kw):
    d = dict(B=3, table_row=100, pages=40, page=16, new_tokens=4, window=0, heads=8, kv_heads=2, head_dim=64, dtype=0,
             scale=0.125, softcap=0.0, reserved=0)
    d.update(kw)
    return na.noble_paged_desc(**d)


def _heads(at, **kw):
    d = dict(data=at, row=512, head=64)
    d.update(kw)
    return na.noble_heads(**d)


def _attention(name, d, ptrs=None, q=None, o=None, size=BIG, lead=()):
    """One attention call; ptrs replaces pointers by their place: cache, table, lengths, then the form's two, slopes, ..."""
    forms = {"noble_attn_tree": 6, "noble_attn_blocks": 5, "noble_attn_weigh": 6}
    p = list(FAKE[:forms[name]])
    p[{"noble_attn_tree": 5, "noble_attn_blocks": 4, "noble_attn_weigh": 3}[name]] = None   # slopes
    scratch = FAKE[20]
    for i, v in (ptrs or {}).items():
        if i == "scratch":
            scratch = v
        else:
            p[i] = v
    q = _heads(FAKE[10]) if q is None else q
    o = _heads(FAKE[11]) if o is None else o
    return getattr(nd.lib(), name)(None if d is None else REF(d), *lead, q and REF(q), *p, o and REF(o), scratch, size, None)


FORMS = [("noble_attn_tree", ()), ("noble_attn_blocks", (60,)), ("noble_attn_weigh", ())]
BAD = [dict(B=-1), dict(table_row=-1), dict(table_row=2 ** 40), dict(pages=-1), dict(pages=2 ** 31), dict(page=4), dict(page=24),
       dict(page=8192), dict(new_tokens=0), dict(new_tokens=-1), dict(new_tokens=2 ** 21), dict(window=1), dict(heads=0),
       dict(heads=7), dict(heads=2048), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0), dict(head_dim=60),
       dict(head_dim=136), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(softcap=-1.0),
       dict(softcap=math.nan), dict(reserved=1), dict(B=2 ** 31)]


@pytest.mark.parametrize("name,lead", FORMS)
@pytest.mark.parametrize("bad", BAD, ids=str)
def test_attention_shapes(name, lead, bad):
    n = ctypes.c_size_t(7)
    assert _attention(name, _desc(**bad), lead=lead) == SHAPE
    assert getattr(nd.lib(), name + "_scratch_size")(REF(_desc(**bad)), *lead, REF(n)) == SHAPE and n.value == 7


@pytest.mark.parametrize("name,lead", FORMS)
def test_attention_pointers_and_strides(name, lead):
    n, L = ctypes.c_size_t(0), nd.lib()
    size = getattr(L, name + "_scratch_size")
    assert size(REF(_desc()), *lead, REF(n)) == 0 and n.value > 0
    assert size(REF(_desc()), *lead, None) == NULL and size(None, *lead, REF(n)) == NULL
    assert _attention(name, None, lead=lead) == NULL
    assert _attention(name, _desc(dtype=2), lead=lead) == DTYPE
    assert _attention(name, _desc(), size=n.value - 1, lead=lead) == WS
    assert _attention(name, _desc(), {"scratch": None}, lead=lead) == NULL
    assert _attention(name, _desc(), {"scratch": FAKE[20] + 8}, lead=lead) == MISAL
    optional = {"noble_attn_tree": {5}, "noble_attn_blocks": {4}, "noble_attn_weigh": {3, 4}}[name]
    for i in range({"noble_attn_blocks": 5}.get(name, 6)):
        if i not in optional:
            assert _attention(name, _desc(), {i: None}, lead=lead) == NULL, i
        assert _attention(name, _desc(), {i: FAKE[i] + (8 if i == 0 else 2)}, lead=lead) == MISAL, i
    for bad, want in ((dict(data=None), NULL), (dict(data=FAKE[10] + 8), MISAL), (dict(row=-8), SHAPE), (dict(row=4), SHAPE),
                      (dict(head=3), SHAPE), (dict(row=2 ** 23), SHAPE)):
        assert _attention(name, _desc(), q=_heads(**{"at": FAKE[10], **bad}), lead=lead) == want, bad
        assert _attention(name, _desc(), o=_heads(**{"at": FAKE[11], **bad}), lead=lead) == want, bad
    assert _attention(name, _desc(), o=_heads(FAKE[11], row=0), lead=lead) == SHAPE    # an output's rows are distinct


def test_own_limits_of_the_forms():
    assert _attention("noble_attn_tree", _desc(new_tokens=257)) == SHAPE
    for count in (0, -1, 65537):
        assert _attention("noble_attn_blocks", _desc(), lead=(count,)) == SHAPE
    # scores of every row and token past what a scratch may hold
    n = ctypes.c_size_t(0)
    d = _desc(B=1024, new_tokens=1024, table_row=2 ** 22, page=256)
    assert nd.lib().noble_attn_weigh_scratch_size(REF(d), REF(n)) == SHAPE


def test_tree_rows():
    f = nd.lib().noble_tree_rows
    for B, n in ((-1, 4), (2, 0), (2, 257), (2, -1), (2 ** 40, 4)):
        assert f(B, n, *FAKE[:5], None) == SHAPE
    for i in range(4):   # parents, lengths, seen, depths; positions may be missing, and then lengths too
        assert f(2, 4, *[None if x == i else p for x, p in enumerate(FAKE[:5])], None) == NULL, i
        assert f(2, 4, *[p + 2 if x == i else p for x, p in enumerate(FAKE[:5])], None) == MISAL, i
    assert f(2, 4, *FAKE[:4], FAKE[4] + 2, None) == MISAL


def _keep(**kw):
    d = dict(B=2, table_row=10, pages=30, most=100, page=16, kv_heads=4, head_dim=64, kept_heads=4, dtype=0, reserved=0)
    d.update(kw)
    return nd.noble_keep_desc(**d)


def test_cache_keep():
    f = nd.lib().noble_cache_keep
    for bad in (dict(B=-1), dict(table_row=-1), dict(pages=-1), dict(most=-1), dict(most=2 ** 31), dict(page=4), dict(page=20),
                dict(kv_heads=0, kept_heads=0), dict(kept_heads=2), dict(kept_heads=0), dict(head_dim=12), dict(head_dim=256),
                dict(reserved=1), dict(kv_heads=1025, kept_heads=1)):
        assert f(REF(_keep(**bad)), *FAKE[:4], None) == SHAPE, bad
    assert f(None, *FAKE[:4], None) == NULL and f(REF(_keep(dtype=3)), *FAKE[:4], None) == DTYPE
    for i in range(3):
        assert f(REF(_keep()), *[None if x == i else p for x, p in enumerate(FAKE[:4])], None) == NULL
    for i in range(4):
        assert f(REF(_keep()), *[p + (8 if i == 0 else 2) if x == i else p for x, p in enumerate(FAKE[:4])], None) == MISAL


def test_page_means():
    f = nd.lib().noble_page_means
    for bad in (dict(B=-1), dict(table_row=-1), dict(pages=-1), dict(page=4), dict(new_tokens=0), dict(kv_heads=0),
                dict(head_dim=12), dict(reserved=1), dict(window=3)):
        assert f(REF(_desc(**bad)), *FAKE[:4], None) == SHAPE, bad
    assert f(None, *FAKE[:4], None) == NULL and f(REF(_desc(dtype=3)), *FAKE[:4], None) == DTYPE
    for i in range(4):
        assert f(REF(_desc()), *[None if x == i else p for x, p in enumerate(FAKE[:4])], None) == NULL
        assert f(REF(_desc()), *[p + (8 if i in (0, 3) else 2) if x == i else p for x, p in enumerate(FAKE[:4])], None) == MISAL


def test_block_select():
    f, n = nd.lib().noble_block_select, ctypes.c_size_t(7)
    q, e = _heads(FAKE[10]), nd.noble_select_desc(6, 1, 2, 0)
    call = lambda d=None, s=e, q=q, p=FAKE[:4], size=BIG: f(REF(d or _desc()), s and REF(s), q and REF(q), *p, FAKE[20], size, None)  # noqa: E731
    for bad in BAD:
        assert call(_desc(**bad)) == SHAPE, bad
    for s in ((0, 0, 1), (6, -1, 1), (6, 0, 0), (6, 5, 2), (65537, 0, 1), (6, 2 ** 31 - 1, 6)):
        assert call(s=nd.noble_select_desc(*s, 0)) == SHAPE, s
    assert call(s=nd.noble_select_desc(6, 1, 2, 1)) == SHAPE and call(s=None) == NULL and call(q=None) == NULL
    for i in range(4):
        assert call(p=[None if x == i else v for x, v in enumerate(FAKE[:4])]) == NULL
        assert call(p=[v + (8 if i == 0 else 2) if x == i else v for x, v in enumerate(FAKE[:4])]) == MISAL
    size = nd.lib().noble_block_select_scratch_size
    assert size(REF(_desc()), REF(e), REF(n)) == 0 and n.value == 0
    assert size(REF(_desc(table_row=20000)), REF(e), REF(n)) == 0 and n.value == 3 * 4 * 2 * 20000 * 8
    assert call(_desc(table_row=20000), size=n.value - 1) == WS
    assert size(REF(_desc()), REF(e), None) == NULL and size(None, REF(e), REF(n)) == NULL


def test_block_select_scratch_of_few_rows_and_many():
    """Few rows of many blocks take scratch for their scores; many rows, or few blocks, take none."""
    f, size, n = nd.lib().noble_block_select, nd.lib().noble_block_select_scratch_size, ctypes.c_size_t(7)
    q, e = _heads(FAKE[10]), nd.noble_select_desc(6, 1, 2, 0)
    for row, B, some in ((511, 3, 0), (512, 3, 1), (640, 3, 1), (640, 50, 0), (16384, 3, 1), (16384, 50, 0)):
        d = _desc(table_row=row, B=B)
        assert size(REF(d), REF(e), REF(n)) == 0 and n.value == some * B * 4 * 2 * row * 8, (row, B)
        if some:
            assert f(REF(d), REF(e), REF(q), *FAKE[:4], FAKE[20], n.value - 1, None) == WS
            assert f(REF(d), REF(e), REF(q), *FAKE[:4], None, n.value, None) == NULL


def test_evict_select():
    f = nd.lib().noble_evict_select
    make = lambda B=2, row=100, heads=4, keep=10, sink=1, recent=2, r=(0, 0): nd.noble_evict_desc(B, row, heads, keep, sink, recent, r)  # noqa: E731
    for bad in (dict(B=-1), dict(row=-1), dict(row=2 ** 31), dict(heads=0), dict(heads=1025), dict(keep=0), dict(sink=-1),
                dict(recent=-1), dict(sink=8, recent=3), dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), dict(r=(1, 0)), dict(r=(0, 1))):
        assert f(REF(make(**bad)), *FAKE[:4], None) == SHAPE, bad
    assert f(None, *FAKE[:4], None) == NULL
    for i in range(3):
        assert f(REF(make()), *[None if x == i else p for x, p in enumerate(FAKE[:4])], None) == NULL
    for i in range(4):
        assert f(REF(make()), *[p + 2 if x == i else p for x, p in enumerate(FAKE[:4])], None) == MISAL


def test_python_refuses_what_is_no_gpu_tensor():
    """CPU tensors, and other things, are refused by every function before the library is called."""
    f, i = torch.zeros, lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    q, cache, table, lens = f(3, 2, 8), f(4, 2, 1, 8, 8), i(3, 1), i(3)
    for call in (lambda: nd.noble_tree_rows(i(3, 1), lens), lambda: nd.noble_attn_tree(q, cache, table, lens, i(3, 1, 1), i(3, 1)),
                 lambda: nd.noble_cache_keep(cache, table, i(3, 1, 4)), lambda: nd.noble_page_means(cache, table, lens, 1),
                 lambda: nd.noble_block_select(q, f(4, 1, 8), table, lens, 2, page=8),
                 lambda: nd.noble_attn_blocks(q, cache, table, lens, i(3, 1, 2)),
                 lambda: nd.noble_attn_weigh(q, cache, table, lens), lambda: nd.noble_evict_select(f(3, 1, 8), lens, 2)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: nd.noble_tree_rows(None, lens), lambda: nd.noble_attn_weigh([1], cache, table, lens),
                 lambda: nd.noble_evict_select(None, lens, 2), lambda: nd.noble_cache_keep(None, table, i(3, 1, 4))):
        with pytest.raises(TypeError):
            call()


def test_paged_cache_refusals():
    c = na.PagedCache(2, 40, 12, kv_heads=1, head_dim=8, page=8, device="cpu")
    c.extend(9)
    with pytest.raises(RuntimeError):
        c.accept([[], []])
    with pytest.raises(ValueError, match="weights"):
        c.evict(4)
    for bad in (torch.zeros(3, 2), torch.zeros(2, 0), torch.zeros(2, 257), torch.zeros(2)):
        with pytest.raises(ValueError):
            c.draft(bad)
    with pytest.raises(ValueError):
        c.draft(torch.zeros(2, 32))
    assert c.held == c.seen == 9
    w = na.PagedCache(2, 40, 12, kv_heads=1, head_dim=8, page=8, device="cpu", weights=True)
    w.extend(9)
    for keep, sink, recent in ((0, 0, 0), (4, 3, 2), (4, -1, 0), (4, 0, -1)):
        with pytest.raises(ValueError):
            w.evict(keep, sink=sink, recent=recent)
    w.evict(9)   # nothing to do
    assert w.held == 9
