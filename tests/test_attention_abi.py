"""The C ABI of the attention side on the CPU: the library exports what include/noble_attn.h declares, the header is plain C,
and bad arguments are refused before any HIP call.  Every call here has exactly one defect, so nothing reaches a
device."""

import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest

from paper_2603_06492_amd import attention as na
from paper_2603_06492_amd import noble

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "noble_attn.h")
NULL, SHAPE, DTYPE, MISAL, WS = 1, 2, 3, 4, 5
FAKE = [0x100000 + 0x1000 * i for i in range(32)]   # aligned, never dereferenced
REF = ctypes.byref


def test_library_exports_every_declared_function():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(noble_[a-z_0-9]+)\s*\(", src))
    assert names == set(na._SIGNATURES)
    for n in names:
        assert hasattr(na.lib(), n), n


@pytest.mark.parametrize("lang,compiler", [("c99", "gcc"), ("c++17", "g++")])
def test_header_compiles_and_structures_match(lang, compiler, tmp_path):
    cc = shutil.which(compiler)
    if cc is None:
        pytest.skip(f"{compiler} not found")
    names = [n for n in dir(na) if n.startswith("noble_") and isinstance(getattr(na, n), type)]
    checks = "\n".join(f"    if (sizeof({n}) != {ctypes.sizeof(getattr(na, n))}) return {i + 1};"
                       for i, n in enumerate(names))
    src = tmp_path / ("h.c" if lang == "c99" else "h.cpp")
    src.write_text(f'#include "noble_attn.h"\nint main(void) {{\n{checks}\n    return 0;\n}}\n')
    exe = tmp_path / "h"
    res = subprocess.run([cc, f"-std={lang}", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I",
                          os.path.join(ROOT, "include"), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    assert len(names) >= 6 and subprocess.run([str(exe)]).returncode == 0


def _rope(**kw):
    d = dict(T=10, x_row=6 * 64, table_rows=16, heads=2, kv_heads=2, head_dim=64, rot=32, interleaved=0, dtype=0,
             eps=1e-6, reserved=0)
    d.update(kw)
    return na.noble_rope_desc(**d)


BAD_ROPE = [dict(T=-1), dict(T=2 ** 31), dict(heads=-1), dict(heads=1025), dict(head_dim=0), dict(head_dim=60),
            dict(head_dim=136, x_row=6 * 136), dict(rot=8), dict(rot=80), dict(rot=-16), dict(x_row=248), dict(x_row=388),
            dict(table_rows=-1), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(reserved=1),
            dict(kv_heads=-1)]


@pytest.mark.parametrize("bad", BAD_ROPE, ids=str)
def test_rope_shapes(bad):
    d, n = _rope(**bad), ctypes.c_size_t(7)
    L = na.lib()
    assert L.noble_qk_rope_fwd(REF(d), *FAKE[:8], None) == SHAPE
    assert L.noble_qk_rope_scratch_size(REF(d), REF(n)) == SHAPE and n.value == 7
    assert L.noble_qk_rope_bwd(REF(d), *FAKE[:12], 1 << 30, None) == SHAPE


def test_rope_pointers():
    L, d = na.lib(), _rope()
    assert L.noble_qk_rope_fwd(None, *FAKE[:8], None) == NULL
    assert L.noble_qk_rope_fwd(REF(_rope(dtype=2)), *FAKE[:8], None) == DTYPE
    for i in (0, 1, 2, 3, 4, 6, 7):   # x, one of the weights, cos, sin, q, k
        assert L.noble_qk_rope_fwd(REF(d), *[None if n == i else p for n, p in enumerate(FAKE[:8])], None) == NULL, i
    for i in range(8):
        off = 1 if i in (1, 2, 5) else 8
        assert L.noble_qk_rope_fwd(REF(d), *[p + off if n == i else p for n, p in enumerate(FAKE[:8])], None) == MISAL, i
    n = ctypes.c_size_t(0)
    assert L.noble_qk_rope_scratch_size(REF(d), REF(n)) == 0 and n.value > 0
    assert L.noble_qk_rope_scratch_size(REF(d), None) == NULL
    assert L.noble_qk_rope_bwd(REF(d), *FAKE[:12], n.value - 1, None) == WS
    for i in (0, 1, 2, 9, 10, 11):   # dq, dk, x, dq_weight, dk_weight of weights that are there, scratch
        args = [None if m == i else p for m, p in enumerate(FAKE[:12])]
        assert L.noble_qk_rope_bwd(REF(d), *args, n.value, None) == NULL, i


def test_append_refusals():
    L = na.lib()
    c = na.noble_cache_desc(4, 16, 0)
    for bad in (dict(kv_heads=0), dict(x_row=5 * 64)):
        assert L.noble_kv_append(REF(_rope(**bad)), REF(c), *FAKE[:9], None) == SHAPE
    for page in (0, 4, 12, 8192):
        assert L.noble_kv_append(REF(_rope()), REF(na.noble_cache_desc(4, page, 0)), *FAKE[:9], None) == SHAPE
    assert L.noble_kv_append(REF(_rope()), REF(na.noble_cache_desc(-1, 16, 0)), *FAKE[:9], None) == SHAPE
    assert L.noble_kv_append(REF(_rope()), None, *FAKE[:9], None) == NULL
    for i in (0, 6, 8):   # x, slots, cache
        assert L.noble_kv_append(REF(_rope()), REF(c), *[None if n == i else p for n, p in enumerate(FAKE[:9])],
                                 None) == NULL, i
    assert L.noble_kv_append(REF(_rope()), REF(c), *[p + 4 if n == 6 else p for n, p in enumerate(FAKE[:9])], None) == MISAL


def _attn(**kw):
    d = dict(Tq=30, Tk=40, offset=10, heads=4, kv_heads=2, head_dim=64, dtype=0, causal=1, scale=0.125, softcap=0.0,
             reserved=0)
    d.update(kw)
    return na.noble_attn_desc(**d)


def _fwd(d, heads=None, lo=None, hi=None, lse=FAKE[5]):
    h = [na.noble_heads(FAKE[i], 256 if i in (0, 3) else 128, 64) for i in range(4)]
    for i, new in (heads or {}).items():
        h[i] = new
    q, k, v, o = (None if x is None else REF(x) for x in h)
    return na.lib().noble_attn_fwd(None if d is None else REF(d), q, k, v, lo, hi, None, o, lse, None)


BAD_ATTN = [dict(Tq=-1), dict(Tk=2 ** 31), dict(offset=2 ** 31), dict(heads=0), dict(heads=3), dict(heads=2048),
            dict(kv_heads=0), dict(head_dim=4), dict(head_dim=12), dict(head_dim=256), dict(scale=0.0), dict(scale=-1.0),
            dict(scale=math.nan), dict(scale=math.inf), dict(softcap=-1.0), dict(softcap=math.nan), dict(reserved=3)]


@pytest.mark.parametrize("bad", BAD_ATTN, ids=str)
def test_attention_shapes(bad):
    n = ctypes.c_size_t(0)
    assert _fwd(_attn(**bad)) == SHAPE
    assert na.lib().noble_attn_bwd_scratch_size(REF(_attn(**bad)), REF(n)) == SHAPE


def test_attention_pointers_and_strides():
    H = na.noble_heads
    assert _fwd(None) == NULL and _fwd(_attn(dtype=7)) == DTYPE
    for i in range(4):
        assert _fwd(_attn(), {i: None}) == NULL
        assert _fwd(_attn(), {i: H(None, 256, 64)}) == NULL
        assert _fwd(_attn(), {i: H(FAKE[i] + 8, 256, 64)}) == MISAL
        for row, head in ((-256, 64), (256, -64), (260, 64), (256, 68), (2 ** 23, 64), (256, 2 ** 41)):
            assert _fwd(_attn(), {i: H(FAKE[i], row, head)}) == SHAPE, (i, row, head)
    for row, head in ((0, 64), (256, 0), (64, 64), (192, 64), (64, 64 * 29)):   # elements of the output would coincide
        assert _fwd(_attn(), {3: H(FAKE[3], row, head)}) == SHAPE, (row, head)
    assert _fwd(_attn(), lo=FAKE[6]) == NULL and _fwd(_attn(), hi=FAKE[6]) == NULL
    assert _fwd(_attn(), lo=FAKE[6] + 2, hi=FAKE[7]) == MISAL
    assert _fwd(_attn(), lse=None) == NULL and _fwd(_attn(), lse=FAKE[5] + 2) == MISAL


def test_attention_backward_refusals():
    L, d = na.lib(), _attn()
    n = ctypes.c_size_t(0)
    assert L.noble_attn_bwd_scratch_size(REF(d), REF(n)) == 0
    assert n.value >= 2 * 4 * 4 * 30   # lse and delta of four heads
    def bwd(swap=None, lse=FAKE[10], scratch=FAKE[11], size=n.value):
        # grad, q, k, v, o, dq, dk, dv
        h = [na.noble_heads(FAKE[i], 128 if i in (2, 3, 6, 7) else 256, 64) for i in range(8)]
        if swap:
            h[swap[0]] = swap[1]
        r = [None if x is None else REF(x) for x in h]
        return L.noble_attn_bwd(REF(d), *r[:5], lse, None, None, None, *r[5:], scratch, size, None)
    for i in range(8):
        assert bwd((i, None)) == NULL and bwd((i, na.noble_heads(FAKE[i] + 4, 256, 64))) == MISAL
    for i in (5, 6, 7):
        assert bwd((i, na.noble_heads(FAKE[i], 0, 64))) == SHAPE
    assert bwd(lse=None) == NULL and bwd(size=n.value - 1) == WS and bwd(scratch=None) == NULL


def _paged(**kw):
    d = dict(B=3, table_row=10, pages=40, page=16, new_tokens=1, window=0, heads=4, kv_heads=2, head_dim=64, dtype=0,
             scale=0.125, softcap=0.0, reserved=0)
    d.update(kw)
    return na.noble_paged_desc(**d)


BAD_PAGED = [dict(B=-1), dict(table_row=-1), dict(table_row=2 ** 31), dict(pages=-1), dict(pages=2 ** 31), dict(page=0),
             dict(page=4), dict(page=24), dict(page=8192), dict(new_tokens=0), dict(new_tokens=2 ** 21), dict(window=-1),
             dict(heads=5), dict(kv_heads=0), dict(head_dim=160), dict(scale=0.0), dict(softcap=-2.0), dict(reserved=1)]


def _call_paged(d, size=1 << 30, swap=None, q=(256, 64), o=(256, 64)):
    p = dict(cache=FAKE[1], table=FAKE[2], lengths=FAKE[3], slopes=FAKE[4], scratch=FAKE[6])
    p.update(swap or {})
    return na.lib().noble_attn_paged(REF(d), REF(na.noble_heads(FAKE[0], *q)), p["cache"], p["table"], p["lengths"],
                                     p["slopes"], REF(na.noble_heads(FAKE[5], *o)), p["scratch"], size, None)


@pytest.mark.parametrize("bad", BAD_PAGED, ids=str)
def test_paged_shapes(bad):
    n = ctypes.c_size_t(0)
    assert _call_paged(_paged(**bad)) == SHAPE
    assert na.lib().noble_attn_paged_scratch_size(REF(_paged(**bad)), REF(n)) == SHAPE


def test_paged_pointers():
    n = ctypes.c_size_t(0)
    d = _paged(table_row=1000)
    assert na.lib().noble_attn_paged_scratch_size(REF(d), REF(n)) == 0 and n.value > 0
    assert na.lib().noble_attn_paged_scratch_size(REF(d), None) == NULL
    assert _call_paged(d, n.value - 1) == WS
    for k in ("cache", "table", "lengths", "scratch"):
        assert _call_paged(d, swap={k: None}) == NULL, k
        assert _call_paged(d, swap={k: FAKE[9] + 2}) == MISAL, k
    assert _call_paged(d, o=(0, 64)) == SHAPE and _call_paged(d, q=(252, 64)) == SHAPE
    assert _call_paged(_paged(dtype=5)) == DTYPE


def test_table_and_mask_refusals():
    L = na.lib()
    def table(length=10, rot=32, cos=FAKE[0], sin=FAKE[1], **kw):
        d = dict(kind=0, reserved=0, base=1e4, factor=1.0, trained=0.0, fast=32.0, slow=1.0, gain=1.0)
        d.update(kw)
        return L.noble_rope_table(REF(na.noble_rope_scaling(**d)), length, rot, cos, sin, None)
    for bad in (dict(length=-1), dict(rot=0), dict(rot=24), dict(rot=144), dict(kind=4), dict(kind=-1), dict(base=1.0),
                dict(base=math.inf), dict(kind=1, factor=0.5), dict(kind=2, factor=math.nan), dict(kind=3), dict(reserved=1),
                dict(kind=3, trained=100.0, fast=1.0), dict(kind=3, trained=100.0, slow=0.0),
                dict(kind=3, trained=100.0, gain=0.0)):
        assert table(**bad) == SHAPE, bad
    assert table(cos=None) == NULL and table(sin=FAKE[1] + 4) == MISAL
    assert L.noble_rope_table(None, 10, 32, FAKE[0], FAKE[1], None) == NULL
    mask = lambda T=5, n=2, a=(0, 1, 2, 3, 4), window=0: L.noble_mask_rows(  # noqa: E731
        T, n, *[None if i is None else FAKE[i] for i in a[:2]], 1, window, *[None if i is None else FAKE[i] for i in a[2:]],
        None)
    assert mask(T=-1) == mask(n=-1) == mask(window=-1) == mask(T=2 ** 31) == SHAPE
    assert mask(a=(None, 1, 2, 3, 4)) == mask(a=(0, 1, None, 3, 4)) == mask(a=(0, 1, 2, None, 4)) == NULL


def test_python_refuses_before_the_library():
    torch = pytest.importorskip("torch")
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU"):
        na.noble_attn_fwd(q, q, q)
    with pytest.raises(ValueError, match="on the GPU"):
        na.noble_qk_rope_fwd(torch.zeros(4, 384), None, None, None, None, None, heads=2, kv_heads=2)
    with pytest.raises(TypeError):
        na.noble_attn_paged("q", None, None, None)
    with pytest.raises(ValueError, match="unknown scaling"):
        na.noble_rope_table(4, 32, scaling="other")
    n = na._native()
    assert n.rope_fwd() is None and n.attn_fwd(*[q] * 12) is None and n.paged(*[None] * 9) is None
    assert n.attn_bwd(*[None] * 16) is None and n.append(*[None] * 13) is None and n.rope_bwd(*[q] * 13) is None
    assert noble.ABI_VERSION == 5
