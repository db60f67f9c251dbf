"""Python binding of libnoble's decoding side (include/noble_decode.h): decoding over the paged cache beyond one token after
the other.

The functions keep the C names and take torch tensors: ``noble_tree_rows``, ``noble_attn_tree``, ``noble_cache_keep``
(trees of drafted tokens and the branch that is accepted); ``noble_page_means``, ``noble_block_select``,
``noble_attn_blocks`` (attention over selected pages); ``noble_attn_weigh``, ``noble_evict_select`` (attention that adds up
the weight each cached token receives, and the tokens with the most of it, which ``noble_cache_keep`` moves together).  They
check their arguments, allocate the outputs that are not given and the scratch, and enqueue all their work on ``stream``
(default: torch's current stream), where the inputs have to be ready, as the functions of ``attention`` do.
``NobleSelfAttention.step`` and ``PagedCache`` there call them.

There is no fallback: without the built library or a gfx950 device, calls raise.
"""

from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import Optional, Tuple

import torch

from . import noble
from .attention import (_cache_shape, _gpu, _heads, _P, _scratch, _served, _tensor, _work, noble_heads, noble_paged_desc)
from .noble import NobleError, _dtype_code

_vp = ctypes.c_void_p
_i64, _i32, _sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t

TREE_MOST = 256   # NOBLE_TREE_MOST


class noble_keep_desc(ctypes.Structure):
    _fields_ = [("B", _i64), ("table_row", _i64), ("pages", _i64), ("most", _i64), ("page", _i32), ("kv_heads", _i32),
                ("head_dim", _i32), ("kept_heads", _i32), ("dtype", _i32), ("reserved", _i32)]


class noble_select_desc(ctypes.Structure):
    _fields_ = [("count", _i32), ("sink", _i32), ("local", _i32), ("reserved", _i32)]


class noble_evict_desc(ctypes.Structure):
    _fields_ = [("B", _i64), ("row", _i64), ("heads", _i32), ("keep", _i32), ("sink", _i32), ("recent", _i32),
                ("reserved", _i32 * 2)]


_pd, _hp = _P(noble_paged_desc), _P(noble_heads)
_SIGNATURES = {
    "noble_tree_rows": [_i64, _i32] + [_vp] * 6,
    "noble_attn_tree_scratch_size": [_pd, _P(_sz)],
    "noble_attn_tree": [_pd, _hp] + [_vp] * 6 + [_hp, _vp, _sz, _vp],
    "noble_cache_keep": [_P(noble_keep_desc)] + [_vp] * 5,
    "noble_page_means": [_pd] + [_vp] * 5,
    "noble_block_select_scratch_size": [_pd, _P(noble_select_desc), _P(_sz)],
    "noble_block_select": [_pd, _P(noble_select_desc), _hp] + [_vp] * 5 + [_sz, _vp],
    "noble_attn_blocks_scratch_size": [_pd, _i32, _P(_sz)],
    "noble_attn_blocks": [_pd, _i32, _hp] + [_vp] * 5 + [_hp, _vp, _sz, _vp],
    "noble_attn_weigh_scratch_size": [_pd, _P(_sz)],
    "noble_attn_weigh": [_pd, _hp] + [_vp] * 6 + [_hp, _vp, _sz, _vp],
    "noble_evict_select": [_P(noble_evict_desc)] + [_vp] * 5,
}
_ready = False


def lib() -> ctypes.CDLL:
    """The loaded libnoble.so with these functions' signatures (raises if it has not been built)."""
    global _ready
    L = noble.lib()
    if not _ready:
        for name, args in _SIGNATURES.items():
            f = getattr(L, name)
            f.restype, f.argtypes = ctypes.c_int, args
        _ready = True
    return L


BINDING_PATH = os.path.join(noble.PKG_DIR, "_noble_decode_torch.so")
_native_module = None


def _native():
    """The native calls (_noble_decode_torch.so), given the library's entry points.  They serve well-formed calls on ordinary
    tensors and the current stream and return None for any other, which the Python code then checks and runs."""
    global _native_module
    if _native_module is None:
        L = lib()
        if not os.path.exists(BINDING_PATH):
            raise RuntimeError(f"{BINDING_PATH} is missing: build it with __graft_entry__.build() "
                               "(or python -m paper_2603_06492_amd._build)")
        spec = importlib.util.spec_from_file_location("_noble_decode_torch", BINDING_PATH)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        m.init(*(ctypes.cast(getattr(L, n), _vp).value for n in (
            "noble_tree_rows", "noble_attn_tree", "noble_attn_tree_scratch_size", "noble_cache_keep", "noble_page_means",
            "noble_block_select", "noble_block_select_scratch_size", "noble_attn_blocks", "noble_attn_blocks_scratch_size",
            "noble_attn_weigh", "noble_attn_weigh_scratch_size", "noble_evict_select")))
        _native_module = m
    return _native_module


def _call(name, *args) -> None:
    st = getattr(lib(), name)(*args)
    if st != 0:
        raise NobleError(st, name)


def _size(name, *args) -> int:
    n = _sz(0)
    _call(name, *args, ctypes.byref(n))
    return n.value


def _need(t, name):
    if t is None:
        raise TypeError(f"{name} must be a torch.Tensor")
    return t


def _whole(**numbers) -> None:
    """Whole numbers as the descriptors' 32 bits hold them."""
    for name, n in numbers.items():
        if not 0 <= n < 2 ** 31:
            raise ValueError(f"{name}={n}")


def _int32(t, name, shape, device):
    return _tensor(_need(t, name), name, torch.int32, shape, device)


class _Sequences:
    """The checked arguments that the attention calls share: q [B n, heads, D], the cache, its page table and lengths."""

    def __init__(self, q, cache, page_table, lengths, slopes, scale, softcap):
        self.dev = dev = _gpu(q, "q")
        if q.dim() != 3 or not isinstance(page_table, torch.Tensor) or page_table.dim() != 2 or page_table.shape[0] < 1:
            raise ValueError("q must be [rows, heads, head_dim] and page_table [sequences, pages]")
        rows, H, D = self.shape = tuple(q.shape)
        B, per = page_table.shape
        if rows % B or rows < B:
            raise ValueError(f"{rows} rows of q are not the same number for each of {B} sequences")
        K = cache.shape[2] if isinstance(cache, torch.Tensor) and cache.dim() == 5 else 0
        pages, page, self.cache = _cache_shape(cache, K, D, q.dtype, dev)
        self.B, self.n, self.K, self.tokens = B, rows // B, K, per * page
        self.dtype, self.q = q.dtype, _heads(q, "q", q.dtype, dev)
        self.table = _int32(page_table, "page_table", (B, per), dev)
        self.lengths = _int32(lengths, "lengths", (B,), dev)
        self.slopes = _tensor(slopes, "slopes", torch.float32, (H,), dev)
        self.desc = noble_paged_desc(B, per, pages, page, self.n, 0, H, K, D, _dtype_code(q),
                                     D ** -0.5 if scale is None else scale, softcap, 0)

    def output(self, o):
        """The given or a new o, and its checked argument."""
        o = torch.empty(self.shape, dtype=self.dtype, device=self.dev) if o is None else o
        return o, ctypes.byref(_heads(o, "o", self.dtype, self.dev, self.shape))


def _buffer(n, device):
    t = _scratch(n, device) if n else None
    return t, None if t is None else t.data_ptr()


# -------------------------------------------------------------------- tree --

def noble_tree_rows(parents, lengths, *, stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(seen, depths, positions) of the trees that each sequence's last n tokens form: parents int32 [B, n], a node's parent
    an earlier node, or -1 (the last token before the tree); any other number: no node, nor what hangs from it.  seen int32
    [B, n, (n + 31) // 32], a bit for each node of the line from the root to the node; depths int32 [B, n] (no node: -1);
    positions int32 [B, n], lengths - n + depth (no node: 0), lengths int32 [B] with the tree's tokens."""
    if stream is None:
        out = _native().tree_rows(parents, lengths)
        if _served(out, "noble_tree_rows"):
            return out
    dev = _gpu(parents, "parents")
    if parents.dim() != 2:
        raise ValueError(f"parents must be [sequences, nodes], got {tuple(parents.shape)}")
    B, n = parents.shape
    i32 = torch.int32
    args = [_int32(parents, "parents", (B, n), dev), _int32(lengths, "lengths", (B,), dev)]
    with _work(dev, stream) as (st, shared):
        out = [torch.empty(s, dtype=i32, device=dev) for s in ((B, n, (n + 31) // 32), (B, n), (B, n))]
        _call("noble_tree_rows", B, n, *args, *[t.data_ptr() or None for t in out], st)
        shared(*out)
    return tuple(out)


def noble_attn_tree(q, cache, page_table, lengths, seen, depths, slopes=None, *, scale: Optional[float] = None,
                    softcap: float = 0.0, o=None, stream=None) -> torch.Tensor:
    """Attention of the nodes of each sequence's tree, its last n tokens, over the paged cache, which holds them already: q
    [B n, heads, D]; seen and depths from noble_tree_rows.  A node sees the tokens before the tree, the nodes above it and
    itself; the bias goes by the difference of positions."""
    if stream is None:
        out = _native().attn_tree(q, cache, page_table, lengths, seen, depths, slopes, scale, softcap, o)
        if _served(out, "noble_attn_tree"):
            return out[0]
    s = _Sequences(q, cache, page_table, lengths, slopes, scale, softcap)
    tree = [_int32(seen, "seen", (s.B, s.n, (s.n + 31) // 32), s.dev), _int32(depths, "depths", (s.B, s.n), s.dev)]
    n = _size("noble_attn_tree_scratch_size", ctypes.byref(s.desc))
    with _work(s.dev, stream) as (st, shared):
        o, po = s.output(o)
        scratch, ps = _buffer(n, s.dev)
        _call("noble_attn_tree", ctypes.byref(s.desc), ctypes.byref(s.q), s.cache, s.table, s.lengths, *tree, s.slopes, po,
              ps, n, st)
        shared(o)
    return o


# -------------------------------------------------------------------- keep --

def noble_cache_keep(cache, page_table, kept, start=None, *, stream=None) -> torch.Tensor:
    """Moves keys and values of token start[b] + kept[b, h, i] of key head h to the place of token start[b] + i, and returns
    the cache: kept int32 [B, kv_heads or 1, most], ascending; entries below their own i (-1 at the end) are skipped; start
    int32 [B] (None: 0).  Different sequences' pages are distinct."""
    if stream is None and _served(_native().keep(cache, page_table, kept, start), "noble_cache_keep"):
        return cache
    dev = _gpu(cache, "cache")
    if cache.dim() != 5 or cache.shape[1] != 2:
        raise ValueError("cache must be [pages, 2, kv_heads, page, head_dim]")
    K, D = cache.shape[2], cache.shape[4]
    pages, page, pc = _cache_shape(cache, K, D, cache.dtype, dev)
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be [sequences, pages]")
    B, per = page_table.shape
    if not isinstance(kept, torch.Tensor) or kept.dim() != 3 or kept.shape[0] != B or kept.shape[1] not in (1, K):
        raise ValueError("kept must be [sequences, kv_heads or 1, tokens]")
    d = noble_keep_desc(B, per, pages, kept.shape[2], page, K, D, kept.shape[1], _dtype_code(cache), 0)
    args = [pc, _int32(page_table, "page_table", (B, per), dev), _int32(kept, "kept", None, dev),
            _tensor(start, "start", torch.int32, (B,), dev)]
    with _work(dev, stream) as (st, shared):
        _call("noble_cache_keep", ctypes.byref(d), *args, st)
        shared(cache)
    return cache


# ---------------------------------------------------------- selected pages --

def noble_page_means(cache, page_table, lengths, new: int, means=None, *, stream=None) -> torch.Tensor:
    """The means of the keys of the pages that hold each sequence's last ``new`` tokens, over the tokens that it holds in
    them, into means [pages, kv_heads, D] (the cache's dtype; None: a new tensor, zeros elsewhere).  ``new`` of the longest
    sequence or more: of all its pages."""
    if stream is None and _served(_native().page_means(cache, page_table, lengths, new, means), "noble_page_means"):
        return means
    dev = _gpu(cache, "cache")
    if cache.dim() != 5 or cache.shape[1] != 2:
        raise ValueError("cache must be [pages, 2, kv_heads, page, head_dim]")
    K, D = cache.shape[2], cache.shape[4]
    pages, page, pc = _cache_shape(cache, K, D, cache.dtype, dev)
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be [sequences, pages]")
    B, per = page_table.shape
    _whole(new=new)
    d = noble_paged_desc(B, per, pages, page, new, 0, K, K, D, _dtype_code(cache), 1.0, 0.0, 0)
    args = [_int32(page_table, "page_table", (B, per), dev), _int32(lengths, "lengths", (B,), dev)]
    with _work(dev, stream) as (st, shared):
        means = torch.zeros((pages, K, D), dtype=cache.dtype, device=dev) if means is None else means
        _call("noble_page_means", ctypes.byref(d), pc, *args, _tensor(means, "means", cache.dtype, (pages, K, D), dev), st)
        shared(means)
    return means


def noble_block_select(q, means, page_table, lengths, count: int, *, page: int, sink: int = 0, local: int = 1, chosen=None,
                       stream=None) -> torch.Tensor:
    """The ``count`` blocks (pages of ``page`` tokens) of its sequence that each row of q [B n, heads, D] and key head reads:
    of those up to the row's own the first ``sink``, the last ``local`` and, of the others, those whose means [pages,
    kv_heads, D] have the largest product with the sum of the queries that share the head.  int32 [B n, kv_heads, count],
    ascending, -1 behind the last."""
    if stream is None:
        out = _native().block_select(q, means, page_table, lengths, count, page, sink, local, chosen)
        if _served(out, "noble_block_select"):
            return out[0]
    dev = _gpu(q, "q")
    if q.dim() != 3 or not isinstance(page_table, torch.Tensor) or page_table.dim() != 2 or page_table.shape[0] < 1:
        raise ValueError("q must be [rows, heads, head_dim] and page_table [sequences, pages]")
    rows, H, D = q.shape
    B, per = page_table.shape
    if rows % B or rows < B:
        raise ValueError(f"{rows} rows of q are not the same number for each of {B} sequences")
    if not isinstance(means, torch.Tensor) or means.dim() != 3:
        raise ValueError("means must be [pages, kv_heads, head_dim]")
    pages, K = means.shape[0], means.shape[1]
    _whole(count=count, page=page, sink=sink, local=local)
    d = noble_paged_desc(B, per, pages, page, rows // B, 0, H, K, D, _dtype_code(q), 1.0, 0.0, 0)
    e = noble_select_desc(count, sink, local, 0)
    args = [_heads(q, "q", q.dtype, dev), _tensor(means, "means", q.dtype, (pages, K, D), dev),
            _int32(page_table, "page_table", (B, per), dev), _int32(lengths, "lengths", (B,), dev)]
    n = _size("noble_block_select_scratch_size", ctypes.byref(d), ctypes.byref(e))
    with _work(dev, stream) as (st, shared):
        chosen = torch.empty((rows, K, count), dtype=torch.int32, device=dev) if chosen is None else chosen
        scratch, ps = _buffer(n, dev)
        _call("noble_block_select", ctypes.byref(d), ctypes.byref(e), ctypes.byref(args[0]), *args[1:],
              _int32(chosen, "chosen", (rows, K, count), dev), ps, n, st)
        shared(chosen)
    return chosen


def noble_attn_blocks(q, cache, page_table, lengths, chosen, slopes=None, *, scale: Optional[float] = None,
                      softcap: float = 0.0, o=None, stream=None) -> torch.Tensor:
    """Attention of each sequence's last tokens, q [B n, heads, D], over the blocks that ``chosen`` int32 [B n, kv_heads,
    count] lists (noble_block_select), up to the row's token.  A list ends before its first entry that is not larger than
    the one before it, negative, or past the row's own block."""
    if stream is None:
        out = _native().attn_blocks(q, cache, page_table, lengths, chosen, slopes, scale, softcap, o)
        if _served(out, "noble_attn_blocks"):
            return out[0]
    s = _Sequences(q, cache, page_table, lengths, slopes, scale, softcap)
    if not isinstance(chosen, torch.Tensor) or chosen.dim() != 3:
        raise ValueError("chosen must be [rows, kv_heads, blocks]")
    count = chosen.shape[2]
    pc = _int32(chosen, "chosen", (s.shape[0], s.K, count), s.dev)
    n = _size("noble_attn_blocks_scratch_size", ctypes.byref(s.desc), count)
    with _work(s.dev, stream) as (st, shared):
        o, po = s.output(o)
        scratch, ps = _buffer(n, s.dev)
        _call("noble_attn_blocks", ctypes.byref(s.desc), count, ctypes.byref(s.q), s.cache, s.table, s.lengths, pc, s.slopes,
              po, ps, n, st)
        shared(o)
    return o


# ---------------------------------------------------- weights and eviction --

def noble_attn_weigh(q, cache, page_table, lengths, weights=None, slopes=None, *, scale: Optional[float] = None,
                     softcap: float = 0.0, o=None, out=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(o, out): attention of each sequence's last tokens over the paged cache as noble_attn_paged's, and the weight that
    every token has received, float32 [B, kv_heads, page_table.shape[1] * page]: what ``weights`` holds for the tokens
    before the new ones (None: nothing) and the sum of the rows' probabilities.  ``out`` may be ``weights`` (None: a new
    tensor, zeros past the sequences' tokens; a given one is left as it is there)."""
    if stream is None:
        served = _native().attn_weigh(q, cache, page_table, lengths, weights, slopes, scale, softcap, o, out)
        if _served(served, "noble_attn_weigh"):
            return served
    s = _Sequences(q, cache, page_table, lengths, slopes, scale, softcap)
    shape = (s.B, s.K, s.tokens)
    pw = _tensor(weights, "weights", torch.float32, shape, s.dev)
    n = _size("noble_attn_weigh_scratch_size", ctypes.byref(s.desc))
    with _work(s.dev, stream) as (st, shared):
        o, po = s.output(o)
        out = torch.zeros(shape, device=s.dev) if out is None else out
        scratch, ps = _buffer(n, s.dev)
        _call("noble_attn_weigh", ctypes.byref(s.desc), ctypes.byref(s.q), s.cache, s.table, s.lengths, s.slopes, pw,
              _tensor(out, "out", torch.float32, shape, s.dev), po, ps, n, st)
        shared(o, out)
    return o, out


def noble_evict_select(weights, lengths, keep: int, *, sink: int = 0, recent: int = 0, kept=None, kept_weights=None,
                       stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(kept, kept_weights): the ``keep`` tokens of each sequence and key head that stay, int32 [B, heads, keep], ascending,
    -1 behind the last, and their weights (0 there).  All, if there are no more; else the first ``sink``, the last
    ``recent`` and, of the others, those with the most of weights float32 [B, heads, tokens]."""
    if stream is None:
        out = _native().evict_select(weights, lengths, keep, sink, recent, kept, kept_weights)
        if _served(out, "noble_evict_select"):
            return out
    dev = _gpu(weights, "weights")
    if weights.dim() != 3:
        raise ValueError(f"weights must be [sequences, heads, tokens], got {tuple(weights.shape)}")
    B, H, row = weights.shape
    _whole(keep=keep, sink=sink, recent=recent)
    if keep > 2 ** 31 - 4096:
        raise ValueError(f"keep={keep}, 2 ** 31 - 4096 at most")
    d = noble_evict_desc(B, row, H, keep, sink, recent)
    args = [_tensor(weights, "weights", torch.float32, None, dev), _int32(lengths, "lengths", (B,), dev)]
    with _work(dev, stream) as (st, shared):
        kept = torch.empty((B, H, keep), dtype=torch.int32, device=dev) if kept is None else kept
        kept_weights = torch.empty((B, H, keep), device=dev) if kept_weights is None else kept_weights
        _call("noble_evict_select", ctypes.byref(d), *args, _int32(kept, "kept", (B, H, keep), dev),
              _tensor(kept_weights, "kept_weights", torch.float32, (B, H, keep), dev), st)
        shared(kept, kept_weights)
    return kept, kept_weights
