"""Python binding of libnoble's attention side (include/noble_attn.h): the operators between the grouped Q/K/V layer and
the O layer of a transformer block.

The functions keep the C names and take torch tensors: ``noble_qk_rope_fwd`` / ``_bwd``, ``noble_kv_append``,
``noble_attn_fwd`` / ``_bwd``, ``noble_attn_paged``, ``noble_rope_table``, ``noble_mask_rows``.  They check their
arguments, allocate the outputs that are not given and the scratch, and enqueue all their work on ``stream`` (default:
torch's current stream), where the inputs have to be ready.  ``QKRope``, ``Attention`` and ``RopeAttention`` are the ``torch.autograd.Function`` forms, ``PagedCache``
keeps the pages of a batch of sequences, and ``NobleSelfAttention`` is the block's attention from x to the O layer's
output, for training, prompts and single tokens.

There is no fallback: without the built library or a gfx950 device, calls raise.
"""

from __future__ import annotations

import contextlib
import ctypes
import importlib.util
import os
from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import noble
from .noble import NobleError, _dtype_code, _on, _stream

_vp = ctypes.c_void_p
_i64, _i32 = ctypes.c_int64, ctypes.c_int32
_f32, _f64 = ctypes.c_float, ctypes.c_double

SCALINGS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3}


class noble_heads(ctypes.Structure):
    _fields_ = [("data", _vp), ("row", _i64), ("head", _i64)]


class noble_rope_desc(ctypes.Structure):
    _fields_ = [("T", _i64), ("x_row", _i64), ("table_rows", _i64), ("heads", _i32), ("kv_heads", _i32),
                ("head_dim", _i32), ("rot", _i32), ("interleaved", _i32), ("dtype", _i32), ("eps", _f32),
                ("reserved", _i32)]


class noble_rope_scaling(ctypes.Structure):
    _fields_ = [("kind", _i32), ("reserved", _i32), ("base", _f64), ("factor", _f64), ("trained", _f64),
                ("fast", _f64), ("slow", _f64), ("gain", _f64)]


class noble_cache_desc(ctypes.Structure):
    _fields_ = [("pages", _i64), ("page", _i32), ("reserved", _i32)]


class noble_attn_desc(ctypes.Structure):
    _fields_ = [("Tq", _i64), ("Tk", _i64), ("offset", _i64), ("heads", _i32), ("kv_heads", _i32),
                ("head_dim", _i32), ("dtype", _i32), ("causal", _i32), ("scale", _f32), ("softcap", _f32),
                ("reserved", _i32)]


class noble_paged_desc(ctypes.Structure):
    _fields_ = [("B", _i64), ("table_row", _i64), ("pages", _i64), ("page", _i32), ("new_tokens", _i32),
                ("window", _i32), ("heads", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("dtype", _i32),
                ("scale", _f32), ("softcap", _f32), ("reserved", _i32)]


_P = ctypes.POINTER
_hp = _P(noble_heads)
_sz = ctypes.c_size_t
_SIGNATURES = {
    "noble_qk_rope_fwd": [_P(noble_rope_desc)] + [_vp] * 9,
    "noble_qk_rope_scratch_size": [_P(noble_rope_desc), _P(_sz)],
    "noble_qk_rope_bwd": [_P(noble_rope_desc)] + [_vp] * 12 + [_sz, _vp],
    "noble_kv_append": [_P(noble_rope_desc), _P(noble_cache_desc)] + [_vp] * 10,
    "noble_rope_table": [_P(noble_rope_scaling), _i64, _i32, _vp, _vp, _vp],
    "noble_attn_fwd": [_P(noble_attn_desc), _hp, _hp, _hp, _vp, _vp, _vp, _hp, _vp, _vp],
    "noble_attn_bwd_scratch_size": [_P(noble_attn_desc), _P(_sz)],
    "noble_attn_bwd": [_P(noble_attn_desc), _hp, _hp, _hp, _hp, _hp, _vp, _vp, _vp, _vp, _hp, _hp, _hp, _vp, _sz, _vp],
    "noble_attn_paged_scratch_size": [_P(noble_paged_desc), _P(_sz)],
    "noble_attn_paged": [_P(noble_paged_desc), _hp, _vp, _vp, _vp, _vp, _hp, _vp, _sz, _vp],
    "noble_mask_rows": [_i64, _i64, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp],
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


BINDING_PATH = os.path.join(noble.PKG_DIR, "_noble_attn_torch.so")
_native_module = None


def _native():
    """The native calls (_noble_attn_torch.so), given the library's entry points.  They serve well-formed calls on
    ordinary tensors and the current stream and return None for any other, which the Python code then checks and runs."""
    global _native_module
    if _native_module is None:
        L = lib()
        if not os.path.exists(BINDING_PATH):
            raise RuntimeError(f"{BINDING_PATH} is missing: build it with __graft_entry__.build() "
                               "(or python -m paper_2603_06492_amd._build)")
        spec = importlib.util.spec_from_file_location("_noble_attn_torch", BINDING_PATH)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        m.init(*(ctypes.cast(getattr(L, n), _vp).value for n in (
            "noble_qk_rope_fwd", "noble_qk_rope_bwd", "noble_qk_rope_scratch_size", "noble_kv_append", "noble_attn_fwd",
            "noble_attn_bwd", "noble_attn_bwd_scratch_size", "noble_attn_paged", "noble_attn_paged_scratch_size")))
        _native_module = m
    return _native_module


def _served(out, name) -> bool:
    """Whether the native code served a call; raises for a status."""
    if isinstance(out, int):
        raise NobleError(out, name)
    return out is not None


def _call(name, *args) -> None:
    st = getattr(lib(), name)(*args)
    if st != 0:
        raise NobleError(st, name)


# ----------------------------------------------------------------- tensors --

def _tensor(t, name, dtype, shape, device):
    """Checks a dense tensor and returns its address."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call runs on {device}: all tensors must share one device")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr() or None


def _heads(t, name, dtype, device, shape=None) -> noble_heads:
    """Checks a [rows, heads, D] tensor whose elements of a head are adjacent; any row and head strides."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call runs on {device}: all tensors must share one device")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{name} must be [rows, heads, head_dim], got {tuple(t.shape)}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"{name} must have adjacent elements along head_dim, got strides {t.stride()}")
    return noble_heads(t.data_ptr() or None, t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0)


def _rows(x, name, cols) -> int:
    """Row stride of a [T, cols] tensor with adjacent columns."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if x.device.type != "cuda":
        raise ValueError(f"{name} must be on the GPU (got {x.device})")
    if x.dim() != 2 or (cols is not None and x.shape[1] != cols):
        raise ValueError(f"{name} must be [tokens, {cols}], got {tuple(x.shape)}")
    if x.shape[1] > 1 and x.stride(1) != 1:
        raise ValueError(f"{name} must have adjacent columns, got strides {x.stride()}")
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


def _gpu(t, name) -> torch.device:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on the GPU (got {t.device})")
    return t.device


@contextlib.contextmanager
def _work(device, stream):
    """Makes ``device`` and, where one is given, ``stream`` current: what a call allocates, fills or copies inside is in that
    stream's order, as its kernels are.  Yields the stream's handle, and a function for the tensors that the call returns:
    new ones come from the stream's memory and are used on the caller's own, given ones the other way round, and either's
    memory is kept for both."""
    handle = _stream(stream, device)
    if stream is None:
        with _on(device):
            yield handle, lambda *tensors: None
        return
    home = torch.cuda.current_stream(device)

    def shared(*tensors):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
                t.record_stream(home)

    with torch.cuda.stream(stream):
        yield handle, shared


def _scratch(n, device):
    return torch.empty(max(n, 16), dtype=torch.uint8, device=device)


# ------------------------------------------------------- norm and rotation --

def noble_rope_table(length: int, rot: int, *, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                     trained: float = 0.0, fast: float = 32.0, slow: float = 1.0, gain: float = 1.0, device="cuda",
                     stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """cos and sin, float32 [length, rot / 2], of the positions 0 .. length - 1.  ``scaling`` for contexts longer than
    the trained ones: "linear" (positions / factor), "base" (a larger base), "ramp" (the slow frequencies / factor,
    the fast ones kept; needs ``trained``)."""
    if scaling not in SCALINGS:
        raise ValueError(f"unknown scaling {scaling!r}; expected one of {sorted(SCALINGS)}")
    dev = torch.empty(0, device=device).device
    if dev.type != "cuda":
        raise ValueError(f"the tables live on the GPU (got {dev})")
    s = noble_rope_scaling(SCALINGS[scaling], 0, base, factor, trained, fast, slow, gain)
    with _work(dev, stream) as (st, shared):
        cos, sin = (torch.empty((max(length, 0), max(rot, 0) // 2), device=dev) for _ in range(2))
        _call("noble_rope_table", ctypes.byref(s), length, rot, cos.data_ptr() or None, sin.data_ptr() or None, st)
        shared(cos, sin)
    return cos, sin


def _rope_args(qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps, interleaved):
    """The descriptor and the addresses of x, the weights, the tables and the positions."""
    dev = _gpu(qkv, "qkv")
    groups = heads + 2 * kv_heads
    if qkv.dim() != 2 or groups < 1 or qkv.shape[1] % groups:
        raise ValueError(f"qkv must be [tokens, (heads + 2 kv_heads) head_dim], got {tuple(qkv.shape)} for {heads} and "
                         f"{kv_heads} heads")
    T, D = qkv.shape[0], qkv.shape[1] // groups
    x_row = _rows(qkv, "qkv", None)
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin must be given together")
    if (q_weight is None) != (k_weight is None):
        raise ValueError("q_weight and k_weight must be given together")
    rows, half = (0, 0) if cos is None else cos.shape if cos.dim() == 2 else (None, None)
    if rows is None:
        raise ValueError(f"cos must be [positions, rot / 2], got {tuple(cos.shape)}")
    f32 = torch.float32
    d = noble_rope_desc(T, x_row, rows, heads, kv_heads, D, 2 * half, int(interleaved), _dtype_code(qkv), eps, 0)
    return dev, d, [qkv.data_ptr() or None, _tensor(q_weight, "q_weight", f32, (D,), dev),
                    _tensor(k_weight, "k_weight", f32, (D,), dev), _tensor(cos, "cos", f32, None, dev),
                    _tensor(sin, "sin", f32, None if cos is None else tuple(cos.shape), dev),
                    _tensor(positions, "positions", torch.int32, (T,), dev)]


def noble_qk_rope_fwd(qkv, q_weight, k_weight, cos, sin, positions, *, heads: int, kv_heads: int, eps: float = 1e-6,
                      interleaved: bool = False, q=None, k=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """q [T, heads, D] and k [T, kv_heads, D] from the Q/K/V layer's rows [T, (heads + 2 kv_heads) D]: each head normed
    (weights float32 [D]; None: not) and its first 2 cos.shape[1] elements rotated by the token's position (int32 [T],
    None: the row's number; cos None: not)."""
    if stream is None:
        out = _native().rope_fwd(qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps, interleaved, q, k)
        if _served(out, "noble_qk_rope_fwd"):
            return out
    dev, d, args = _rope_args(qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps, interleaved)
    T, D = d.T, d.head_dim
    with _work(dev, stream) as (st, shared):
        q = torch.empty((T, heads, D), dtype=qkv.dtype, device=dev) if q is None else q
        k = torch.empty((T, kv_heads, D), dtype=qkv.dtype, device=dev) if k is None else k
        out = [_tensor(q, "q", qkv.dtype, (T, heads, D), dev), _tensor(k, "k", qkv.dtype, (T, kv_heads, D), dev)]
        _call("noble_qk_rope_fwd", ctypes.byref(d), *args, *out, st)
        shared(q, k)
    return q, k


def noble_qk_rope_bwd(dq, dk, qkv, q_weight, k_weight, cos, sin, positions, *, heads: int, kv_heads: int,
                      eps: float = 1e-6, interleaved: bool = False, dqkv=None, stream=None):
    """(dqkv, dq_weight, dk_weight): the query and key columns of dqkv are written, the value columns left as they are
    (zeros in a tensor allocated here).  The weights' gradients are None without weights."""
    if stream is None and dqkv is not None:
        out = _native().rope_bwd(dq, dk, qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps, interleaved,
                                 dqkv)
        if _served(out, "noble_qk_rope_bwd"):
            return dqkv, *out
    dev, d, args = _rope_args(qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps, interleaved)
    T, D = d.T, d.head_dim
    grads = [_tensor(dq, "dq", qkv.dtype, (T, heads, D), dev), _tensor(dk, "dk", qkv.dtype, (T, kv_heads, D), dev)]
    with _work(dev, stream) as (st, shared):
        if dqkv is None:
            dqkv = torch.zeros_like(qkv, memory_format=torch.contiguous_format)
        if dqkv.device != dev or dqkv.dtype != qkv.dtype or dqkv.shape != qkv.shape:
            raise ValueError("dqkv must have qkv's shape, dtype and device")
        if _rows(dqkv, "dqkv", qkv.shape[1]) != d.x_row and T > 1:
            qkv = qkv.contiguous() if dqkv.is_contiguous() else qkv
            if _rows(qkv, "qkv", None) != dqkv.stride(0):
                raise ValueError("dqkv must have qkv's row stride, or be contiguous")
            d.x_row, args[0] = dqkv.stride(0), qkv.data_ptr()
        w = [None, None] if q_weight is None else [torch.empty(D, device=dev) for _ in range(2)]
        n = _sz(0)
        _call("noble_qk_rope_scratch_size", ctypes.byref(d), ctypes.byref(n))
        scratch = _scratch(n.value if q_weight is not None else 0, dev)
        _call("noble_qk_rope_bwd", ctypes.byref(d), *grads, *args, dqkv.data_ptr() or None,
              *[None if t is None else t.data_ptr() for t in w], scratch.data_ptr(), scratch.numel(), st)
        shared(dqkv, *w)
    return dqkv, w[0], w[1]


def _cache_shape(cache, kv_heads, D, dtype, dev):
    if not isinstance(cache, torch.Tensor) or cache.dim() != 5 or cache.shape[1] != 2:
        raise ValueError("cache must be [pages, 2, kv_heads, page, head_dim]")
    pages, _, _, page, _ = cache.shape
    return pages, page, _tensor(cache, "cache", dtype, (pages, 2, kv_heads, page, D), dev)


def noble_kv_append(qkv, q_weight, k_weight, cos, sin, positions, slots, cache, *, heads: int, kv_heads: int,
                    eps: float = 1e-6, interleaved: bool = False, q=None, stream=None) -> torch.Tensor:
    """Writes each row's keys, normed and rotated, and values to its slot (int64 [T], page number x page size + place;
    outside the cache: not written) of cache [pages, 2, kv_heads, page, D], and returns the queries, normed and
    rotated."""
    if stream is None:
        out = _native().append(qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps, interleaved, slots, cache,
                               q)
        if _served(out, "noble_kv_append"):
            return out[0]
    dev, d, args = _rope_args(qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps, interleaved)
    T, D = d.T, d.head_dim
    pages, page, pc = _cache_shape(cache, kv_heads, D, qkv.dtype, dev)
    c = noble_cache_desc(pages, page, 0)
    with _work(dev, stream) as (st, shared):
        q = torch.empty((T, heads, D), dtype=qkv.dtype, device=dev) if q is None else q
        rest = [_tensor(slots, "slots", torch.int64, (T,), dev), _tensor(q, "q", qkv.dtype, (T, heads, D), dev), pc]
        _call("noble_kv_append", ctypes.byref(d), ctypes.byref(c), *args, *rest, st)
        shared(q)
    return q


# --------------------------------------------------------------- attention --

def noble_mask_rows(starts, T: int, *, prefix=None, causal: bool = True, window: int = 0, stream=None):
    """(key_lo, key_hi, positions), int32 [T], of packed documents: document n holds the rows starts[n] .. starts[n + 1]
    - 1 (int32 [documents + 1]).  A row sees its document up to itself (``causal``) or all of it, the document's first
    prefix[n] rows in any case, and with a window only that many rows, the last ones."""
    dev = _gpu(starts, "starts")
    if starts.dim() != 1 or starts.shape[0] < 1:
        raise ValueError("starts must be int32 [documents + 1]")
    n = starts.shape[0] - 1
    with _work(dev, stream) as (st, shared):
        out = [torch.empty(max(T, 0), dtype=torch.int32, device=dev) for _ in range(3)]
        _call("noble_mask_rows", T, n, _tensor(starts, "starts", torch.int32, (n + 1,), dev),
              _tensor(prefix, "prefix", torch.int32, (n,), dev), int(causal), window,
              *[t.data_ptr() or None for t in out], st)
        shared(*out)
    return tuple(out)


def _attn_args(q, k, v, key_lo, key_hi, slopes, causal, offset, scale, softcap):
    dev = _gpu(q, "q")
    code, dt = _dtype_code(q), q.dtype
    if q.dim() != 3 or not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("q, k and v must be [rows, heads, head_dim]")
    (Tq, H, D), (Tk, K, _) = q.shape, k.shape
    heads = [_heads(q, "q", dt, dev), _heads(k, "k", dt, dev, (Tk, K, D)), _heads(v, "v", dt, dev, (Tk, K, D))]
    i32 = torch.int32
    if (key_lo is None) != (key_hi is None):
        raise ValueError("key_lo and key_hi must be given together")
    mask = [_tensor(key_lo, "key_lo", i32, (Tq,), dev), _tensor(key_hi, "key_hi", i32, (Tq,), dev),
            _tensor(slopes, "slopes", torch.float32, (H,), dev)]
    d = noble_attn_desc(Tq, Tk, Tk - Tq if offset is None else offset, H, K, D, code, int(causal),
                        D ** -0.5 if scale is None else scale, softcap, 0)
    return dev, d, heads, mask


def noble_attn_fwd(q, k, v, key_lo=None, key_hi=None, slopes=None, *, causal: bool = False, offset: Optional[int] = None,
                   scale: Optional[float] = None, softcap: float = 0.0, o=None, lse=None, stream=None):
    """(o, lse) of attention of q [Tq, heads, D] over k, v [Tk, kv_heads, D] (any row and head strides): row i sees the
    keys [key_lo[i], key_hi[i]) (int32; None: all), with ``causal`` only those up to i + offset (default: the last row
    sees the last key).  Scores are scale q.k (default D^-1/2), capped by softcap tanh(. / softcap) and lowered by
    slopes[head] |i + offset - j|.  o: like q, dense; lse: float32 [heads, Tq]."""
    if stream is None:
        out = _native().attn_fwd(q, k, v, key_lo, key_hi, slopes, causal, offset, scale, softcap, o, lse)
        if _served(out, "noble_attn_fwd"):
            return out
    dev, d, heads, mask = _attn_args(q, k, v, key_lo, key_hi, slopes, causal, offset, scale, softcap)
    shape = tuple(q.shape)
    with _work(dev, stream) as (st, shared):
        o = torch.empty(shape, dtype=q.dtype, device=dev) if o is None else o
        lse = torch.empty(shape[1::-1], device=dev) if lse is None else lse
        _call("noble_attn_fwd", ctypes.byref(d), *map(ctypes.byref, heads), *mask,
              ctypes.byref(_heads(o, "o", q.dtype, dev, shape)), _tensor(lse, "lse", torch.float32, shape[1::-1], dev), st)
        shared(o, lse)
    return o, lse


def noble_attn_bwd(do, q, k, v, o, lse, key_lo=None, key_hi=None, slopes=None, *, causal: bool = False,
                   offset: Optional[int] = None, scale: Optional[float] = None, softcap: float = 0.0, dq=None, dk=None,
                   dv=None, stream=None):
    """(dq, dk, dv) for the upstream gradient ``do`` of noble_attn_fwd's o, with the same inputs and its o and lse."""
    if stream is None:
        out = _native().attn_bwd(do, o, lse, q, k, v, key_lo, key_hi, slopes, causal, offset, scale, softcap, dq, dk, dv)
        if _served(out, "noble_attn_bwd"):
            return out
    dev, d, heads, mask = _attn_args(q, k, v, key_lo, key_hi, slopes, causal, offset, scale, softcap)
    dt, sq, sk = q.dtype, tuple(q.shape), tuple(k.shape)
    g, oo = _heads(do, "do", dt, dev, sq), _heads(o, "o", dt, dev, sq)
    n = _sz(0)
    _call("noble_attn_bwd_scratch_size", ctypes.byref(d), ctypes.byref(n))
    with _work(dev, stream) as (st, shared):
        dq, dk, dv = (torch.empty(s, dtype=dt, device=dev) if t is None else t for t, s in ((dq, sq), (dk, sk), (dv, sk)))
        outs = [_heads(t, n, dt, dev, s) for t, n, s in ((dq, "dq", sq), (dk, "dk", sk), (dv, "dv", sk))]
        scratch = _scratch(n.value, dev)
        _call("noble_attn_bwd", ctypes.byref(d), ctypes.byref(g), *map(ctypes.byref, heads), ctypes.byref(oo),
              _tensor(lse, "lse", torch.float32, sq[1::-1], dev), *mask, *map(ctypes.byref, outs), scratch.data_ptr(),
              scratch.numel(), st)
        shared(dq, dk, dv)
    return dq, dk, dv


def noble_attn_paged(q, cache, page_table, lengths, slopes=None, *, scale: Optional[float] = None, softcap: float = 0.0,
                     window: int = 0, o=None, stream=None) -> torch.Tensor:
    """Attention of each sequence's last tokens over the paged cache, which holds them already: q [B n, heads, D], n rows
    a sequence; page_table int32 [B, pages of a sequence], lengths int32 [B] (the tokens held).  The row of token t
    sees the tokens 0 .. t, with a window only its last ``window``."""
    if stream is None:
        out = _native().paged(q, cache, page_table, lengths, slopes, scale, softcap, window, o)
        if _served(out, "noble_attn_paged"):
            return out[0]
    dev = _gpu(q, "q")
    if q.dim() != 3 or not isinstance(page_table, torch.Tensor) or page_table.dim() != 2 or page_table.shape[0] < 1:
        raise ValueError("q must be [rows, heads, head_dim] and page_table [sequences, pages]")
    rows, H, D = q.shape
    B, per = page_table.shape
    if rows % B or rows < B:
        raise ValueError(f"{rows} rows of q are not the same number for each of {B} sequences")
    K = cache.shape[2] if isinstance(cache, torch.Tensor) and cache.dim() == 5 else 0
    pages, page, pc = _cache_shape(cache, K, D, q.dtype, dev)
    i32 = torch.int32
    d = noble_paged_desc(B, per, pages, page, rows // B, window, H, K, D, _dtype_code(q),
                         D ** -0.5 if scale is None else scale, softcap, 0)
    n = _sz(0)
    _call("noble_attn_paged_scratch_size", ctypes.byref(d), ctypes.byref(n))
    with _work(dev, stream) as (st, shared):
        o = torch.empty((rows, H, D), dtype=q.dtype, device=dev) if o is None else o
        scratch = _scratch(n.value, dev) if n.value else None
        _call("noble_attn_paged", ctypes.byref(d), ctypes.byref(_heads(q, "q", q.dtype, dev)), pc,
              _tensor(page_table, "page_table", i32, (B, per), dev), _tensor(lengths, "lengths", i32, (B,), dev),
              _tensor(slopes, "slopes", torch.float32, (H,), dev),
              ctypes.byref(_heads(o, "o", q.dtype, dev, (rows, H, D))),
              None if scratch is None else scratch.data_ptr(), n.value, st)
        shared(o)
    return o


# ---------------------------------------------------------------- autograd --

class QKRope(torch.autograd.Function):
    """``noble_qk_rope_fwd`` and ``_bwd``: apply(qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps,
    interleaved) -> (q, k)."""

    @staticmethod
    def forward(ctx, qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps=1e-6, interleaved=False):
        ctx.how = dict(heads=heads, kv_heads=kv_heads, eps=eps, interleaved=interleaved)
        ctx.save_for_backward(qkv, q_weight, k_weight, cos, sin, positions)
        return noble_qk_rope_fwd(qkv, q_weight, k_weight, cos, sin, positions, **ctx.how)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        dqkv, dqw, dkw = noble_qk_rope_bwd(dq.contiguous(), dk.contiguous(), *ctx.saved_tensors, **ctx.how)
        return (dqkv, dqw, dkw) + (None,) * 7


class Attention(torch.autograd.Function):
    """``noble_attn_fwd`` and ``_bwd``: apply(q, k, v, key_lo, key_hi, slopes, causal, scale, softcap) -> o.  The mask and
    the slopes are constants."""

    @staticmethod
    def forward(ctx, q, k, v, key_lo=None, key_hi=None, slopes=None, causal=False, scale=None, softcap=0.0):
        ctx.how = dict(causal=causal, scale=scale, softcap=softcap)
        o, lse = noble_attn_fwd(q, k, v, key_lo, key_hi, slopes, **ctx.how)
        ctx.save_for_backward(q, k, v, o, lse, key_lo, key_hi, slopes)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        return noble_attn_bwd(do.contiguous(), *ctx.saved_tensors, **ctx.how) + (None,) * 6


class RopeAttention(torch.autograd.Function):
    """From the Q/K/V layer's rows to the O layer's: norm, rotation and attention, apply(qkv, q_weight, k_weight, cos, sin,
    positions, key_lo, key_hi, slopes, heads, kv_heads, eps, interleaved, causal, scale, softcap) -> o [T, heads, D].  The
    backward writes every part of dqkv in place, the values' by the attention, the others' by the rotation."""

    @staticmethod
    def forward(ctx, qkv, q_weight, k_weight, cos, sin, positions, key_lo, key_hi, slopes, heads, kv_heads, eps=1e-6,
                interleaved=False, causal=False, scale=None, softcap=0.0):
        ctx.rope = dict(heads=heads, kv_heads=kv_heads, eps=eps, interleaved=interleaved)
        ctx.attn = dict(causal=causal, scale=scale, softcap=softcap)
        q, k = noble_qk_rope_fwd(qkv, q_weight, k_weight, cos, sin, positions, **ctx.rope)
        o, lse = noble_attn_fwd(q, k, _values(qkv, k), key_lo, key_hi, slopes, **ctx.attn)
        ctx.save_for_backward(qkv, q_weight, k_weight, cos, sin, positions, q, k, o, lse, key_lo, key_hi, slopes)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        qkv, q_weight, k_weight, cos, sin, positions, q, k, o, lse, *mask = ctx.saved_tensors
        dqkv = torch.empty_like(qkv)
        dq, dk, _ = noble_attn_bwd(do.contiguous(), q, k, _values(qkv, k), o, lse, *mask, dv=_values(dqkv, k), **ctx.attn)
        _, dqw, dkw = noble_qk_rope_bwd(dq, dk, qkv, q_weight, k_weight, cos, sin, positions, dqkv=dqkv, **ctx.rope)
        return (dqkv, dqw, dkw) + (None,) * 13


def _values(qkv, k):
    """The value columns of Q/K/V rows as [T, kv_heads, D]."""
    T, K, D = k.shape
    return qkv[:, qkv.shape[1] - K * D:].view(T, K, D)


# ------------------------------------------------------------- paged cache --

class PagedCache:
    """Keys and values of a batch of sequences in pages of ``page`` tokens, for ``layers`` layers that share one page table
    (``data[layer]`` is [pages, 2, kv_heads, page, head_dim]).  Which page belongs to which sequence is kept here.

    ``means``: also the means of every page's keys (``means[layer]``), by which ``NobleSelfAttention.step`` selects pages.
    ``weights``: also the attention weight that every token has received from the tokens that were not drafted
    (``weights[layer]``, float32 [sequences, kv_heads, tokens]), by which ``evict`` goes.  A step over such a cache takes 4 bytes
    of scratch for each new token, query head and token of ``longest``: long prompts go in in parts."""

    def __init__(self, sequences: int, longest: int, pages: int, *, kv_heads: int, head_dim: int, page: int = 16,
                 layers: int = 1, dtype=torch.bfloat16, device="cuda", means: bool = False, weights: bool = False):
        per = -(-longest // page)
        self.page, self.longest = page, longest
        self.data = [torch.empty((pages, 2, kv_heads, page, head_dim), dtype=dtype, device=device) for _ in range(layers)]
        self.page_table = torch.full((sequences, per), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        new = lambda keep, *shape, **kw: [torch.zeros(*shape, device=device, **kw) for _ in range(layers)] if keep else None  # noqa: E731
        self.means = new(means, (pages, kv_heads, head_dim), dtype=dtype)
        self.weights = new(weights, (sequences, kv_heads, per * page))
        self._table = [[] for _ in range(sequences)]
        self._held = [0] * sequences
        self._seen = [0] * sequences   # tokens that the sequence has had, evicted ones among them
        self._free = list(range(pages - 1, -1, -1))
        self._drafted, self._parents = 0, None

    def _room(self, new: int):
        """Pages for ``new`` more tokens of every sequence, and their slots."""
        if new < 0:
            raise ValueError(f"{new} new tokens")
        if self._drafted:
            raise RuntimeError("a draft is in the cache: accept what is to stay of it first")
        if max(self._held) + new > self.longest:
            raise ValueError(f"sequences of up to {self.longest} tokens: {max(self._held)} held, {new} more")
        need = [-(-(n + new) // self.page) - len(t) for n, t in zip(self._held, self._table)]
        if sum(need) > len(self._free):
            raise MemoryError(f"{sum(need)} more pages needed, {len(self._free)} free")
        slots = []
        for b, pages in enumerate(self._table):
            pages += [self._free.pop() for _ in range(need[b])]
            slots += [pages[t // self.page] * self.page + t % self.page for t in range(self._held[b], self._held[b] + new)]
            self._held[b] += new
            self._seen[b] += new
        if any(need):
            self._write_table()
        self.lengths += new
        return torch.tensor(slots, dtype=torch.int64, device=self.lengths.device)

    def _write_table(self) -> None:
        per = self.page_table.shape[1]
        self.page_table.copy_(torch.tensor([p + [-1] * (per - len(p)) for p in self._table], dtype=torch.int32))

    def extend(self, new: int):
        """Room for ``new`` more tokens of every sequence: (positions int32, slots int64), both [sequences * new], a
        sequence's tokens in a row.  Raises MemoryError when the pages run out and ValueError past ``longest``; nothing has
        changed then."""
        slots = self._room(new)
        positions = [t for n in self._seen for t in range(n - new, n)]
        return torch.tensor(positions, dtype=torch.int32, device=slots.device), slots

    def draft(self, parents):
        """Room for a tree of n drafted tokens of every sequence, parents int32 [sequences, n] as noble_tree_rows takes them:
        (positions, slots, tree), for ``NobleSelfAttention.step(..., tree=tree)`` in every layer.  ``accept`` says which of
        them stay, before anything else is put into the cache.  Raises as ``extend`` does."""
        from . import decoding
        parents = parents.to(device=self.lengths.device, dtype=torch.int32).contiguous()
        if parents.dim() != 2 or parents.shape[0] != len(self._held) or not 1 <= parents.shape[1] <= decoding.TREE_MOST:
            raise ValueError(f"parents must be [{len(self._held)} sequences, 1 to {decoding.TREE_MOST} nodes], got "
                             f"{tuple(parents.shape)}")
        slots = self._room(parents.shape[1])
        self._drafted, self._parents = parents.shape[1], parents.clone()
        seen, depths, positions = decoding.noble_tree_rows(parents, self.lengths)
        gone = [s - n for s, n in zip(self._seen, self._held)]
        if any(gone):
            positions += torch.tensor(gone, dtype=torch.int32, device=slots.device)[:, None]
        return positions.view(-1), slots, (seen, depths)

    def accept(self, kept) -> None:
        """Of the drafted tree only the nodes kept[b] stay in sequence b, one after the other; the pages of the others are
        given back.  kept[b] is a branch: a list of node numbers whose first has the parent -1 and each other the one before it,
        or empty.  Raises ValueError for any other list; nothing has changed then."""
        from . import decoding
        n = self._drafted
        if not n:
            raise RuntimeError("no draft is in the cache")
        if len(kept) != len(self._held) or any(x < 0 or x >= n or (i and x <= k[i - 1]) for k in kept for i, x in enumerate(k)):
            raise ValueError(f"kept must be {len(self._held)} lists of ascending numbers below {n}")
        for b, (k, parents) in enumerate(zip(kept, self._parents.tolist())):
            if any(parents[x] != above for above, x in zip([-1, *k], k)):   # its key stands at another place than it would have
                raise ValueError(f"kept[{b}]={list(k)} is no branch of the tree with the parents {parents}")
        start = [h - n for h in self._held]
        table = torch.tensor([[list(k) + [-1] * (n - len(k))] for k in kept], dtype=torch.int32, device=self.lengths.device)
        first = torch.tensor(start, dtype=torch.int32, device=self.lengths.device)
        for data in self.data:
            decoding.noble_cache_keep(data, self.page_table, table, first)
        for w in self.weights or ():   # they have received nothing yet
            for b, k in enumerate(kept):
                w[b, :, start[b]:start[b] + len(k)] = 0
        self._drafted, self._parents = 0, None
        self._seen = [s - n + len(k) for s, k in zip(self._seen, kept)]
        self._cut([s + len(k) for s, k in zip(start, kept)], n)

    def evict(self, keep: int, *, sink: int = 0, recent: int = 0) -> None:
        """Of every sequence with more than ``keep`` tokens, each layer and key head keeps that many: the first ``sink``, the
        last ``recent`` and, of the others, those that have received the most attention weight (``weights``), in their order.
        Later tokens' positions go on from all the sequence has had; a window and the distance bias count the tokens that
        are left."""
        from . import decoding
        if self.weights is None:
            raise ValueError("a cache without weights")
        if self._drafted:
            raise RuntimeError("a draft is in the cache: accept what is to stay of it first")
        if keep < 1 or sink < 0 or recent < 0 or sink + recent > keep:
            raise ValueError(f"keep={keep} tokens, the first {sink} and the last {recent} among them")
        if max(self._held) <= keep:
            return
        for data, weights in zip(self.data, self.weights):
            kept, left = decoding.noble_evict_select(weights, self.lengths, keep, sink=sink, recent=recent)
            decoding.noble_cache_keep(data, self.page_table, kept)
            weights[:, :, :keep] = left
        self._cut([min(h, keep) for h in self._held], keep)

    def _cut(self, held, changed: int) -> None:
        """The sequences hold so many tokens from now on, of which the last ``changed`` have other places than before."""
        from . import decoding
        for b, n in enumerate(held):
            used = -(-n // self.page)
            self._free += reversed(self._table[b][used:])
            del self._table[b][used:]
        self._held = held
        self._write_table()
        self.lengths.copy_(torch.tensor(held, dtype=torch.int32))
        for data, means in zip(self.data, self.means or ()):
            decoding.noble_page_means(data, self.page_table, self.lengths, changed, means)

    @property
    def held(self) -> int:
        """Tokens of the sequence that holds the most."""
        return max(self._held, default=0)

    @property
    def seen(self) -> int:
        """Tokens that the longest sequence has had, evicted ones among them."""
        return max(self._seen, default=0)

    def release(self, sequence: int) -> None:
        """Gives a sequence's pages back; it holds no tokens then."""
        if self._drafted:
            raise RuntimeError("a draft is in the cache: accept what is to stay of it first")
        self._free += reversed(self._table[sequence])
        self._table[sequence], self._held[sequence], self._seen[sequence] = [], 0, 0
        self.page_table[sequence] = -1
        self.lengths[sequence] = 0


# ------------------------------------------------------------------ module --

class NobleSelfAttention(torch.nn.Module):
    """The attention half of a transformer block: a NOBLE layer for Q, K and V (one call, a branch for each where the
    widths allow it), norm and rotation of the heads, attention, and a NOBLE layer for O.  Parameters and initialisation
    of the two layers are NobleLinear's; the norms' weights are float32 ones.

    ``forward`` takes packed rows or a batch and trains; ``step`` serves prompts and single tokens from a PagedCache.
    Positions are rotated up to ``longest`` tokens; longer sequences are refused (in packed rows, whose lengths only the
    device knows, their later tokens come out as NaN)."""

    def __init__(self, d: int, heads: int, r: int, *, kv_heads: Optional[int] = None, head_dim: Optional[int] = None,
                 rot: Optional[int] = None, base: float = 10000.0, longest: int = 2048, scaling: Optional[dict] = None,
                 norm: bool = True, eps: float = 1e-6, interleaved: bool = False, softcap: float = 0.0, alibi: bool = False,
                 dtype=torch.bfloat16, device="cuda", seed: int = 0, **layer):
        super().__init__()
        self.heads, self.kv_heads = heads, heads if kv_heads is None else kv_heads
        self.head_dim = d // heads if head_dim is None else head_dim
        self.softcap, self.longest = softcap, longest
        self.how = dict(heads=self.heads, kv_heads=self.kv_heads, eps=eps, interleaved=interleaved)
        D = self.head_dim
        self.qkv = noble.NobleLinear(d, (self.heads + 2 * self.kv_heads) * D, r, dtype=dtype, device=device, seed=seed,
                                     groups=3 if self.heads == self.kv_heads and r else 1, **layer)
        self.out = noble.NobleLinear(self.heads * D, d, r, dtype=dtype, device=device, seed=seed + 1, **layer)
        ones = lambda: torch.nn.Parameter(torch.ones(D, device=device)) if norm else None  # noqa: E731
        self.q_weight, self.k_weight = ones(), ones()
        rot = D // 16 * 16 if rot is None else rot
        cos, sin = noble_rope_table(longest, rot, base=base, device=device, **(scaling or {})) if rot else (None, None)
        self.register_buffer("cos", cos, persistent=False)
        self.register_buffer("sin", sin, persistent=False)
        slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], device=device) if alibi else None
        self.register_buffer("slopes", slopes, persistent=False)

    def mask(self, starts, T: int, prefix=None, causal: bool = True, window: int = 0):
        """The mask of packed rows, for every layer and step over them: noble_mask_rows."""
        return noble_mask_rows(starts, T, prefix=prefix, causal=causal, window=window)

    def _fits(self, tokens: int) -> None:
        if self.cos is not None and tokens > self.longest:
            raise ValueError(f"a sequence of {tokens} tokens, the positions' tables hold longest={self.longest}")

    def forward(self, x, mask=None, causal: bool = True):
        """x [T, d] (one sequence, or packed documents with their ``mask``) or [B, S, d]."""
        shape = x.shape
        x = x.reshape(-1, shape[-1])
        T = x.shape[0]
        if mask is None:
            S = shape[-2]
            self._fits(S)
            mask = self.mask(torch.arange(0, T + 1, max(S, 1), dtype=torch.int32, device=x.device), T, causal=causal)
        key_lo, key_hi, positions = mask
        o = RopeAttention.apply(self.qkv(x), self.q_weight, self.k_weight, self.cos, self.sin, positions, key_lo, key_hi,
                                self.slopes, self.heads, self.kv_heads, self.how["eps"], self.how["interleaved"], False,
                                None, self.softcap)
        return self.out(o.reshape(T, -1)).reshape(shape)

    @torch.no_grad()
    def step(self, x, cache: PagedCache, positions, slots, layer: int = 0, window: int = 0, *, tree=None, blocks: int = 0,
             sink: int = 0, local: int = 1):
        """The newest tokens of every sequence, x [sequences * new, d], with the positions and slots that
        ``cache.extend(new)`` gave: their keys and values go into the cache, their attention runs over it.  A whole prompt
        is a step too.  A token sees those up to itself, with a ``window`` (the one that ``mask`` took for training) only
        that many; a mask with a prefix or without ``causal`` has no such form: feed its tokens to ``forward``.

        ``tree``: the tokens are drafted ones, from ``cache.draft(parents)``, and see the nodes above them.  ``blocks``: each
        token and key head sees that many pages of its sequence, the first ``sink``, the last ``local`` and those whose means
        (of a cache with ``means``) its queries favour.  With a cache that keeps ``weights`` the weight that every token
        receives is added up, but for a tree's step, which adds none, its accepted nodes' rows neither: over such a cache
        ``evict`` goes by the tokens of the other steps alone.  These go one at a time, and without a window."""
        from . import decoding
        self._fits(cache.seen)
        new = x.shape[0] // max(cache.lengths.shape[0], 1)
        forms = [name for name, on in (("tree", tree is not None), ("blocks", blocks), ("weights", cache.weights is not None and
                                                                                       tree is None)) if on]
        if len(forms) > 1 or (forms and window):
            raise ValueError(f"{' and '.join(forms + ['window'] * bool(window))} in one step")
        if blocks and cache.means is None:
            raise ValueError("blocks are selected by a cache's means: PagedCache(..., means=True)")
        data, held = cache.data[layer], (cache.data[layer], cache.page_table, cache.lengths)
        q = noble_kv_append(self.qkv(x), self.q_weight, self.k_weight, self.cos, self.sin, positions, slots, data, **self.how)
        how = dict(softcap=self.softcap)
        if tree is not None:
            o = decoding.noble_attn_tree(q, *held, *tree, self.slopes, **how)
            return self.out(o.reshape(x.shape[0], -1))
        if cache.means is not None and new:
            decoding.noble_page_means(*held, new, cache.means[layer])
        if blocks:
            chosen = decoding.noble_block_select(q, cache.means[layer], *held[1:], blocks, page=cache.page, sink=sink, local=local)
            o = decoding.noble_attn_blocks(q, *held, chosen, self.slopes, **how)
        elif cache.weights is not None:
            o, _ = decoding.noble_attn_weigh(q, *held, cache.weights[layer], self.slopes, out=cache.weights[layer], **how)
        else:
            o = noble_attn_paged(q, *held, self.slopes, window=window, **how)
        return self.out(o.reshape(x.shape[0], -1))

    def param_groups(self, lr):
        """Optimizer parameter groups: the two layers' learning-rate multipliers, the base rate for the norms."""
        groups = self.qkv.param_groups(lr) + self.out.param_groups(lr)
        return groups + ([{"params": [self.q_weight, self.k_weight], "lr": lr}] if self.q_weight is not None else [])
