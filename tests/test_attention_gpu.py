"""The attention operators on the GPU against plain float64 forms: forward and gradients over lengths, masks, head
layouts, strides and types; the norm and rotation; the paged cache; refusals."""

import math

import pytest
import torch

from _attention import attention, check, close, dense_mask, heads_norm_rope
from paper_2603_06492_amd import attention as na
from paper_2603_06492_amd import noble

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(g, shape, dt=F32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dt)


def _intervals(kind, Tq, Tk):
    """Key intervals on the CPU (None: none), as the mask's name says."""
    i = torch.arange(Tq, dtype=torch.int32)
    at = i + (Tk - Tq)
    if kind in ("full", "causal"):
        return None, None
    if kind == "docs":   # documents of growing length, the last tenth of the rows in none
        n = max(1, Tk // 7)
        lo = at // n * n
        hi = at + 1
        lo, hi = (torch.where(i < Tq - Tq // 10, t, 0) for t in (lo, hi))
    elif kind == "prefix":
        lo, hi = torch.zeros_like(i), torch.clamp(at + 1, min=Tk // 3)
    elif kind == "window":
        lo, hi = torch.clamp(at - 40, min=0), at + 1
    elif kind == "ragged":   # no order at all, empty rows and intervals beyond the keys among them
        g = torch.Generator().manual_seed(Tq * 31 + Tk)
        lo = torch.randint(-5, Tk + 5, (Tq,), generator=g, dtype=torch.int32)
        hi = lo + torch.randint(-3, Tk + 5, (Tq,), generator=g, dtype=torch.int32)
    elif kind == "none":
        lo, hi = torch.zeros_like(i), torch.zeros_like(i)
    return lo.to(torch.int32).contiguous(), hi.to(torch.int32).contiguous()


def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda")


CASES = [
    # Tq, Tk, heads, kv_heads, D, mask, dtype, softcap, bias
    (1, 1, 1, 1, 64, "full", BF, 0.0, False),
    (1, 300, 4, 2, 128, "causal", BF, 0.0, True),
    (2, 3, 2, 1, 8, "causal", BF, 20.0, False),
    (31, 31, 2, 2, 128, "causal", BF, 0.0, False),
    (33, 65, 4, 1, 64, "causal", BF, 30.0, True),
    (64, 64, 1, 1, 72, "full", BF, 0.0, False),
    (127, 129, 2, 1, 96, "window", BF, 0.0, False),
    (129, 127, 2, 2, 128, "causal", BF, 0.0, False),   # the first rows see nothing
    (197, 197, 3, 3, 64, "full", BF, 0.0, False),
    (300, 300, 8, 2, 128, "docs", BF, 50.0, True),
    (333, 333, 4, 4, 80, "prefix", BF, 0.0, True),
    (260, 400, 6, 2, 128, "ragged", BF, 0.0, False),
    (520, 520, 2, 1, 128, "ragged", BF, 15.0, False),
    (70, 70, 2, 2, 64, "none", BF, 0.0, False),
    (1100, 1100, 2, 1, 128, "docs", BF, 0.0, False),
    # enough workgroups of 128 rows for the form with its own rows for each wave
    (300, 300, 96, 96, 128, "causal", BF, 0.0, False),
    (260, 290, 96, 96, 64, "ragged", BF, 20.0, True),
    (333, 333, 160, 80, 128, "docs", BF, 50.0, False),
    (170, 170, 120, 120, 96, "prefix", BF, 0.0, True),
    (150, 150, 128, 128, 40, "window", BF, 0.0, False),
    (257, 257, 96, 96, 128, "none", BF, 0.0, False),
    (1, 1, 1, 1, 128, "full", F32, 0.0, False),
    (5, 200, 4, 2, 64, "causal", F32, 0.0, True),
    (65, 65, 2, 1, 128, "docs", F32, 25.0, True),
    (197, 130, 3, 1, 40, "ragged", F32, 0.0, False),
    (260, 260, 2, 2, 128, "prefix", F32, 0.0, False),
    (300, 300, 4, 1, 64, "window", F32, 30.0, False),
]


def _run(q, k, v, do, lo, hi, slopes, **kw):
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    o, lse = na.noble_attn_fwd(q, k, v, dev(lo), dev(hi), slopes, **kw)
    dq, dk, dv = na.noble_attn_bwd(do, q, k, v, o, lse, dev(lo), dev(hi), slopes, **kw)
    torch.cuda.synchronize()
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_attention(c):
    Tq, Tk, H, K, D, mask, dt, cap, bias = c
    print(f"[attn] {c}", flush=True)
    g = _gen(Tq * 7 + Tk)
    q, k, v, do = (_rand(g, s, dt) for s in ((Tq, H, D), (Tk, K, D), (Tk, K, D), (Tq, H, D)))
    lo, hi = _intervals(mask, Tq, Tk)
    slopes = _slopes(H) if bias else None
    got = _run(q, k, v, do, lo, hi, slopes, causal=mask == "causal", softcap=cap)
    want = attention(q, k, v, dense_mask(Tq, Tk, lo, hi, mask == "causal"), softcap=cap, slopes=slopes, do=do)
    for n in got:
        check(n, got[n], want[n], dt)


# the last: workgroups of 128 rows
STRIDED = pytest.mark.parametrize("dt,H,K,D", [(BF, 4, 2, 64), (F32, 4, 2, 64), (BF, 96, 96, 64), (BF, 96, 96, 128)],
                                  ids=["bf16", "f32", "bf16_wide64", "bf16_wide128"])


@STRIDED
def test_strides_and_broadcasts(dt, H, K, D):
    """q, k, v as columns of one buffer, heads outermost, and keys shared by expansion; gradients into columns of one
    buffer, whose other columns stay."""
    T = 150
    print(f"[attn] strides {dt} {H} {K} {D}", flush=True)
    g = _gen(3)
    qkv = _rand(g, (T, (H + 2 * K) * D + 32), dt)
    q, k, v = (qkv[:, a * D:b * D].view(T, b - a, D) for a, b in ((0, H), (H, H + K), (H + K, H + 2 * K)))
    do = _rand(g, (H, T, D), dt).transpose(0, 1)
    want = attention(q, k, v, dense_mask(T, T, causal=True), do=do)
    o = torch.full((H, T, D), math.nan, dtype=dt, device="cuda").transpose(0, 1)
    dqkv = torch.full_like(qkv, 7.0)
    dq, dk, dv = (dqkv[:, a * D:b * D].view(T, b - a, D) for a, b in ((0, H), (H, H + K), (H + K, H + 2 * K)))
    _, lse = na.noble_attn_fwd(q, k, v, causal=True, o=o)
    na.noble_attn_bwd(do, q, k, v, o, lse, causal=True, dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    for n, t in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(n, t, want[n], dt)
    assert bool((dqkv[:, (H + 2 * K) * D:] == 7.0).all())
    # one key head for all query heads, by expansion
    k1, v1 = (t[:, :1].expand(T, H, D) for t in (k, v))
    o2, lse2 = na.noble_attn_fwd(q, k1, v1, causal=True)
    want2 = attention(q, k1, v1, dense_mask(T, T, causal=True))
    check("o", o2, want2["o"], dt)
    check("lse", lse2, want2["lse"], dt)


def test_gradient_against_differences():
    """Float32 gradients against central differences of the kernels' own forward, along random directions: with steps
    of 1e-2 the difference's own error is about h^2 |third derivative| + 1e-6 / h of a sum of order one."""
    T, H, K, D = 40, 4, 2, 32
    g = _gen(9)
    x = [_rand(g, s) for s in ((T, H, D), (T, K, D), (T, K, D))]
    do, slopes = _rand(g, (T, H, D)), _slopes(H)
    lo, hi = (t.cuda() for t in _intervals("prefix", T, T))
    kw = dict(softcap=8.0)
    f = lambda y: float((na.noble_attn_fwd(*y, lo, hi, slopes, **kw)[0].double() * do.double()).sum())  # noqa: E731
    o, lse = na.noble_attn_fwd(*x, lo, hi, slopes, **kw)
    grads = na.noble_attn_bwd(do, *x, o, lse, lo, hi, slopes, **kw)
    for n in range(3):
        d = _rand(g, x[n].shape)
        d /= d.norm()
        h = 1e-2
        num = (f([t + h * d if i == n else t for i, t in enumerate(x)]) -
               f([t - h * d if i == n else t for i, t in enumerate(x)])) / (2 * h)
        ana = float((grads[n].double() * d.double()).sum())
        assert abs(num - ana) <= 2e-3 * max(1.0, float(grads[n].norm())), (n, num, ana)


@pytest.mark.parametrize("H,K", [(4, 2), (64, 32)])
def test_repeated_backward_is_bitwise_equal(H, K):
    T, D = 700, 128
    g = _gen(5)
    q, k, v, do = (_rand(g, s, BF) for s in ((T, H, D), (T, K, D), (T, K, D), (T, H, D)))
    lo, hi = _intervals("docs", T, T)
    a = _run(q, k, v, do, lo, hi, None)
    for _ in range(2):
        b = _run(q, k, v, do, lo, hi, None)
        assert all(bool((a[n] == b[n]).all()) for n in a)


@pytest.mark.parametrize("dt,H,K,D,T", [(BF, 96, 48, 128, 300), (BF, 192, 64, 64, 260), (BF, 8, 1, 128, 200),
                                        (BF, 12, 2, 40, 131), (F32, 6, 1, 72, 97), (F32, 24, 8, 64, 150)])
def test_heads_dealt_to_parts(dt, H, K, D, T):
    """Few key heads with several query heads each: their gradients are summed over parts of the query heads.  Twice the
    same bits, and an infinite value in one row reaches the keys that the row sees."""
    print(f"[attn] parts {dt} {H} {K} {D} {T}", flush=True)
    g = _gen(T + H)
    q, k, v, do = (_rand(g, (T, n, D), dt) for n in (H, K, K, H))
    lo, hi = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*[(0, 60) if i < 60 else (60, T) for i in range(T)]))
    slopes = _slopes(H)
    got = _run(q, k, v, do, lo, hi, slopes, causal=True, offset=0)
    seen = dense_mask(T, T, lo.cpu(), hi.cpu(), causal=True)
    want = attention(q, k, v, seen, slopes=slopes, do=do)
    for name in ("o", "lse", "dq", "dk", "dv"):
        check(name, got[name], want[name], dt)
    for name, x in _run(q, k, v, do, lo, hi, slopes, causal=True, offset=0).items():
        assert torch.equal(x, got[name]), name
    do[80, H - 1, 3] = math.inf
    bad = _run(q, k, v, do, lo, hi, slopes, causal=True, offset=0)
    rest = torch.ones(T, dtype=torch.bool)
    rest[60:81] = False
    for name in ("dk", "dv"):
        assert torch.equal(bad[name][:, :K - 1], got[name][:, :K - 1])   # the other key heads
        check(name, bad[name].cpu()[rest], [t[rest] for t in want[name]], dt)
    assert not bad["dv"][60:81, K - 1, 3].isfinite().any()


def test_large_scores():
    """Scores of some hundreds: the softmax stays in range and rows take one key nearly alone."""
    T, H, D = 200, 2, 64
    g = _gen(6)
    q, k, v, do = (_rand(g, (T, H, D), BF, s) for s in (12.0, 12.0, 1.0, 1.0))
    got = _run(q, k, v, do, None, None, None, causal=True)
    want = attention(q, k, v, dense_mask(T, T, causal=True), do=do)
    check("o", got["o"], want["o"], BF)
    check("lse", got["lse"], want["lse"], BF)


@STRIDED
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, True)])
def test_unseen_infinities_and_nan(dt, H, K, D, cap, bias):
    """Rows of no document, and one document, hold infinities and NaN in every input: the other documents' results are
    those of clean inputs, an empty row's are zero, and the one that sees them is not finite."""
    T = 300
    print(f"[attn] nan {dt} {H} {K} {D} {cap} {bias}", flush=True)
    g = _gen(11)
    starts = torch.tensor([3, 60, 61, 130, 131, 290], dtype=torch.int32, device="cuda")   # document 3 is row 130 alone
    lo, hi, _ = na.noble_mask_rows(starts, T, causal=False)
    q, k, v, do = (_rand(g, s, dt) for s in ((T, H, D), (T, K, D), (T, K, D), (T, H, D)))
    slopes = _slopes(H) if bias else None
    seen = dense_mask(T, T, lo.cpu(), hi.cpu())
    want = attention(q, k, v, seen, softcap=cap, slopes=slopes, do=do)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[:3] = bad[290:] = bad[130] = True
    for n, t in enumerate((q, k, v, do)):
        t[bad] = (math.nan, math.inf, -math.inf, math.nan)[n]
    got = _run(q, k, v, do, lo.cpu(), hi.cpu(), slopes, softcap=cap)
    ok = ~bad.cpu()
    for n, t in got.items():
        pick = (lambda x: x[:, ok]) if n == "lse" else (lambda x: x[ok])
        check(n, pick(t.cpu()), tuple(map(pick, want[n])), dt)
    empty = torch.cat([torch.arange(3), torch.arange(290, T)])
    for n in ("o", "dq", "dk", "dv"):
        assert bool((got[n][empty] == 0).all()), n
        assert not got[n][130].isfinite().any(), n
    assert bool((got["lse"][:, empty] == -math.inf).all())


def test_one_nan_reaches_the_rows_that_see_it():
    T, H, D = 200, 1, 128
    g = _gen(12)
    q, k, v, do = (_rand(g, (T, H, D), BF) for _ in range(4))
    v[100, 0, 5] = math.nan
    got = _run(q, k, v, do, None, None, None, causal=True)
    assert got["o"][:100].isfinite().all() and got["o"][100:, 0, 5].isnan().all()
    assert got["o"][100:, 0, :5].isfinite().all() and got["o"][100:, 0, 6:].isfinite().all()
    assert got["dq"][:100].isfinite().all()
    k[100, 0, 5], v[100, 0, 5] = math.inf, 0.0
    got = _run(q, k, v, do, None, None, None, causal=True)
    assert got["o"][:100].isfinite().all() and got["dq"][:100].isfinite().all()


# ------------------------------------------------------- norm and rotation --

ROPE = [
    # T, heads, kv_heads, D, rot, interleaved, norm, dtype
    (1, 1, 1, 8, 0, False, True, BF),
    (1, 16, 16, 128, 128, False, True, BF),
    (5, 4, 2, 64, 64, True, True, BF),
    (300, 3, 1, 96, 48, False, True, BF),
    (77, 2, 2, 80, 32, True, False, BF),
    (33, 8, 0, 128, 64, False, True, BF),
    (1000, 2, 1, 128, 128, False, False, BF),
    (5000, 4, 4, 64, 16, False, True, BF),
    (1, 2, 1, 64, 32, False, True, F32),
    (259, 6, 2, 128, 128, True, True, F32),
    (64, 1, 1, 16, 16, False, True, F32),
    (3000, 4, 2, 72, 64, False, True, F32),
]


@pytest.mark.parametrize("c", ROPE, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_qk_rope(c):
    T, H, K, D, rot, inter, norm, dt = c
    print(f"[rope] {c}", flush=True)
    g = _gen(T + D)
    C = (H + 2 * K) * D
    qkv = _rand(g, (T, C), dt)
    wq, wk = (1 + _rand(g, (D,), F32, 0.2), 1 + _rand(g, (D,), F32, 0.2)) if norm else (None, None)
    cos, sin = na.noble_rope_table(512, rot) if rot else (None, None)
    pos = torch.randint(0, 512, (T,), generator=g, device="cuda", dtype=torch.int32)
    dq, dk = _rand(g, (T, H, D), dt), _rand(g, (T, K, D), dt)
    kw = dict(heads=H, kv_heads=K, interleaved=inter, eps=1e-5)
    q, k = na.noble_qk_rope_fwd(qkv, wq, wk, cos, sin, pos, **kw)
    dqkv = torch.full_like(qkv, 3.0)
    _, dwq, dwk = na.noble_qk_rope_bwd(dq, dk, qkv, wq, wk, cos, sin, pos, dqkv=dqkv, **kw)
    torch.cuda.synchronize()
    at = pos.long()
    tabs = (None, None) if cos is None else (cos[at], sin[at])
    for n, a, b, w, y, dy, dw in (("q", 0, H, wq, q, dq, dwq), ("k", H, H + K, wk, k, dk, dwk)):
        if a == b:
            continue
        x = qkv[:, a * D:b * D].reshape(T, b - a, D).double().requires_grad_(True)
        wd = None if w is None else w.double().requires_grad_(True)
        ref = heads_norm_rope(x, wd, *tabs, inter, 1e-5)
        close(n, y, ref, dt)
        gr = torch.autograd.grad(ref, [x] if wd is None else [x, wd], dy.double())
        # the gradient's terms: r w dy and its projection on the head, at most twice the row's
        close("d" + n, dqkv[:, a * D:b * D].reshape(T, b - a, D), gr[0], dt,
              scale=None if wd is None else (2 * dy.double().square().mean(-1, keepdim=True).sqrt() *
                                             torch.rsqrt(x.detach().square().mean(-1, keepdim=True) + 1e-5)).cpu())
        if wd is not None:   # a sum over T x heads of products of order one
            assert float((dw.double() - gr[1]).abs().max()) <= 1e-6 * math.sqrt(T * (b - a)) * 8, n
    assert bool((dqkv[:, (H + K) * D:] == 3.0).all())


def test_positions_outside_the_tables_are_nan():
    g = _gen(1)
    qkv = _rand(g, (4, 3 * 64), BF)
    cos, sin = na.noble_rope_table(10, 32)
    pos = torch.tensor([0, 10, -1, 9], dtype=torch.int32, device="cuda")
    q, k = na.noble_qk_rope_fwd(qkv, None, None, cos, sin, pos, heads=1, kv_heads=1)
    for t in (q, k):
        assert t[[1, 2], :, :32].isnan().all() and not t[[0, 3]].isnan().any() and not t[..., 32:].isnan().any()


@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "ramp"])
def test_rope_table(scaling):
    """Against the formulas in float64: one rounding to float32 of the double result (its own error below 1e-9)."""
    rot, n, base, s, trained = 64, 5000, 10000.0, 4.0, 1024.0
    cos, sin = na.noble_rope_table(n, rot, base=base, scaling=scaling, factor=s, trained=trained, gain=1.1)
    i = torch.arange(rot // 2, dtype=torch.float64)
    f = (base * (s ** (rot / (rot - 2)) if scaling == "base" else 1.0)) ** (-2 * i / rot)
    gain = 1.0
    if scaling == "linear":
        f = f / s
    if scaling == "ramp":
        a, b = (rot / 2 * math.log(trained / (2 * math.pi * t)) / math.log(base) for t in (32.0, 1.0))
        w = ((i - a) / (b - a)).clamp(0, 1)
        f, gain = f * (1 - w) + f / s * w, 1.1
    ang = torch.arange(n, dtype=torch.float64)[:, None] * f
    assert float((cos.double().cpu() - gain * torch.cos(ang)).abs().max()) <= 1.1 * 2.0 ** -24 * 1.01 + 1e-9
    assert float((sin.double().cpu() - gain * torch.sin(ang)).abs().max()) <= 1.1 * 2.0 ** -24 * 1.01 + 1e-9


@pytest.mark.parametrize("causal,prefix,window", [(True, False, 0), (True, True, 0), (False, False, 0),
                                                  (True, False, 5), (False, False, 4)])
def test_mask_rows(causal, prefix, window):
    starts, T = [2, 9, 9, 40, 41], 50   # rows 0, 1 and 41 .. are in no document; one document is empty
    pre = [3, 0, 12, 1]
    s = torch.tensor(starts, dtype=torch.int32, device="cuda")
    p = torch.tensor(pre, dtype=torch.int32, device="cuda") if prefix else None
    lo, hi, pos = (t.tolist() for t in na.noble_mask_rows(s, T, prefix=p, causal=causal, window=window))
    for i in range(T):
        doc = next((n for n in range(4) if starts[n] <= i < starts[n + 1]), None)
        want = (0, 0, 0)
        if doc is not None:
            a, b = starts[doc], starts[doc + 1]
            end = i + 1 if causal else b
            if prefix:
                end = max(end, min(b, a + pre[doc]))
            want = (max(a, end - window) if window else a, end, i - a)
        assert (lo[i], hi[i], pos[i]) == want, i


# ------------------------------------------------------------ paged cache --

PAGED = [
    # lengths, new, heads, kv_heads, D, page, window, dtype, softcap, bias
    ([1], 1, 1, 1, 64, 8, 0, BF, 0.0, False),
    ([0, 5, 33], 1, 4, 2, 128, 16, 0, BF, 0.0, False),        # an empty sequence gives zeros
    ([1000], 1, 16, 16, 128, 16, 0, BF, 0.0, True),
    ([31, 32, 33, 700], 1, 8, 1, 128, 32, 0, BF, 30.0, False),
    ([100, 2, 64], 3, 6, 2, 96, 8, 0, BF, 0.0, True),         # more new tokens than one sequence holds
    ([90, 257], 7, 16, 2, 64, 64, 0, BF, 0.0, False),         # several tiles of 16 rows
    ([300, 77], 2, 4, 4, 128, 128, 50, BF, 0.0, False),
    ([2000, 9], 1, 2, 2, 40, 16, 33, BF, 20.0, True),
    ([5000], 1, 4, 1, 64, 4096, 0, BF, 0.0, False),
    ([65, 300], 2, 4, 2, 128, 16, 0, F32, 25.0, True),
    ([1000, 1], 1, 2, 1, 64, 8, 100, F32, 0.0, False),
]


@pytest.mark.parametrize("c", PAGED, ids=lambda c: "-".join(str(x).replace("torch.", "").replace(" ", "") for x in c))
def test_append_and_paged_attention(c):
    """Tokens appended in two calls (a prompt, then the new ones), then attention of the new ones over the cache, whose
    unused slots hold NaN."""
    lengths, new, H, K, D, page, window, dt, cap, bias = c
    print(f"[paged] {c}", flush=True)
    B, g = len(lengths), _gen(sum(lengths))
    per = max(1, -(-max(lengths) // page))
    n_pages = B * per + 2
    cache = torch.full((n_pages, 2, K, page, D), math.nan, dtype=dt, device="cuda")
    table = torch.randperm(n_pages, generator=g, device="cuda")[:B * per].view(B, per).to(torch.int32)
    cos, sin = na.noble_rope_table(max(max(lengths), 1), D // 16 * 16)
    wq, wk = 1 + _rand(g, (D,), F32, 0.1), 1 + _rand(g, (D,), F32, 0.1)
    kw = dict(heads=H, kv_heads=K, interleaved=False)
    qkv = [_rand(g, (n, (H + 2 * K) * D), dt) for n in lengths]
    queries = torch.zeros(B * new, H, D, dtype=dt, device="cuda")
    for b, n in enumerate(lengths):
        for first, end in ((0, max(n - new, 0)), (max(n - new, 0), n)):
            if first == end:
                continue
            at = torch.arange(first, end, device="cuda")
            slots = table[b].long()[at // page] * page + at % page
            x = qkv[b][first:end]
            pad = _rand(g, (1, x.shape[1]), dt)   # a padded row, whose slot is none
            y = na.noble_kv_append(torch.cat([x, pad]), wq, wk, cos, sin, torch.cat([at, at[:1]]).to(torch.int32),
                                   torch.cat([slots, slots.new_tensor([-1])]), cache, **kw)
            if end == n:
                queries[(b + 1) * new - (end - first):(b + 1) * new] = y[:-1]
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    slopes = _slopes(H) if bias else None
    o = na.noble_attn_paged(queries, cache, table, lens, slopes, softcap=cap, window=window)
    torch.cuda.synchronize()
    assert int((~cache.isnan()).sum()) == sum(lengths) * 2 * K * D   # every slot once, and no other
    for b, n in enumerate(lengths):
        if n:
            t = torch.arange(n, device="cuda")
            held = [cache[table[b].long()[t // page], i, :, t % page] for i in (0, 1)]   # [n, K, D]
            x = qkv[b].view(n, H + 2 * K, D)
            close("k", held[0], heads_norm_rope(x[:, H:H + K], wk, cos[t], sin[t], False, 1e-6), dt)
            assert bool((held[1] == x[:, H + K:]).all())
        else:
            held = [torch.zeros(0, K, D, dtype=dt, device="cuda")] * 2
        at = torch.arange(n - new, n)
        lo = torch.clamp(at - window + 1, min=0) if window else torch.zeros_like(at)
        seen = dense_mask(new, n, lo, at + 1)
        want = attention(queries[b * new:(b + 1) * new], *held, seen, softcap=cap, slopes=slopes)
        check("o", o[b * new:(b + 1) * new], want["o"], dt)


def test_paged_window_leaves_older_slots_alone():
    """Slots before the window hold NaN, as those of pages that a program has given away may."""
    g = _gen(7)
    page, D, n, window = 16, 64, 200, 37
    cache = _rand(g, (16, 2, 2, page, D), BF)
    table = torch.arange(13, dtype=torch.int32, device="cuda")[None]
    q = _rand(g, (1, 4, D), BF)
    t = torch.arange(n, device="cuda")
    held = [cache[t // page, i, :, t % page] for i in (0, 1)]
    want = attention(q, *(x[n - window:] for x in held), dense_mask(1, window))
    old = torch.arange(n - window, device="cuda")
    for i in (0, 1):
        cache[old // page, i, :, old % page] = math.nan
    o = na.noble_attn_paged(q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), window=window)
    check("o", o, want["o"], BF)


@pytest.mark.parametrize("dt,D", [(BF, 64), (BF, 128), (F32, 96)])
@pytest.mark.parametrize("window", [0, 40])
def test_paged_nan_reaches_the_tokens_that_see_it(dt, D, window):
    """Several new tokens in one tile of rows, and tokens at their windows' starts: each token's result is that of the
    tokens it sees, as a call without the others gives it."""
    print(f"[paged] nan {dt} {D} {window}", flush=True)
    g = _gen(11)
    page, n, new, H, K = 16, 150, 6, 4, 2
    cache = _rand(g, (12, 2, K, page, D), dt)
    table = torch.arange(10, dtype=torch.int32, device="cuda")[None] + 1
    q = _rand(g, (new, H, D), dt)
    slot = lambda t: (int(table[0, t // page]), t % page)  # noqa: E731
    marks = [(n - 2, 1, math.nan), (n - 4, 0, math.inf)] + ([(n - new - window + 3, 1, -math.inf)] if window else [])
    for t, i, x in marks:
        cache[slot(t)[0], i, 0, slot(t)[1], 5] = x
    o = na.noble_attn_paged(q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), window=window)
    t = torch.arange(n, device="cuda")
    held = [cache[table[0].long()[t // page], i, :, t % page] for i in (0, 1)]
    for r in range(new):
        first, end = max(n - new + r - window + 1, 0) if window else 0, n - new + r + 1
        ref, mag = attention(q[r:r + 1], *(x[first:end] for x in held), torch.ones(1, end - first, dtype=torch.bool))["o"]
        assert bool((torch.isfinite(o[r, H // K:].cpu())).all())   # the second key head has no marks
        if any(first <= t < end for t, _, _ in marks):
            assert bool((torch.isfinite(o[r].cpu()) | ~torch.isfinite(ref[0])).all())
        else:
            check("o", o[r:r + 1], (ref, mag), dt)
    assert not bool(o[new - 1].isfinite().all())


def test_paged_pages_outside_the_cache_are_not_seen():
    g = _gen(8)
    cache = _rand(g, (4, 2, 1, 8, 64), BF)
    q = _rand(g, (1, 1, 64), BF)
    table = torch.tensor([[2, 9, 1, -1]], dtype=torch.int32, device="cuda")
    o = na.noble_attn_paged(q, cache, table, torch.tensor([30], dtype=torch.int32, device="cuda"))
    k, v = (torch.cat([cache[2, i, 0], cache[1, i, 0]])[:, None] for i in (0, 1))
    check("o", o, attention(q, k, v, dense_mask(1, 16))["o"], BF)


def test_cache_past_4_gib():
    """Pages on both sides of byte 2^32 of the cache."""
    g = _gen(2)
    page, K, D = 64, 4, 128
    n_pages = 2 ** 32 // (2 * K * page * D * 2) + 40
    cache = torch.zeros((n_pages, 2, K, page, D), dtype=BF, device="cuda")
    table = torch.tensor([[n_pages - 1, 3, n_pages - 20, 2 ** 32 // (2 * K * page * D * 2)]], dtype=torch.int32, device="cuda")
    n = 4 * page
    qkv = _rand(g, (n, (8 + 2 * K) * D), BF)
    at = torch.arange(n, device="cuda")
    slots = table[0].long()[at // page] * page + at % page
    q = na.noble_kv_append(qkv, None, None, None, None, None, slots, cache, heads=8, kv_heads=K)
    o = na.noble_attn_paged(q[-1:].contiguous(), cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    x = qkv.view(n, 8 + 2 * K, D)
    assert bool((cache[table[0].long()][:, 0].transpose(1, 2).reshape(n, K, D) == x[:, 8:8 + K]).all())
    check("o", o, attention(x[-1:, :8], x[:, 8:8 + K], x[:, 8 + K:], dense_mask(1, n))["o"], BF)


# ---------------------------------------------------------------- streams --

def test_other_stream_and_graph():
    """A call on a stream that is not the current one, and forward and backward captured in a graph and replayed, with
    eager work and synchronizations between: the eager results, bit for bit."""
    T, H, K, D = 260, 4, 2, 64
    g = _gen(4)
    q, k, v, do = (_rand(g, s, BF) for s in ((T, H, D), (T, K, D), (T, K, D), (T, H, D)))
    want = _run(q, k, v, do, None, None, None, causal=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o, lse = na.noble_attn_fwd(q, k, v, causal=True, stream=side)
    dq, dk, dv = na.noble_attn_bwd(do, q, k, v, o, lse, causal=True, stream=side)
    side.synchronize()
    assert all(bool((a == b).all()) for a, b in zip((o, lse, dq, dk, dv), want.values()))
    outs = {n: torch.empty_like(t) for n, t in want.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        na.noble_attn_fwd(q, k, v, causal=True, o=outs["o"], lse=outs["lse"])
        na.noble_attn_bwd(do, q, k, v, outs["o"], outs["lse"], causal=True, dq=outs["dq"], dk=outs["dk"], dv=outs["dv"])
    for _ in range(3):
        for t in outs.values():
            t.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((outs[n] == want[n]).all()) for n in want)
        _run(q, k, v, do, None, None, None)


# --------------------------------------------------------------- refusals --

def test_refusals():
    T, H, K, D = 16, 4, 2, 64
    g = _gen(0)
    q, k, v = (_rand(g, s, BF) for s in ((T, H, D), (T, K, D), (T, K, D)))
    lo = torch.zeros(T, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="on the GPU"):
        na.noble_attn_fwd(q.cpu(), k, v)
    with pytest.raises(ValueError, match="given together"):
        na.noble_attn_fwd(q, k, v, lo)
    with pytest.raises(TypeError, match="key_lo"):
        na.noble_attn_fwd(q, k, v, lo.long(), lo.long())
    with pytest.raises(TypeError, match="v must be"):
        na.noble_attn_fwd(q, k, v.float())
    with pytest.raises(ValueError, match="adjacent"):
        na.noble_attn_fwd(q.transpose(1, 2).contiguous().transpose(1, 2), k, v)
    with pytest.raises(noble.NobleError, match="BAD_SHAPE"):
        na.noble_attn_fwd(q[:, :3].contiguous(), k, v)       # 3 query heads over 2
    with pytest.raises(noble.NobleError, match="BAD_SHAPE"):
        na.noble_attn_fwd(q, k, v, o=q.new_empty(T, 1, D).expand(T, H, D))   # an output that overlaps itself
    with pytest.raises(noble.NobleError, match="BAD_SHAPE"):
        na.noble_attn_fwd(q, k, v, softcap=-1.0)
    with pytest.raises(noble.NobleError, match="MISALIGNED"):
        na.noble_attn_fwd(torch.empty(T * H * D + 8, dtype=BF, device="cuda")[4:4 + T * H * D].view(T, H, D), k, v)
    with pytest.raises(ValueError, match="qkv"):
        na.noble_qk_rope_fwd(q.view(T, -1), None, None, None, None, None, heads=3, kv_heads=1)
    cos, sin = na.noble_rope_table(16, 32)
    with pytest.raises(noble.NobleError, match="BAD_SHAPE"):
        na.noble_qk_rope_fwd(q.view(T, -1), None, None, cos[:, :5].contiguous(), sin[:, :5].contiguous(), None, heads=2,
                             kv_heads=1)
    with pytest.raises(ValueError, match="cache"):
        na.noble_attn_paged(q, k, lo[None], lo[:1])
    with pytest.raises(noble.NobleError, match="BAD_SHAPE"):
        na.noble_attn_paged(q[:1], torch.zeros(2, 2, 2, 12, D, dtype=BF, device="cuda"), lo[None, :1].contiguous(), lo[:1])
