"""The attention operators at the edges of their arguments: other streams, windows, infinities, caps, one row, second
derivatives, lengths."""

import math

import pytest
import torch

from _attention import attention, check, dense_mask
from paper_2603_06492_amd import attention as na

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(g, shape, dt=F32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dt)


# ---------------------------------------------------------------- streams --

def test_calls_on_another_stream_while_the_current_one_is_busy():
    """Every call on a stream of its own, its inputs ready, while the current stream has work queued on tensors that have
    been freed since: the results are those of the current stream, bit for bit, and the queued work is not disturbed."""
    T, H, K, D = 200, 4, 2, 64
    g = _gen(21)
    wide = _rand(g, (T, (H + 2 * K) * D + 64), BF)
    qkv = wide[:, :(H + 2 * K) * D]
    w = 1 + _rand(g, (D,), F32, 0.1)
    dq, dk, do = _rand(g, (T, H, D), BF), _rand(g, (T, K, D), BF), _rand(g, (T, H, D), BF)
    starts = torch.tensor([0, 70, 71, 190], dtype=torch.int32, device="cuda")
    slots = torch.arange(T, device="cuda") + 8
    table = torch.arange(1, 27, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([T], dtype=torch.int32, device="cuda")
    caches = [torch.zeros((27, 2, K, 8, D), dtype=BF, device="cuda") for _ in range(2)]
    given = [torch.full((T, (H + 2 * K) * D), 5.0, dtype=BF, device="cuda") for _ in range(2)]
    how = dict(heads=H, kv_heads=K)

    def everything(cache, into, **on):
        cos, sin = na.noble_rope_table(256, 32, **on)
        lo, hi, pos = na.noble_mask_rows(starts, T, **on)
        rope = (qkv, w, w, cos, sin, pos)
        q, k = na.noble_qk_rope_fwd(*rope, **how, **on)
        v = qkv[:, (H + K) * D:].view(T, K, D)
        o, lse = na.noble_attn_fwd(q, k, v, lo, hi, **on)
        grads = na.noble_attn_bwd(do, q, k, v, o, lse, lo, hi, **on)
        zeroed = na.noble_qk_rope_bwd(dq, dk, *rope, **how, **on)                # its gradient's tensor is zeroed inside
        copied = na.noble_qk_rope_bwd(dq, dk, *rope, dqkv=into, **how, **on)     # its rows are copied inside
        qa = na.noble_kv_append(*rope, slots, cache, **how, **on)
        op = na.noble_attn_paged(qa[-3:], cache, table, lens, **on)
        return [cos, sin, lo, hi, pos, q, k, o, lse, *grads, *zeroed, *copied, qa, op]

    want = everything(caches[0], given[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(2048, 2048, device="cuda", generator=g)
    for _ in range(2):   # the second time with blocks that the first one's tensors left
        caches[1].zero_()
        given[1].fill_(5.0)
        torch.cuda.synchronize()
        sums = []
        for n in (16, 4096, T * H * D * 2, T * (H + 2 * K) * D * 2, 1 << 20):   # queued work on blocks that are free at once
            x = torch.ones(n, dtype=torch.uint8, device="cuda")
            for _ in range(20):
                big = torch.tanh(big @ big)
            sums.append((n, x.sum(dtype=torch.int64) + 0 * big[0, 0].nan_to_num().long()))
            del x
        got = everything(caches[1], given[1], stream=side)
        side.synchronize()
        torch.cuda.synchronize()
        for n, s in sums:
            assert int(s) == n
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), i
        assert torch.equal(caches[0], caches[1])
        del got


# -------------------------------------------------------------------- caps --

CAP_SIZES = pytest.mark.parametrize("dt,H,K,D", [(BF, 4, 2, 64), (F32, 4, 2, 64), (BF, 96, 96, 64), (BF, 96, 48, 128)],
                                    ids=["bf16", "f32", "bf16_wide64", "bf16_wide128"])


def _slope_slack(q, k, v, do, seen, cap):
    """1e-6 of what dq and dk would sum without the cap's slope."""
    (T, H, D), K = q.shape, k.shape[1]
    q, do = (x.double().cpu().transpose(0, 1) for x in (q, do))
    k, v = (x.double().cpu().transpose(0, 1).repeat_interleave(H // K, 0) for x in (k, v))
    p = torch.softmax((cap * torch.tanh(q @ k.transpose(1, 2) * D ** -0.5 / cap)).masked_fill(~seen, -math.inf), -1)
    m = 1e-6 * D ** -0.5 * p * ((do @ v.transpose(1, 2)).abs() + (do * (p @ v)).sum(-1, keepdim=True).abs())
    return (m @ k.abs()).transpose(0, 1), (m.transpose(1, 2) @ q.abs()).view(K, H // K, T, D).sum(1).transpose(0, 1)


@CAP_SIZES
@pytest.mark.parametrize("cap", [0.5, 1.0, 4.0])
def test_scores_up_to_many_times_the_cap(dt, H, K, D, cap):
    """Scores of standard deviation 1 to 3 under caps of half to four: below, near and far above the cap, in one tile and in
    one lane.  1 - tanh^2 is a float32 difference of numbers up to 1: 1e-6 of what the score gradients would be
    without it joins their bounds."""
    print(f"[attn] capped {dt} {H} {K} {D} {cap}", flush=True)
    T = 150
    g = _gen(75)
    q, k, v, do = (_rand(g, s, dt) for s in ((T, H, D), (T, K, D), (T, K, D), (T, H, D)))
    q *= torch.linspace(0.2, 3.0, T, device="cuda")[:, None, None].to(dt)
    o, lse = na.noble_attn_fwd(q, k, v, causal=True, softcap=cap)
    dq, dk, dv = na.noble_attn_bwd(do, q, k, v, o, lse, causal=True, softcap=cap)
    seen = dense_mask(T, T, causal=True)
    want = attention(q, k, v, seen, softcap=cap, do=do)
    slack_q, slack_k = _slope_slack(q, k, v, do, seen, cap)
    for n, t in dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv).items():
        ref, mag = want[n]
        u = 2.0 ** -8 if dt == BF else 2e-5
        check(n, t, (ref, mag + {"dq": slack_q / u, "dk": slack_k / u}.get(n, 0.0)), dt)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("cap", [0.5, 2.0])
@pytest.mark.parametrize("new", [1, 3])
def test_paged_scores_up_to_many_times_the_cap(dt, cap, new):
    print(f"[paged] capped {dt} {cap} {new}", flush=True)
    n, H, K, D, page = 333, 8, 2, 64, 16
    g = _gen(76)
    cache = _rand(g, (22, 2, K, page, D), dt)
    table = torch.arange(22, dtype=torch.int32, device="cuda")[None]
    q = _rand(g, (new, H, D), dt) * torch.linspace(0.3, 3.0, H, device="cuda")[:, None].to(dt)
    o = na.noble_attn_paged(q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), softcap=cap)
    t = torch.arange(n, device="cuda")
    k, v = (cache[t // page, i, :, t % page] for i in (0, 1))
    check("o", o, attention(q, k, v, dense_mask(new, n, causal=True), softcap=cap)["o"], dt)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("cap", [1e-30, 1e-12, 1e-6, 1e30])
def test_caps_of_any_size(dt, cap):
    """A cap far below the scores leaves them all alike, one far above leaves them as they are.  There 1 - tanh^2 is 0 in
    float64 and up to a float32 rounding here, 1e-6 of the uncapped score gradients, themselves below 10."""
    print(f"[attn] cap {dt} {cap}", flush=True)
    T, H, K, D = 70, 4, 2, 64
    g = _gen(71)
    q, k, v, do = (_rand(g, s, dt) for s in ((T, H, D), (T, K, D), (T, K, D), (T, H, D)))
    o, lse = na.noble_attn_fwd(q, k, v, causal=True, softcap=cap)
    dq, dk, dv = na.noble_attn_bwd(do, q, k, v, o, lse, causal=True, softcap=cap)
    want = attention(q, k, v, dense_mask(T, T, causal=True), softcap=cap, do=do)
    names = ("o", "lse", "dv") + (("dq", "dk") if cap > 1 else ())
    for n in names:
        check(n, dict(o=o, lse=lse, dv=dv, dq=dq, dk=dk)[n], want[n], dt)
    if cap < 1:
        assert float(dq.float().abs().max()) <= 1e-4 and float(dk.float().abs().max()) <= 1e-4


def test_large_caps_near_their_scores():
    """A cap of 1e6 and scores of 0.02 to 0.9 times it, one key a row: lse is the score, within the tanh's error (1e-7 below
    1, relative 3e-8 up to 1/2) and four float32 roundings, 6e-7."""
    T, D = 44, 64
    x = torch.linspace(0.02, 0.9, T)
    q = torch.full((T, 1, D), 125.0, dtype=BF, device="cuda")
    k = (x * 1e6 / D / 125.0)[:, None, None].expand(T, 1, D).to(BF).cuda().contiguous()
    i = torch.arange(T, dtype=torch.int32, device="cuda")
    _, lse = na.noble_attn_fwd(q, k, k, i, i + 1, scale=1.0, softcap=1e6)
    want = 1e6 * torch.tanh(D * 125.0 * k[:, 0, 0].double().cpu() / 1e6)
    assert float((lse[0].double().cpu() / want - 1).abs().max()) <= 6e-7 + 1e-7 / 0.5


# ----------------------------------------------------------------- windows --

@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 5, 1 << 30, 64, 40])
@pytest.mark.parametrize("lengths,new", [([3, 40, 0], 7), ([2, 64], 1)])
def test_paged_windows_up_to_the_largest(lengths, new, window):
    """Windows that hide nothing, up to the largest number, and sequences that hold fewer tokens than are new: the rows
    of tokens before the first see nothing, the others what they see without a window."""
    print(f"[paged] window {window} {lengths} {new}", flush=True)
    H, K, D, page = 4, 2, 64, 16
    g = _gen(31)
    cache = _rand(g, (20, 2, K, page, D), BF)
    table = torch.randperm(20, generator=g, device="cuda")[:len(lengths) * 4].view(-1, 4).to(torch.int32)
    q = _rand(g, (len(lengths) * new, H, D), BF)
    o = na.noble_attn_paged(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), window=window)
    for b, n in enumerate(lengths):
        t = torch.arange(n, device="cuda")
        k, v = (cache[table[b].long()[t // page], i, :, t % page] for i in (0, 1))
        at = torch.arange(n - new, n)
        rows = slice(b * new, (b + 1) * new)
        check("o", o[rows], attention(q[rows], k, v, dense_mask(new, n, (at - window + 1).clamp(min=0), at + 1))["o"], BF)


# ------------------------------------------------- elements not rotated --

@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 16), (128, 64), (72, 32)])
def test_infinities_past_the_rotated_elements_stay_alone(dt, inter, D, rot):
    """Without a norm the elements past the rotated ones come out as they went in, infinite ones too, and reach no other
    element; so do their gradients."""
    print(f"[rope] inf {dt} {inter} {D} {rot}", flush=True)
    T, H, K = 11, 3, 2
    g = _gen(41)
    qkv, dq, dk = (_rand(g, s, dt) for s in ((T, (H + 2 * K) * D), (T, H, D), (T, K, D)))
    cos, sin = na.noble_rope_table(T, rot)
    heads = lambda x, a, b: x[:, a * D:b * D].view(T, b - a, D)  # noqa: E731

    def run():
        q, k = na.noble_qk_rope_fwd(qkv, None, None, cos, sin, None, heads=H, kv_heads=K, interleaved=inter)
        d, _, _ = na.noble_qk_rope_bwd(dq, dk, qkv, None, None, cos, sin, None, heads=H, kv_heads=K, interleaved=inter)
        return [q, k, heads(d, 0, H), heads(d, H, H + K)]

    clean = run()
    ins = [heads(qkv, 0, H), heads(qkv, H, H + K), dq, dk]
    for x in ins:
        x[3, 0, rot], x[5, 1, rot + 5], x[7, :, D - 1] = math.inf, -math.inf, math.inf
    for x, was, now in zip(ins, clean, run()):
        assert torch.equal(now[..., rot:], x[..., rot:])
        assert torch.equal(now[..., :rot], was[..., :rot])


# ----------------------------------------------------------------- one row --

@pytest.mark.parametrize("T", [1, 2])
def test_gradient_rows_need_adjacent_columns(T):
    """A given gradient of the Q/K/V rows with spread columns is refused whatever the number of rows; columns of a wider
    buffer are not."""
    H, K, D = 2, 1, 16
    C = (H + 2 * K) * D
    g = _gen(51)
    qkv, dq, dk = _rand(g, (T, 2 * C), BF)[:, :C], _rand(g, (T, H, D), BF), _rand(g, (T, K, D), BF)
    wide = torch.full((T, 2 * C), 7.0, dtype=BF, device="cuda")
    with pytest.raises(ValueError, match="adjacent columns"):
        na.noble_qk_rope_bwd(dq, dk, qkv, None, None, None, None, None, heads=H, kv_heads=K, dqkv=wide[:, ::2])
    assert bool((wide == 7.0).all())
    into = wide[:, 16:16 + C]
    na.noble_qk_rope_bwd(dq, dk, qkv, None, None, None, None, None, heads=H, kv_heads=K, dqkv=into)
    assert torch.equal(into[:, :H * D], dq.view(T, -1)) and torch.equal(into[:, H * D:(H + K) * D], dk.view(T, -1))
    assert bool((wide[:, :16] == 7.0).all()) and bool((wide[:, 16 + (H + K) * D:] == 7.0).all())


# ------------------------------------------- scores of minus infinity alone --

@pytest.mark.parametrize("dt,H,K,D", [(BF, 4, 2, 64), (F32, 4, 2, 64), (BF, 96, 96, 64), (BF, 96, 48, 128)],
                         ids=["bf16", "f32", "bf16_wide64", "bf16_wide128"])
@pytest.mark.parametrize("bias", [False, True])
def test_rows_that_see_only_scores_of_minus_infinity(dt, H, K, D, bias):
    """One document's keys are minus infinity before positive queries: its rows' exponentials are all 0 / 0.  Its results
    are not numbers, the other documents' those of clean inputs, an empty row's zeros."""
    print(f"[attn] -inf {dt} {H} {K} {D} {bias}", flush=True)
    T, a, z = 150, 61, 70
    g = _gen(61)
    starts = torch.tensor([0, a, z, 140], dtype=torch.int32, device="cuda")
    lo, hi, _ = na.noble_mask_rows(starts, T)
    q, k, v, do = (_rand(g, s, dt) for s in ((T, H, D), (T, K, D), (T, K, D), (T, H, D)))
    q = q.abs() + 0.125
    slopes = torch.linspace(0.1, 1.0, H, device="cuda") if bias else None
    want = attention(q, k, v, dense_mask(T, T, lo.cpu(), hi.cpu()), slopes=slopes, do=do)
    k[a:z] = -math.inf
    o, lse = na.noble_attn_fwd(q, k, v, lo, hi, slopes)
    grads = na.noble_attn_bwd(do, q, k, v, o, lse, lo, hi, slopes)
    ok = torch.ones(T, dtype=torch.bool)
    ok[a:z] = False
    for n, t in zip(("o", "dq", "dk", "dv"), (o, *grads)):
        assert bool(t[a:z].isnan().all()), n
        check(n, t.cpu()[ok], tuple(x[ok] for x in want[n]), dt)
        assert n == "o" or bool((t[140:] == 0).all())
    assert bool((o[140:] == 0).all()) and bool((lse[:, a:z] == -math.inf).all())
    check("lse", lse.cpu()[:, ok], tuple(x[:, ok] for x in want["lse"]), dt)
    k[a] = 0.5   # one of them is an ordinary score: it takes the rows alone
    o, _ = na.noble_attn_fwd(q, k, v, lo, hi, slopes)
    one = v[a].repeat_interleave(H // K, 0).float().cpu()
    for i in range(a, z):
        assert float((o[i].float().cpu() - one).abs().max()) <= 2.0 ** -7 * float(one.abs().max())


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("n,window", [(1, 0), (9, 0), (3000, 0), (3000, 40)])
@pytest.mark.parametrize("new", [1, 2])
def test_paged_rows_that_see_only_scores_of_minus_infinity(dt, n, window, new):
    """Over the cache: not numbers, and zeros for a row that sees nothing, its pages outside the cache or its token before
    the first."""
    print(f"[paged] -inf {dt} {n} {window} {new}", flush=True)
    H, K, D, page = 4, 2, 64, 16
    per = -(-n // page)
    g = _gen(62)
    cache = _rand(g, (per + 1, 2, K, page, D), dt)
    cache[:, 0] = -math.inf
    table = torch.stack([torch.randperm(per + 1, generator=g, device="cuda")[:per], torch.full((per,), -1, device="cuda"),
                         torch.zeros(per, dtype=torch.int64, device="cuda")]).to(torch.int32)
    q = _rand(g, (3 * new, H, D), dt).abs() + 0.125
    lens = torch.tensor([n, n, 0], dtype=torch.int32, device="cuda")
    o = na.noble_attn_paged(q, cache, table, lens, window=window).view(3, new, H, D)
    assert bool((o[1:] == 0).all())
    for t in range(new):
        assert bool(o[0, t].isnan().all()) if n - new + t >= 0 else bool((o[0, t] == 0).all())


# ----------------------------------------------------- what not-a-number costs --

def _ms(f, n=3):
    f()
    torch.cuda.synchronize()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / n


@pytest.mark.parametrize("what", ["do", "v", "q"])
def test_a_step_of_nan_takes_milliseconds(what):
    """A training step whose values or upstream gradient have all turned into NaN: a row or key whose sums are NaN already
    is done.  About 64 rows a wave, a few microseconds each: ten times the clean step and a millisecond leave room."""
    print(f"[attn] cost {what}", flush=True)
    T, H, K, D = 2048, 8, 8, 128
    g = _gen(81)
    x = dict(q=_rand(g, (T, H, D), BF), k=_rand(g, (T, K, D), BF), v=_rand(g, (T, K, D), BF), do=_rand(g, (T, H, D), BF))

    def step():
        o, lse = na.noble_attn_fwd(x["q"], x["k"], x["v"])
        return na.noble_attn_bwd(x["do"], x["q"], x["k"], x["v"], o, lse)

    clean = _ms(step)
    x[what].fill_(math.nan)
    bad = _ms(step)
    print(f"clean {clean:.3f} ms, {what} NaN {bad:.3f} ms", flush=True)
    assert bad <= 10 * clean + 1.0
    dq, dk, dv = step()
    assert bool(dk.isnan().all()) and bool(dq.isnan().all())
    assert bool(dv.isnan().all()) == (what != "v")


@pytest.mark.parametrize("dt,H,K,D", [(BF, 4, 2, 64), (F32, 4, 2, 64), (BF, 96, 96, 128), (BF, 8, 1, 96)])
def test_infinite_gradients_over_many_documents(dt, H, K, D):
    """Infinite upstream gradients in one row of every third document: the keys that the row sees, in their documents and
    between their tiles, and no other."""
    print(f"[attn] inf documents {dt} {H} {K} {D}", flush=True)
    T = 450
    g = _gen(82)
    starts = torch.cat([torch.arange(0, T, 50), torch.tensor([T])]).to(torch.int32).cuda()
    lo, hi, _ = na.noble_mask_rows(starts, T)
    q, k, v, do = (_rand(g, s, dt) for s in ((T, H, D), (T, K, D), (T, K, D), (T, H, D)))
    want = attention(q, k, v, dense_mask(T, T, lo.cpu(), hi.cpu()), do=do)
    hit = torch.zeros(T, dtype=torch.bool)
    for a in range(0, T, 150):
        do[a + 20, 0, 3] = math.inf
        hit[a:a + 21] = True
    o, lse = na.noble_attn_fwd(q, k, v, lo, hi)
    dq, dk, dv = na.noble_attn_bwd(do, q, k, v, o, lse, lo, hi)
    for n, t in (("dk", dk), ("dv", dv)):
        check(n, t.cpu()[~hit], tuple(x[~hit] for x in want[n]), dt)
    assert bool((dv[hit.cuda(), 0, 3] == math.inf).all()) and not bool(dk[hit.cuda(), 0].isfinite().any())
    rest = torch.arange(D) != 3   # the value's other elements
    check("dv", dv.cpu()[hit][..., rest], tuple(x[hit][..., rest] for x in want["dv"]), dt)


# ------------------------------------------------------ second derivatives --

def test_second_derivatives_are_refused():
    """The backwards are not differentiable: a penalty on a gradient raises, it is not taken for a constant."""
    T, H, K, D = 20, 2, 1, 32
    g = _gen(91)
    qkv = _rand(g, (T, (H + 2 * K) * D)).requires_grad_(True)
    w = torch.ones(D, device="cuda", requires_grad=True)
    cos, sin = na.noble_rope_table(T, 32)

    def whole():
        return na.RopeAttention.apply(qkv, w, w, cos, sin, None, None, None, None, H, K)

    def rope():
        return torch.cat(na.QKRope.apply(qkv, w, w, cos, sin, None, H, K), 1)

    def attn():
        q, k, v = (qkv[:, a * D:b * D].reshape(T, b - a, D) for a, b in ((0, H), (H, H + K), (H + K, H + 2 * K)))
        return na.Attention.apply(q, k, v)

    for f in (whole, rope, attn):
        first, = torch.autograd.grad(f().square().sum(), qkv, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiate twice"):
            (qkv.sum() + first.square().sum()).backward()


# ------------------------------------------------------------------ module --

def test_lengths_past_the_tables_are_refused():
    """Sequences longer than the module's positions: refused where the host knows the length, in a batch, one sequence and a
    cache; a module that rotates nothing takes them."""
    m = na.NobleSelfAttention(64, 2, 8, longest=16)
    x = torch.randn(2, 17, 64, device="cuda", generator=_gen(95)).to(BF)
    for y in (x, x[0]):
        with pytest.raises(ValueError, match="longest"):
            m(y)
    assert bool(m(x[:, :16]).isfinite().all())
    cache = na.PagedCache(2, 40, 12, kv_heads=2, head_dim=32, page=8)
    assert cache.held == 0
    assert bool(m.step(x[:, :16].reshape(-1, 64), cache, *cache.extend(16)).isfinite().all()) and cache.held == 16
    with pytest.raises(ValueError, match="longest"):
        m.step(x[:, 16].contiguous(), cache, *cache.extend(1))
    still = na.NobleSelfAttention(64, 2, 8, longest=16, rot=0)
    assert bool(still(x).isfinite().all())
    assert bool(still.step(x[:, 16].contiguous(), cache, *cache.extend(1)).isfinite().all())


@pytest.mark.parametrize("window", [7, 20])
def test_module_decodes_with_the_window_that_it_trains_with(window):
    """A forward with a window, and a prompt and single tokens with the same: the same sums in another order, 1% of the
    output's norm."""
    B, S, d = 2, 33, 128
    m = na.NobleSelfAttention(d, 4, 16, kv_heads=2, longest=64, seed=4)
    x = torch.randn(B, S, d, device="cuda", generator=_gen(101)).to(BF)
    starts = torch.arange(0, B * S + 1, S, dtype=torch.int32, device="cuda")
    with torch.no_grad():
        whole = m(x, m.mask(starts, B * S, window=window))
        assert float((whole - m(x)).norm() / whole.norm()) > 0.05   # the window matters here
    cache = na.PagedCache(B, 64, 40, kv_heads=2, head_dim=m.head_dim, page=8)
    outs = [m.step(x[:, :20].reshape(-1, d), cache, *cache.extend(20), window=window).view(B, 20, d)]
    for t in range(20, S):
        outs.append(m.step(x[:, t].contiguous(), cache, *cache.extend(1), window=window)[:, None])
    off = torch.cat(outs, 1).float() - whole.float()
    assert float(off.norm() / whole.float().norm()) <= 1e-2


# --------------------------------------------------------------- long rows --

@pytest.mark.parametrize("dt,T,H,K,D,kind", [(BF, 2100, 8, 2, 128, "causal"), (BF, 2100, 8, 8, 64, "documents"),
                                             (F32, 1300, 2, 1, 64, "causal")])
def test_rows_of_thousands_of_keys(dt, T, H, K, D, kind):
    """Enough rows of few heads for workgroups of 128 rows, and many tiles in each; bounds as at every size."""
    print(f"[attn] long {dt} {T} {H} {K} {D} {kind}", flush=True)
    g = _gen(111)
    q, k, v, do = (_rand(g, s, dt) for s in ((T, H, D), (T, K, D), (T, K, D), (T, H, D)))
    lo = hi = None
    if kind == "documents":   # of 1000, 1 and 1088 rows, the last 11 in none
        lo, hi, _ = na.noble_mask_rows(torch.tensor([0, 1000, 1001, 2089], dtype=torch.int32, device="cuda"), T)
    causal = kind == "causal"
    o, lse = na.noble_attn_fwd(q, k, v, lo, hi, causal=causal, softcap=3.0)
    dq, dk, dv = na.noble_attn_bwd(do, q, k, v, o, lse, lo, hi, causal=causal, softcap=3.0)
    seen = dense_mask(T, T, *((None, None) if lo is None else (lo.cpu(), hi.cpu())), causal)
    want = attention(q, k, v, seen, softcap=3.0, do=do)
    for n, t in dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv).items():
        check(n, t, want[n], dt)


@pytest.mark.parametrize("dt,H,K,D,page,window", [(BF, 16, 2, 128, 16, 0), (BF, 4, 4, 64, 64, 150), (F32, 4, 1, 96, 8, 0)])
def test_prompts_over_the_cache(dt, H, K, D, page, window):
    """Hundreds of new tokens a sequence, a whole prompt and a chunk of a longer one."""
    print(f"[paged] prompt {dt} {H} {K} {D} {page} {window}", flush=True)
    lengths, new = [300, 777], 300
    g = _gen(112)
    per = -(-max(lengths) // page)
    cache = _rand(g, (2 * per + 1, 2, K, page, D), dt)
    table = torch.randperm(2 * per + 1, generator=g, device="cuda")[:2 * per].view(2, per).to(torch.int32)
    q = _rand(g, (2 * new, H, D), dt)
    o = na.noble_attn_paged(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), window=window,
                            softcap=3.0)
    for b, n in enumerate(lengths):
        t = torch.arange(n, device="cuda")
        k, v = (cache[table[b].long()[t // page], i, :, t % page] for i in (0, 1))
        at = torch.arange(n - new, n)
        lo = (at - window + 1).clamp(min=0) if window else torch.zeros_like(at)
        rows = slice(b * new, (b + 1) * new)
        check("o", o[rows], attention(q[rows], k, v, dense_mask(new, n, lo, at + 1), softcap=3.0)["o"], dt)
