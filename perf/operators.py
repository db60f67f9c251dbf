"""Performance cases of the operators between the grouped Q/K/V layer and the O layer of a transformer block: the norm and
rotation of the heads, the paged cache, and attention for training, prompts and single tokens.

``kind`` names the operator:

* ``rope``:   norm and rotation of queries and keys, forward and backward, of a training step;
* ``append``: new tokens of a batch of sequences into a paged cache, their queries normed and rotated;
* ``attn``:   attention over a batch of B sequences of S tokens, forward, or forward and backward;
* ``paged``:  attention of the last tokens of each sequence over the paged cache.

Where ``own`` is false, ``run`` computes the operators from their formulas in float32.
"""

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BASE = 10000.0
LARGEST_PAIRS = 16 * 16384 * 16384   # score entries (heads x rows x keys) that a drawn attention case may have


def _rope(name, T, heads, kv_heads, D, rot, dtype="bf16", interleaved=False, norm=True):
    return dict(name=name, kind="rope", T=T, heads=heads, kv_heads=kv_heads, D=D, rot=rot, dtype=dtype,
                interleaved=interleaved, norm=norm)


def _append(name, B, new, past, heads, kv_heads, D, rot, page, dtype="bf16", interleaved=False, norm=True):
    return dict(name=name, kind="append", B=B, new=new, past=past, heads=heads, kv_heads=kv_heads, D=D, rot=rot,
                page=page, dtype=dtype, interleaved=interleaved, norm=norm)


def _attn(name, B, S, heads, kv_heads, D, mask, dtype="bf16", softcap=0.0, alibi=False, backward=True):
    return dict(name=name, kind="attn", B=B, S=S, heads=heads, kv_heads=kv_heads, D=D, mask=mask, dtype=dtype,
                softcap=softcap, alibi=alibi, backward=backward)


def _paged(name, B, new, shortest, longest, heads, kv_heads, D, page, dtype="bf16", softcap=0.0, alibi=False):
    return dict(name=name, kind="paged", B=B, new=new, shortest=shortest, longest=longest, heads=heads,
                kv_heads=kv_heads, D=D, page=page, dtype=dtype, softcap=softcap, alibi=alibi)


def listed():
    return [
        # the four-block stack's training step, 16 x 2048 tokens: 16 heads of 128, norm and the whole head rotated
        _rope("rope_stack_32768", 32768, 16, 16, 128, 128),
        # a small model in full precision, an odd number of tokens: shared key heads, a quarter of each pair rotated
        _rope("rope_f32_partial", 2047, 8, 2, 64, 32, dtype="f32", interleaved=True),
        # one decoding step of 16 sequences into a cache of pages of 16 tokens
        _append("append_decode16", 16, 1, 777, 16, 16, 128, 128, 16),
        # four prompts of 777 tokens of a model with shared key heads
        _append("append_prompts", 4, 777, 0, 16, 4, 128, 64, 64, interleaved=True),
        # the 250M model's training step: 8 sequences of 1024 tokens, 8 heads of 128, causal
        _attn("train_250m", 8, 1024, 8, 8, 128, "causal"),
        # the 1.5B stack's training step: 16 x 2048 tokens, several documents packed in each row, capped scores
        _attn("train_stack_docs_cap", 16, 2048, 16, 16, 128, "docs", softcap=50.0),
        # ViT-B training: 128 images x 197 tokens, 12 heads of 64, every token sees its image
        _attn("train_vitb", 128, 197, 12, 12, 64, "full"),
        # a long prompt with a prefix that sees itself, shared key heads, the bias that grows with distance
        _attn("prompt_16384_prefix", 1, 16384, 16, 4, 128, "prefix", alibi=True, backward=False),
        # a toy model in full precision, odd lengths: packed documents, forward and backward
        _attn("tiny_f32_docs", 3, 333, 4, 2, 64, "docs", dtype="f32", alibi=True),
        # one token of one sequence: the smallest call of a decoding loop
        _paged("decode1", 1, 1, 1000, 1000, 16, 16, 128, 16),
        # one token of each of 16 sequences of very different lengths, capped scores
        _paged("decode16_ragged", 16, 1, 130, 8192, 16, 16, 128, 16, softcap=30.0),
        # 64 long sequences, shared key heads, a cache of 4.3 GB
        _paged("decode64_long", 64, 1, 16384, 32768, 16, 4, 128, 64),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges: 1 to 32768 tokens, sequences of 1 to 16384 tokens, caches of up to 64
    sequences, heads of 32 to 128, key heads shared by 1 to 8 query heads."""
    while True:
        kind = rng.choice(("rope", "append", "attn", "attn", "attn", "paged", "paged"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        D = rng.choice((32, 64, 64, 80, 96, 128, 128, 128))
        kv_heads = rng.choice((1, 2, 4, 8, 12, 16))
        share = rng.choice((1, 1, 2, 4, 8))
        heads = kv_heads * share
        if heads > 32:
            continue
        rot = rng.choice((16, 32, D // 32 * 16, D, D))
        inter, norm = rng.random() < 0.5, rng.random() < 0.7
        page = rng.choice((8, 16, 32, 64, 128))
        softcap = rng.choice((0.0, 0.0, 30.0, 50.0))
        alibi = rng.random() < 0.3
        if kind == "rope":
            c = _rope("", _spread(rng, 1, 32768), heads, kv_heads, D, rot, dtype, inter, norm)
        elif kind == "append":
            B = _spread(rng, 1, 64)
            c = _append("", B, rng.choice((1, 1, _spread(rng, 1, 2048))), _spread(rng, 1, 4096) - 1, heads, kv_heads, D,
                        rot, page, dtype, inter, norm)
        elif kind == "attn":
            S, B = _spread(rng, 1, 16384), _spread(rng, 1, 64)
            backward = rng.random() < 0.6
            c = _attn("", B, S, heads, kv_heads, D, rng.choice(("causal", "docs", "prefix", "full")), dtype, softcap,
                      alibi, backward)
        else:
            longest = _spread(rng, 1, 32768)
            new = rng.choice((1, 1, 1, 2, 5))
            if new > longest:
                continue
            c = _paged("", _spread(rng, 1, 64), new, max(new, longest // rng.choice((1, 2, 64))), longest, heads, kv_heads,
                       D, page, dtype, softcap, alibi)
        del c["name"]
        if _fits(c):
            return c


def _fits(c):
    if c["kind"] == "rope":
        return c["T"] * (c["heads"] + c["kv_heads"]) * c["D"] <= 32768 * 32 * 128
    if c["kind"] == "append":
        return c["B"] * c["new"] <= 32768 and c["B"] * (c["past"] + c["new"]) * c["kv_heads"] * c["D"] <= 1 << 28
    if c["kind"] == "attn":
        scale = 4 if c["dtype"] == "f32" else 1
        return c["B"] * c["S"] <= 32768 and c["B"] * c["S"] ** 2 * c["heads"] * (4 if c["backward"] else 1) * scale <= LARGEST_PAIRS
    return c["B"] * c["longest"] * c["kv_heads"] * c["D"] * (2 if c["dtype"] == "f32" else 1) <= 64 * 32768 * 4 * 128


# ------------------------------------------------------------------ inputs --

def _documents(c):
    """(first, end, prefix) of the documents of each sequence, in tokens of that sequence, by the mask's kind.  Packed
    documents leave some tokens at the end of a sequence that belong to none and see nothing."""
    S = c["S"]
    if c["mask"] == "docs":
        rng, rows = random.Random(S * 1000 + c["B"]), []
        for _ in range(c["B"]):
            at, end, docs = 0, max(1, S - rng.randrange(0, S // 16 + 1)), []
            while at < end:
                n = min(end - at, _spread(rng, 1, max(1, S)))
                docs.append((at, at + n, 0))
                at += n
            rows.append(docs)
        return rows
    return [[(0, S, S // 3 if c["mask"] == "prefix" else 0)]] * c["B"]


def _intervals(c):
    """The keys [lo, hi) that each row sees, as int32 [B, S] in tokens of the row's own sequence."""
    S = c["S"]
    i = torch.arange(S, dtype=torch.int32)
    lo, hi = torch.zeros(c["B"], S, dtype=torch.int32), torch.zeros(c["B"], S, dtype=torch.int32)
    for b, docs in enumerate(_documents(c)):
        for first, end, prefix in docs:
            rows = i[first:end]
            lo[b, first:end] = first
            hi[b, first:end] = end if c["mask"] == "full" else torch.clamp(rows + 1, min=first + prefix)
    return lo, hi


def _lengths(c):
    """Cached tokens of each sequence, the new ones among them: spread evenly between the shortest and the longest."""
    B, a, z = c["B"], c["shortest"], c["longest"]
    return [z if B == 1 else a + (z - a) * ((b * 37) % B) // (B - 1) for b in range(B)]


def _slopes(heads):
    """One slope per head, a geometric series from 2^(-8/heads) down to 2^-8."""
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], dtype=torch.float32, device="cuda")


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _pages(g, B, per, n_pages):
    """A page table [B, per] of distinct pages in no order."""
    return torch.randperm(n_pages, generator=g, device="cuda")[:B * per].view(B, per).to(torch.int32)


def _tables(length, rot):
    """cos and sin of position x frequency, float32 [length, rot / 2], as a program keeps them."""
    f = BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(length, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cos(a).float(), torch.sin(a).float()


def prepare(case, seed):
    c, g = case, _generator(seed)
    dt, D, H, K = DTYPES[c["dtype"]], c["D"], c["heads"], c["kv_heads"]
    s = {"case": c}
    if c["kind"] in ("rope", "append"):
        T = c["T"] if c["kind"] == "rope" else c["B"] * c["new"]
        s["qkv"] = _normal(g, (T, (H + 2 * K) * D), dt)
        s["q_weight"], s["k_weight"] = ((1.0 + _normal(g, (D,), torch.float32, 0.1)) if c["norm"] else None
                                        for _ in range(2))
    if c["kind"] == "rope":
        # rows of sequences of at most 2048 tokens
        s["positions"] = (torch.arange(T, device="cuda") % 2048).to(torch.int32)
        s["cos"], s["sin"] = _tables(2048, c["rot"])
        s["dq"], s["dk"] = _normal(g, (T, H, D), dt), _normal(g, (T, K, D), dt)
        s["dqkv"] = torch.zeros_like(s["qkv"])
    elif c["kind"] == "append":
        length = c["past"] + c["new"]
        per = -(-length // c["page"])
        n_pages = c["B"] * per + 3
        s["cache"] = _normal(g, (n_pages, 2, K, c["page"], D), dt)
        table = _pages(g, c["B"], per, n_pages).long()
        at = torch.arange(c["past"], length, device="cuda")
        s["slots"] = (table[:, at // c["page"]] * c["page"] + at % c["page"]).reshape(-1)
        s["positions"] = at.to(torch.int32).repeat(c["B"])
        s["cos"], s["sin"] = _tables(length, c["rot"])
    elif c["kind"] == "attn":
        B, S = c["B"], c["S"]
        s["qkv"] = _normal(g, (B * S, (H + 2 * K) * D), dt)
        first = (torch.arange(B, dtype=torch.int32) * S)[:, None]
        lo, hi = _intervals(c)
        s["key_lo"], s["key_hi"] = ((t + first).reshape(-1).cuda() for t in (lo, hi))
        s["slopes"] = _slopes(H) if c["alibi"] else None
        if c["backward"]:
            s["do"] = _normal(g, (B * S, H, D), dt)
            s["dqkv"] = torch.zeros_like(s["qkv"])
    else:
        B, lengths = c["B"], _lengths(c)
        per = -(-c["longest"] // c["page"])
        n_pages = B * per + 3
        s["cache"] = _normal(g, (n_pages, 2, K, c["page"], D), dt)
        s["page_table"] = _pages(g, B, per, n_pages)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["q"] = _normal(g, (B * c["new"], H, D), dt)
        s["slopes"] = _slopes(H) if c["alibi"] else None
    return s


def _split(c, x):
    """The query, key and value columns of a Q/K/V row as [T, heads, D] views."""
    D, H, K = c["D"], c["heads"], c["kv_heads"]
    T = x.shape[0]
    return (x[:, :H * D].view(T, H, D), x[:, H * D:(H + K) * D].view(T, K, D), x[:, (H + K) * D:].view(T, K, D))


# -------------------------------------------------------------- plain forms --

def _partners(x, rot, interleaved):
    """The first and second elements of each rotated pair."""
    if interleaved:
        return x[..., 0:rot:2], x[..., 1:rot:2]
    return x[..., :rot // 2], x[..., rot // 2:rot]


def _rotated(x, cos, sin, rot, interleaved, back=False):
    a, b = _partners(x, rot, interleaved)
    if back:
        sin = -sin
    y = x.clone()
    ya, yb = _partners(y, rot, interleaved)
    ya.copy_(a * cos - b * sin)
    yb.copy_(b * cos + a * sin)
    return y


def _plain_heads(x, weight, cos, sin, rot, interleaved):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight
    return _rotated(x, cos, sin, rot, interleaved)


def _plain_heads_back(dy, x, weight, cos, sin, rot, interleaved):
    du = _rotated(dy.float(), cos, sin, rot, interleaved, back=True)
    if weight is None:
        return du, None
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    wdu = du * weight
    return r * (wdu - n * (n * wdu).mean(-1, keepdim=True)), (n * du).sum((0, 1))


def _plain_rope(s):
    c = s["case"]
    q, k, _ = _split(c, s["qkv"])
    cos, sin = (s[n][s["positions"].long()][:, None] for n in ("cos", "sin"))
    how = (cos, sin, c["rot"], c["interleaved"])
    out = {"q": _plain_heads(q, s["q_weight"], *how).to(q.dtype), "k": _plain_heads(k, s["k_weight"], *how).to(q.dtype)}
    dq, dqw = _plain_heads_back(s["dq"], q, s["q_weight"], *how)
    dk, dkw = _plain_heads_back(s["dk"], k, s["k_weight"], *how)
    T = q.shape[0]
    out["dqk"] = torch.cat([dq.reshape(T, -1), dk.reshape(T, -1)], 1).to(q.dtype)
    out.update(dq_weight=dqw, dk_weight=dkw)
    return out


def _plain_append(s):
    c = s["case"]
    q, k, v = _split(c, s["qkv"])
    cos, sin = (s[n][s["positions"].long()][:, None] for n in ("cos", "sin"))
    how = (cos, sin, c["rot"], c["interleaved"])
    page, off = s["slots"] // c["page"], s["slots"] % c["page"]
    s["cache"][page, 0, :, off] = _plain_heads(k, s["k_weight"], *how).to(k.dtype)
    s["cache"][page, 1, :, off] = v
    return {"q": _plain_heads(q, s["q_weight"], *how).to(q.dtype), "cache": s["cache"]}


def _plain_scores(c, q, k, slopes, at, keys):
    """Scores before the mask, and tanh of the capped ones: q [..., rows, D], k [..., keys, D] in float32."""
    z = (q * c["D"] ** -0.5) @ k.transpose(-1, -2).contiguous()
    t = None
    if c["softcap"]:
        t = torch.tanh(z / c["softcap"])
        z = t * c["softcap"]
    if slopes is not None:
        z = z - slopes[:, None, None] * (at[..., :, None] - keys).abs()
    return z, t


def _plain_softmax(z, seen):
    """exp of the scores over the keys seen, their sum, and its logarithm: zero and minus infinity for an empty row."""
    z = z.masked_fill(~seen, -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(z - m)
    total = p.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    return p / torch.where(total > 0, total, 1.0), lse


def _plain_attn(s):
    c = s["case"]
    B, S, H, K, D = c["B"], c["S"], c["heads"], c["kv_heads"], c["D"]
    g = H // K

    def heads(x, n):   # [B, heads, S, D] in float32, a shared key head once for each of its query heads
        return x.float().view(B, S, n, D).transpose(1, 2).repeat_interleave(H // n, 1)

    qs, ks, vs = _split(c, s["qkv"])
    q, k, v = heads(qs, H), heads(ks, K), heads(vs, K)
    first = (torch.arange(B, device="cuda") * S)[:, None]
    lo, hi = s["key_lo"].view(B, S) - first, s["key_hi"].view(B, S) - first
    j = torch.arange(S, device="cuda")
    seen = ((j >= lo[..., None]) & (j < hi[..., None]))[:, None]
    z, t = _plain_scores(c, q, k, s["slopes"], j, j)
    p, lse = _plain_softmax(z, seen)
    o = p @ v
    rows = lambda x: x.transpose(1, 2).reshape(B * S, -1, D)  # noqa: E731
    out = {"o": rows(o).to(qs.dtype), "lse": lse[..., 0].transpose(0, 1).reshape(H, B * S)}
    if not c["backward"]:
        return out
    do = heads(s["do"], H)
    dv = p.transpose(-1, -2).contiguous() @ do
    dz = p * (do @ v.transpose(-1, -2).contiguous() - (do * o).sum(-1, keepdim=True)) * D ** -0.5
    if t is not None:
        dz = dz * (1.0 - t * t)
    dq, dk = dz @ k, dz.transpose(-1, -2).contiguous() @ q
    shared = lambda x: x.view(B, K, g, S, D).sum(2)  # noqa: E731
    out["dqkv"] = torch.cat([rows(x) for x in (dq, shared(dk), shared(dv))], 1).to(qs.dtype).view(B * S, -1)
    return out


def _plain_paged(s):
    c = s["case"]
    B, n, H, K, D, page = c["B"], c["new"], c["heads"], c["kv_heads"], c["D"], c["page"]
    table = s["page_table"].long()
    L = table.shape[1] * page
    held = s["cache"][table]   # [B, pages, 2, K, page, D]
    k, v = (held[:, :, i].float().transpose(1, 2).reshape(B, K, 1, L, D) for i in (0, 1))
    j = torch.arange(L, device="cuda")
    at = s["lengths"][:, None] - n + torch.arange(n, device="cuda")   # [B, n]
    seen = (j <= at[..., None])[:, None, None]
    q = s["q"].float().view(B, n, K, H // K, D).permute(0, 2, 3, 1, 4)   # [B, K, heads that share, n, D]
    slopes = None if s["slopes"] is None else s["slopes"].view(K, H // K)
    z, _ = _plain_scores(c, q.reshape(B, K, -1, D)[:, :, None], k, None, at, j)
    z = z.view(B, K, H // K, n, L)
    if slopes is not None:
        z = z - slopes[..., None, None] * (at[:, None, None, :, None] - j).abs()
    p, _ = _plain_softmax(z, seen)
    o = p.view(B, K, 1, -1, L) @ v
    return {"o": o.view(B, K, H // K, n, D).permute(0, 3, 1, 2, 4).reshape(B * n, H, D).to(s["q"].dtype)}


# ------------------------------------------------------------------- passes --

def run(state):
    s, c = state, state["case"]
    if not own:
        return {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn, "paged": _plain_paged}[c["kind"]](s)
    from paper_2603_06492_amd import attention as na
    if c["kind"] in ("rope", "append"):
        how = dict(heads=c["heads"], kv_heads=c["kv_heads"], eps=EPS, interleaved=c["interleaved"])
        given = (s["qkv"], s["q_weight"], s["k_weight"], s["cos"], s["sin"], s["positions"])
        if c["kind"] == "append":
            return {"q": na.noble_kv_append(*given, s["slots"], s["cache"], **how), "cache": s["cache"]}
        q, k = na.noble_qk_rope_fwd(*given, **how)
        dqkv, dqw, dkw = na.noble_qk_rope_bwd(s["dq"], s["dk"], *given, dqkv=s["dqkv"], **how)
        return {"q": q, "k": k, "dqk": dqkv[:, :(c["heads"] + c["kv_heads"]) * c["D"]], "dq_weight": dqw,
                "dk_weight": dkw}
    if c["kind"] == "paged":
        return {"o": na.noble_attn_paged(s["q"], s["cache"], s["page_table"], s["lengths"], s["slopes"],
                                         softcap=c["softcap"])}
    q, k, v = _split(c, s["qkv"])
    mask = (s["key_lo"], s["key_hi"], s["slopes"])
    o, lse = na.noble_attn_fwd(q, k, v, *mask, softcap=c["softcap"])
    out = {"o": o, "lse": lse}
    if c["backward"]:
        dq, dk, dv = _split(c, s["dqkv"])
        na.noble_attn_bwd(s["do"], q, k, v, o, lse, *mask, softcap=c["softcap"], dq=dq, dk=dk, dv=dv)
        out["dqkv"] = s["dqkv"]
    return out


def _pairs(c):
    """(row, key) pairs of one head that an attention case's mask lets through."""
    if c["kind"] == "paged":
        return sum(sum(n - c["new"] + 1 + i for i in range(c["new"])) for n in _lengths(c))
    lo, hi = _intervals(c)
    return int((hi.long() - lo.long()).clamp(min=0).sum())


def work(case):
    c = case
    D, H, K = c["D"], c["heads"], c["kv_heads"]
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rope":
        n = c["T"] * (H + K) * D
        # x read and q, k written; dq, dk and x read and their gradient written; the tables once
        return {"bytes": float(n * es * 5 + c["T"] * 4 + min(c["T"], 2048) * c["rot"] * 4), "flops": 30.0 * n}
    if c["kind"] == "append":
        T = c["B"] * c["new"]
        return {"bytes": float(T * (H + 2 * K) * D * es * 2 + T * 12 + c["new"] * c["rot"] * 4),
                "flops": 10.0 * T * (H + K) * D}
    pairs = _pairs(c) * H
    if c["kind"] == "paged":
        rows, keys = c["B"] * c["new"], sum(_lengths(c))
        return {"bytes": float(keys * 2 * K * D * es + 2 * rows * H * D * es + keys / c["page"] * 4),
                "flops": 4.0 * D * pairs}
    T = c["B"] * c["S"]
    nbytes = T * (2 * H + 2 * K) * D * es + T * H * 4 + T * 8
    if c["backward"]:
        nbytes += T * (4 * H + 4 * K) * D * es + T * H * 4
    return {"bytes": float(nbytes), "flops": (14.0 if c["backward"] else 4.0) * D * pairs}


# -------------------------------------------------------------------- exact --

def _exact_rotation(u, position, rot, interleaved, back=False):
    """Each pair of u [T, heads, D] as a complex number, times exp(i position frequency) or its conjugate, the angle's
    cosine and sine as the program's tables hold them."""
    table = torch.complex(*(t.double() for t in position))[:, None]   # [T, 1, rot / 2]
    if back:
        table = table.conj()
    pairs = u[..., :rot].reshape(*u.shape[:-1], rot // 2, 2) if interleaved else \
        u[..., :rot].reshape(*u.shape[:-1], 2, rot // 2).transpose(-1, -2)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * table)
    if not interleaved:
        turned = turned.transpose(-1, -2)
    return torch.cat([turned.reshape(*u.shape[:-1], rot), u[..., rot:]], -1)


def _exact_heads(s, c, x, w, dy=None):
    at = s["positions"].long()
    angle = (s["cos"][at], s["sin"][at])
    x = x.double().requires_grad_(dy is not None)
    w = None if w is None else w.double().requires_grad_(dy is not None)
    u = x if w is None else x / (x.square().sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * w
    y = _exact_rotation(u, angle, c["rot"], c["interleaved"])
    if dy is None:
        return y
    g = torch.autograd.grad(y, [x] if w is None else [x, w], dy.double())
    return y.detach(), g[0], None if w is None else g[1]


def _exact_attention(c, q, k, v, lo, hi, slopes, at, do=None):
    """One group of query heads [heads, rows, D] over one key head [keys, D]: o, lse and, for a given do, the gradients."""
    need = do is not None
    q, k, v = (x.double().requires_grad_(need) for x in (q, k, v))
    z = q @ k.t().contiguous() / math.sqrt(c["D"])
    if c["softcap"]:
        z = c["softcap"] * torch.tanh(z / c["softcap"])
    j = torch.arange(k.shape[0], device="cuda")
    if slopes is not None:
        z = z - slopes.double()[:, None, None] * (at[:, None] - j[None]).abs()
    hidden = (j[None] < lo[:, None]) | (j[None] >= hi[:, None])
    empty = hidden.all(-1)
    z = torch.where(hidden & ~empty[:, None], -math.inf, z)   # an empty row is taken out below
    lse = torch.logsumexp(z, -1)
    o = torch.exp(z - lse[..., None]) @ v
    o = torch.where(empty[:, None], 0.0, o)
    grads = torch.autograd.grad(o, [q, k, v], do.double()) if need else None
    return o.detach(), torch.where(empty, -math.inf, lse).detach(), grads


def exact(case, seed):
    c, s = case, prepare(case, seed)
    D, H, K = c["D"], c["heads"], c["kv_heads"]
    g = H // K
    if c["kind"] == "rope":
        q, k, _ = _split(c, s["qkv"])
        yq, dq, dqw = _exact_heads(s, c, q, s["q_weight"], s["dq"])
        yk, dk, dkw = _exact_heads(s, c, k, s["k_weight"], s["dk"])
        return {"q": yq, "k": yk, "dqk": torch.cat([dq.flatten(1), dk.flatten(1)], 1), "dq_weight": dqw, "dk_weight": dkw}
    if c["kind"] == "append":
        q, k, v = _split(c, s["qkv"])
        cache = s["cache"].double()
        for t, slot in enumerate(zip(_exact_heads(s, c, k, s["k_weight"]), v.double(), s["slots"].tolist())):
            kt, vt, at = slot
            cache[at // c["page"], 0, :, at % c["page"]] = kt
            cache[at // c["page"], 1, :, at % c["page"]] = vt
        return {"q": _exact_heads(s, c, q, s["q_weight"]), "cache": cache}
    if c["kind"] == "attn":
        B, S = c["B"], c["S"]
        q, k, v = _split(c, s["qkv"])
        o = torch.empty(B * S, H, D, dtype=torch.float64, device="cuda")
        lse = torch.empty(H, B * S, dtype=torch.float64, device="cuda")
        grad = torch.empty(s["qkv"].shape, dtype=torch.float64, device="cuda") if c["backward"] else None
        at = torch.arange(S, device="cuda")
        for b in range(B):
            r = slice(b * S, (b + 1) * S)
            lo, hi = (s[n][r].long() - b * S for n in ("key_lo", "key_hi"))
            for h in range(K):
                for x in range(h * g, (h + 1) * g) if S > 4096 else [None]:   # one query head at a time where it is long
                    hs = slice(h * g, (h + 1) * g) if x is None else slice(x, x + 1)
                    sl = None if s["slopes"] is None else s["slopes"][hs]
                    do = s["do"][r, hs].transpose(0, 1) if c["backward"] else None
                    oo, ll, gr = _exact_attention(c, q[r, hs].transpose(0, 1), k[r, h], v[r, h], lo, hi, sl, at, do)
                    o[r, hs], lse[hs, r] = oo.transpose(0, 1), ll
                    if gr is not None:
                        dq, dk, dv = _split(c, grad)
                        dq[r, hs] = gr[0].transpose(0, 1)
                        for part, new in ((dk, gr[1]), (dv, gr[2])):
                            part[r, h] = new if x in (None, h * g) else part[r, h] + new
        out = {"o": o, "lse": lse}
        return {**out, "dqkv": grad} if c["backward"] else out
    n, o = c["new"], torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(_lengths(c)):
        pages = s["page_table"][b].long()
        for h in range(K):
            kv = [s["cache"][pages, i, h].reshape(-1, D)[:length] for i in (0, 1)]
            at = torch.arange(length - n, length, device="cuda")
            hs, r = slice(h * g, (h + 1) * g), slice(b * n, (b + 1) * n)
            sl = None if s["slopes"] is None else s["slopes"][hs]
            oo, _, _ = _exact_attention(c, s["q"][r, hs].transpose(0, 1), *kv, torch.zeros_like(at), at + 1, sl, at)
            o[r, hs] = oo.transpose(0, 1)
    return {"o": o}
