"""Performance cases of decoding over the paged cache: a tree of drafted tokens, blocks that a cheap score selects, and a
cache that is kept short by the attention weight its tokens have received.

``kind`` names the operator:

* ``tree``:   the rows of a tree of drafted tokens, and their attention over the cache;
* ``accept``: the accepted branch of each sequence's tree, moved to the front of the tree's place in the cache;
* ``sparse``: means of the pages that the new tokens are in, selection of pages for each new token and key head, and
  attention over the selected pages;
* ``weigh``:  attention over the cache that adds up the weight that every cached token receives;
* ``evict``:  selection of each key head's heaviest tokens, which then fill the first places of the cache.

Where ``own`` is false, ``run`` computes the operators from their formulas in float32 (scores that only select, and the
means that they come from, in float64).
"""

import functools
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGEST_CACHE = 64 * 32768 * 4 * 128   # elements of keys that a drawn case's sequences may hold


def _tree(name, B, new, shortest, longest, heads, kv_heads, D, page, dtype="bf16", softcap=0.0, alibi=False):
    return dict(name=name, kind="tree", B=B, new=new, shortest=shortest, longest=longest, heads=heads, kv_heads=kv_heads,
                D=D, page=page, dtype=dtype, softcap=softcap, alibi=alibi)


def _accept(name, B, new, shortest, longest, kv_heads, D, page, dtype="bf16"):
    return dict(name=name, kind="accept", B=B, new=new, shortest=shortest, longest=longest, heads=kv_heads,
                kv_heads=kv_heads, D=D, page=page, dtype=dtype)


def _sparse(name, B, new, shortest, longest, heads, kv_heads, D, page, count, dtype="bf16", softcap=0.0, sink=1, local=2):
    return dict(name=name, kind="sparse", B=B, new=new, shortest=shortest, longest=longest, heads=heads,
                kv_heads=kv_heads, D=D, page=page, count=count, dtype=dtype, softcap=softcap, sink=sink, local=local)


def _weigh(name, B, new, shortest, longest, heads, kv_heads, D, page, dtype="bf16", softcap=0.0, alibi=False):
    return dict(name=name, kind="weigh", B=B, new=new, shortest=shortest, longest=longest, heads=heads,
                kv_heads=kv_heads, D=D, page=page, dtype=dtype, softcap=softcap, alibi=alibi)


def _evict(name, B, shortest, longest, kv_heads, D, page, keep, dtype="bf16", sink=4, recent=64):
    return dict(name=name, kind="evict", B=B, new=1, shortest=shortest, longest=longest, heads=kv_heads,
                kv_heads=kv_heads, D=D, page=page, keep=keep, dtype=dtype, sink=sink, recent=recent)


def listed():
    return [
        # four drafted tokens of one sequence: the smallest call of speculative decoding
        _tree("tree4_1000", 1, 4, 1000, 1000, 16, 16, 128, 16),
        # a batch of very different lengths, trees of up to 32 tokens, capped scores
        _tree("tree32_ragged_cap", 16, 32, 130, 8192, 16, 16, 128, 16, softcap=30.0),
        # a small batch of long sequences, shared key heads, trees of up to 64 tokens
        _tree("tree64_long", 8, 64, 16384, 32768, 16, 4, 128, 64),
        # the branch of four drafted tokens that one sequence keeps
        _accept("accept4", 1, 4, 1000, 1000, 16, 128, 16),
        # a large batch's accepted branches of trees of 64
        _accept("accept64", 64, 64, 1000, 4096, 16, 128, 16),
        # one token of one long sequence: 32 of its 512 pages
        _sparse("sparse1_32768", 1, 1, 32768, 32768, 16, 4, 128, 64, 32),
        # a toy model in full precision, odd lengths, small pages, three new tokens a sequence
        _sparse("sparse_f32_odd", 5, 3, 333, 2047, 4, 2, 64, 16, 24, dtype="f32"),
        # 64 long sequences, shared key heads, a cache of 4.3 GB, an eighth of it read
        _sparse("sparse64_long", 64, 1, 16384, 32768, 16, 4, 128, 64, 64),
        # one token of 16 sequences of very different lengths, every key head's weights kept
        _weigh("weigh16_ragged", 16, 1, 130, 8192, 16, 16, 128, 16),
        # 64 long sequences, shared key heads
        _weigh("weigh64_long", 64, 1, 16384, 32768, 16, 4, 128, 64),
        # one sequence of a small model, a quarter of its tokens stay
        _evict("evict1_4096", 1, 4096, 4096, 8, 64, 16, 1024),
        # 64 long sequences of shared key heads, each cut to 8192 tokens
        _evict("evict64_long", 64, 16384, 32768, 4, 128, 64, 8192),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges: up to 64 sequences of 1 to 32768 tokens, 1 to 64 new ones, heads of 32 to
    128, key heads shared by 1 to 8 query heads, pages of 8 to 128 tokens."""
    while True:
        kind = rng.choice(("tree", "tree", "sparse", "sparse", "weigh", "weigh", "evict", "accept"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        D = rng.choice((32, 64, 64, 80, 96, 128, 128, 128))
        kv_heads = rng.choice((1, 2, 4, 8, 12, 16))
        heads = kv_heads * rng.choice((1, 1, 2, 4, 8))
        page = rng.choice((8, 16, 32, 64, 128))
        softcap = rng.choice((0.0, 0.0, 30.0, 50.0))
        alibi = rng.random() < 0.3
        B, longest = _spread(rng, 1, 64), _spread(rng, 1, 32768)
        new = {"tree": _spread(rng, 1, 64), "accept": _spread(rng, 1, 64), "sparse": rng.choice((1, 1, 1, 2, 5)),
               "weigh": rng.choice((1, 1, 1, 2, 5, _spread(rng, 1, 64))), "evict": 1}[kind]
        shortest = max(new, longest // rng.choice((1, 2, 64)))
        if heads > 32 or new > longest:
            continue
        if kind == "tree":
            c = _tree("", B, new, shortest, longest, heads, kv_heads, D, page, dtype, softcap, alibi)
        elif kind == "accept":
            c = _accept("", B, new, shortest, longest, kv_heads, D, page, dtype)
        elif kind == "sparse":
            sink, local = rng.choice((0, 1, 2)), rng.choice((1, 2, 4))
            c = _sparse("", B, new, shortest, longest, heads, kv_heads, D, page,
                        sink + local + _spread(rng, 1, max(1, longest // page // 2)), dtype, softcap, sink, local)
        elif kind == "weigh":
            c = _weigh("", B, new, shortest, longest, heads, kv_heads, D, page, dtype, softcap, alibi)
        else:
            sink, recent = rng.choice((0, 1, 4)), rng.choice((0, 1, 32, 64))
            c = _evict("", B, shortest, longest, kv_heads, D, page, sink + recent + _spread(rng, 1, max(1, longest // 2)),
                       dtype, sink, recent)
        del c["name"]
        if _fits(c):
            return c


def _fits(c):
    scale = 2 if c["dtype"] == "f32" else 1
    if c["B"] * c["longest"] * c["kv_heads"] * c["D"] * scale > LARGEST_CACHE:
        return False
    # the plain forms hold every row's scores, or the selected keys of every row, at once
    pairs = c["B"] * c["new"] * c["longest"] * c["heads"]
    if c["kind"] == "sparse":
        return c["B"] * c["new"] * c["count"] * c["page"] * c["kv_heads"] * c["D"] <= LARGEST_CACHE // 4
    return c["kind"] in ("accept", "evict") or pairs * scale <= 8 * 64 * 32768 * 16


# ------------------------------------------------------------------ inputs --

def _lengths(c):
    """Cached tokens of each sequence, the new ones among them: spread evenly between the shortest and the longest."""
    B, a, z = c["B"], c["shortest"], c["longest"]
    return [z if B == 1 else a + (z - a) * ((b * 37) % B) // (B - 1) for b in range(B)]


def _parents(c, seed):
    """A tree of each sequence: a node's parent is one of those shortly before it, or -1, the last token before the tree;
    some sequences drafted fewer nodes (-2: none)."""
    rng, rows = random.Random(seed), []
    for _ in range(c["B"]):
        nodes = rng.randint((c["new"] + 1) // 2, c["new"])
        rows.append([max(-1, i - 1 - int(rng.expovariate(0.4))) if i < nodes else -2 for i in range(c["new"])])
    return rows


def _branches(c, parents, seed):
    """The accepted branch of each sequence: the nodes from the root to one of the tree's, in order, then -1."""
    rng, rows = random.Random(seed + 1), []
    for p in parents:
        n = rng.randrange(sum(x > -2 for x in p))
        path = []
        while n >= 0:
            path.insert(0, n)
            n = p[n]
        rows.append(path + [-1] * (c["new"] - len(path)))
    return rows


def _slopes(heads):
    """One slope per head, a geometric series from 2^(-8/heads) down to 2^-8."""
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], dtype=torch.float32, device="cuda")


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _ints(rows):
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda").manual_seed(int(seed))
    dt, D, H, K, B, page = DTYPES[c["dtype"]], c["D"], c["heads"], c["kv_heads"], c["B"], c["page"]
    per = -(-c["longest"] // page)
    n_pages = B * per + 3
    s = {"case": c}
    # pages that differ in the mean of their keys, as pages about different matters do
    s["cache"] = torch.empty((n_pages, 2, K, page, D), dtype=dt, device="cuda")
    s["cache"].normal_(generator=g)
    s["cache"][:, 0] += _normal(g, (n_pages, K, 1, D), dt, 0.5)
    s["page_table"] = torch.randperm(n_pages, generator=g, device="cuda")[:B * per].view(B, per).to(torch.int32)
    s["lengths"] = _ints(_lengths(c))
    if c["kind"] in ("tree", "sparse", "weigh"):
        s["q"] = _normal(g, (B * c["new"], H, D), dt)
        s["slopes"] = _slopes(H) if c.get("alibi") else None
    if c["kind"] in ("tree", "accept"):
        parents = _parents(c, seed)
        s["parents"] = _ints(parents)
        if c["kind"] == "accept":
            s["kept"] = _ints(_branches(c, parents, seed))[:, None]
            s["start"] = s["lengths"] - c["new"]
    elif c["kind"] == "sparse":
        s["means"] = s["cache"][:, 0].mean(2, dtype=torch.float64).to(dt)
    elif c["kind"] == "weigh":
        # what some twenty rows before have left
        s["weights"] = torch.rand((B, K, per * page), generator=g, device="cuda") ** 4 * (100.0 * H / K / c["longest"])
        s["weighed"] = torch.zeros_like(s["weights"])
    else:
        # many tokens have not been attended to at all
        s["weights"] = (torch.rand((B, K, per * page), generator=g, device="cuda") - 0.25).clamp(min=0.0) ** 4
    return s


# -------------------------------------------------------------- plain forms --

def _held(s):
    """Keys and values of every sequence, float32 [B, K, tokens, D], and the tokens' numbers."""
    c = s["case"]
    held = s["cache"][s["page_table"].long()]   # [B, pages, 2, K, page, D]
    B, per = held.shape[:2]
    k, v = (held[:, :, i].float().transpose(1, 2).reshape(B, c["kv_heads"], per * c["page"], c["D"]) for i in (0, 1))
    return k, v, torch.arange(per * c["page"], device="cuda")


def _rows_of_heads(c, q):
    """q [B n, H, D] as float32 [B, K, heads that share, n, D]."""
    B, n, H, K, D = c["B"], c["new"], c["heads"], c["kv_heads"], c["D"]
    return q.float().view(B, n, K, H // K, D).permute(0, 2, 3, 1, 4)


def _softmax(z, seen):
    """exp of the scores over the keys seen, divided by their sum: zeros for a row that sees none."""
    z = z.masked_fill(~seen, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, 1.0)


def _attend(s, k, v, seen, distance):
    """o [B n, H, D] and the probabilities [B, K, heads that share, n, keys] of k, v [B, K, keys, D]; seen and distance
    [B, n, keys]."""
    c = s["case"]
    B, n, H, K, D = c["B"], c["new"], c["heads"], c["kv_heads"], c["D"]
    q = _rows_of_heads(c, s["q"]).reshape(B, K, -1, D) * D ** -0.5
    z = (q @ k.transpose(-1, -2).contiguous()).view(B, K, H // K, n, -1)
    if c["softcap"]:
        z = c["softcap"] * torch.tanh(z / c["softcap"])
    if s["slopes"] is not None:
        z = z - s["slopes"].view(K, H // K)[..., None, None] * distance[:, None, None]
    p = _softmax(z, seen[:, None, None])
    o = (p.view(B, K, -1, p.shape[-1]) @ v).view(B, K, H // K, n, D)
    return o.permute(0, 3, 1, 2, 4).reshape(B * n, H, D).to(s["q"].dtype), p


def _plain_tree(s):
    c, parents = s["case"], s["parents"].long()
    B, n = parents.shape
    i = torch.arange(n, device="cuda")
    child = (parents[..., None] == i).float() * (parents < i)[..., None]   # [node, its parent]
    steps = max(1, (n - 1).bit_length())
    line = functools.reduce(lambda m, _: (m @ m).clamp(max=1.0), range(steps), child + torch.eye(n, device="cuda"))
    line = line * ((line @ (parents == -1).float()[..., None]) > 0)   # a node whose line does not begin at the root is none
    depth = (line.sum(-1) - 1).long()   # -1: no node
    first = s["lengths"].long()[:, None] - n   # tokens before the tree
    k, v, j = _held(s)
    seen = (j < first[..., None]) & (depth >= 0)[..., None]
    at = first + depth
    place = (j - first[..., None]).clamp(0, n - 1).expand(B, n, -1)
    in_tree = (j >= first[..., None]) & (j < s["lengths"][:, None, None])
    seen = seen | (in_tree & (line.gather(2, place) > 0))
    where = torch.where(in_tree[:, 0], at.gather(1, place[:, 0]), j)   # position of every key
    o, _ = _attend(s, k, v, seen, (at[..., None] - where[:, None]).abs())
    return {"o": o, "positions": torch.where(depth >= 0, at, 0).to(torch.int32)}


def _plain_accept(s):
    c, kept = s["case"], s["kept"][:, 0].long()
    place = torch.arange(kept.shape[1], device="cuda").expand_as(kept)
    b, i = torch.nonzero(kept >= 0, as_tuple=True)
    first = s["start"].long()[b]
    src, dst = first + kept[b, i], first + place[b, i]
    page = lambda t: s["page_table"].long()[b, t // c["page"]]  # noqa: E731
    s["cache"][page(dst), :, :, dst % c["page"]] = s["cache"][page(src), :, :, src % c["page"]]
    return {"cache": s["cache"]}


def _plain_means(s):
    """The means of the pages that hold each sequence's last new tokens, over the tokens that it holds."""
    c, page = s["case"], s["case"]["page"]
    lengths = s["lengths"].long()[:, None]
    touched = (lengths - c["new"]) // page + torch.arange((c["new"] + page - 2) // page + 1, device="cuda")
    b, t = torch.nonzero(touched * page < lengths, as_tuple=True)
    number = touched[b, t]
    pages = s["page_table"].long()[b, number]
    held = (lengths[b, 0] - number * page).clamp(max=page)
    within = torch.arange(page, device="cuda") < held[:, None]
    k = s["cache"][pages, 0].double() * within[:, None, :, None]
    s["means"][pages] = (k.sum(2) / held[:, None, None]).to(s["means"].dtype)
    return s["means"]


def _plain_selection(s):
    c = s["case"]
    B, n, H, K, D, page = c["B"], c["new"], c["heads"], c["kv_heads"], c["D"], c["page"]
    means = s["means"][s["page_table"].long()].double().permute(0, 2, 3, 1).contiguous()   # [B, K, D, blocks]
    q = s["q"].double().view(B, n, K, H // K, D).sum(3).transpose(1, 2)
    score = (q @ means).transpose(1, 2)   # [B, n, K, blocks]
    block = torch.arange(means.shape[-1], device="cuda")
    at = (s["lengths"].long()[:, None] - n + torch.arange(n, device="cuda")) // page
    at = at[:, :, None, None]
    always = (block < c["sink"]) | ((block > at - c["local"]) & (block <= at))
    score = score.masked_fill(always, math.inf).masked_fill(block > at, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :c["count"]]
    none = means.shape[-1]
    best = torch.where(best <= at, best, none).sort(-1).values
    best = torch.nn.functional.pad(best, (0, c["count"] - best.shape[-1]), value=none)
    return torch.where(best < none, best, -1)


def _plain_sparse(s):
    c = s["case"]
    B, n, H, K, D, page = c["B"], c["new"], c["heads"], c["kv_heads"], c["D"], c["page"]
    means = _plain_means(s)
    chosen = _plain_selection(s)   # [B, n, K, count]
    b = torch.arange(B, device="cuda")[:, None, None, None]
    pages = s["page_table"].long()[b, chosen.clamp(min=0)]
    head = torch.arange(K, device="cuda")[:, None]
    k, v = (s["cache"][pages, i, head].float().reshape(B, n, K, -1, D) for i in (0, 1))
    keys = (chosen[..., None] * page + torch.arange(page, device="cuda")).view(B, n, K, -1)
    at = s["lengths"].long()[:, None] - n + torch.arange(n, device="cuda")
    seen = (keys >= 0) & (keys <= at[:, :, None, None])
    q = s["q"].float().view(B, n, K, H // K, D) * D ** -0.5
    z = q @ k.transpose(-1, -2).contiguous()
    if c["softcap"]:
        z = c["softcap"] * torch.tanh(z / c["softcap"])
    o = _softmax(z, seen[..., None, :]) @ v
    return {"o": o.reshape(B * n, H, D).to(s["q"].dtype), "means": means,
            "chosen": chosen.view(B * n, K, -1).to(torch.int32)}


def _plain_weigh(s):
    c = s["case"]
    k, v, j = _held(s)
    lengths = s["lengths"].long()[:, None]
    at = lengths - c["new"] + torch.arange(c["new"], device="cuda")
    o, p = _attend(s, k, v, j <= at[..., None], (at[..., None] - j).abs())
    old = torch.where((j < lengths - c["new"])[:, None], s["weights"], 0.0)
    s["weighed"].copy_(torch.where((j < lengths)[:, None], old + p.sum((2, 3)), s["weighed"]))
    return {"o": o, "weights": s["weighed"]}


def _plain_evict(s):
    c = s["case"]
    page, keep = c["page"], c["keep"]
    j = torch.arange(s["weights"].shape[2], device="cuda")
    lengths = s["lengths"].long()[:, None, None]
    always = (j < c["sink"]) | (j >= lengths - c["recent"])
    rank = s["weights"].masked_fill(always, math.inf).masked_fill(j >= lengths, -math.inf)
    none = j.shape[0]
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    best = torch.where(best < lengths, best, none).sort(-1).values
    best = torch.nn.functional.pad(best, (0, keep - best.shape[-1]), value=none)
    kept = torch.where(best < none, best, -1)
    weights = torch.where(kept >= 0, s["weights"].gather(2, best.clamp(max=none - 1)), 0.0)
    b, h, i = torch.nonzero(kept >= 0, as_tuple=True)
    src = kept[b, h, i]
    where = lambda t: s["page_table"].long()[b, t // page]  # noqa: E731
    s["cache"][where(i), :, h, i % page] = s["cache"][where(src), :, h, src % page]
    return {"kept": kept.to(torch.int32), "weights": weights, "cache": s["cache"]}


# ------------------------------------------------------------------- passes --

def run(state):
    s, c = state, state["case"]
    if not own:
        return {"tree": _plain_tree, "accept": _plain_accept, "sparse": _plain_sparse, "weigh": _plain_weigh,
                "evict": _plain_evict}[c["kind"]](s)
    from paper_2603_06492_amd import decoding as nd
    cache = (s["cache"], s["page_table"], s["lengths"])
    if c["kind"] == "tree":
        seen, depths, positions = nd.noble_tree_rows(s["parents"], s["lengths"])
        return {"o": nd.noble_attn_tree(s["q"], *cache, seen, depths, s["slopes"], softcap=c["softcap"]),
                "positions": positions}
    if c["kind"] == "accept":
        return {"cache": nd.noble_cache_keep(s["cache"], s["page_table"], s["kept"], s["start"])}
    if c["kind"] == "sparse":
        nd.noble_page_means(*cache, c["new"], s["means"])
        chosen = nd.noble_block_select(s["q"], s["means"], s["page_table"], s["lengths"], c["count"], page=c["page"],
                                       sink=c["sink"], local=c["local"])
        return {"o": nd.noble_attn_blocks(s["q"], *cache, chosen, s["slopes"], softcap=c["softcap"]), "means": s["means"],
                "chosen": chosen}
    if c["kind"] == "weigh":
        o, _ = nd.noble_attn_weigh(s["q"], *cache, s["weights"], s["slopes"], softcap=c["softcap"], out=s["weighed"])
        return {"o": o, "weights": s["weighed"]}
    kept, weights = nd.noble_evict_select(s["weights"], s["lengths"], c["keep"], sink=c["sink"], recent=c["recent"])
    return {"kept": kept, "weights": weights, "cache": nd.noble_cache_keep(s["cache"], s["page_table"], kept)}


def work(case):
    c = case
    D, H, K, B, n, page = c["D"], c["heads"], c["kv_heads"], c["B"], c["new"], c["page"]
    es = 2 if c["dtype"] == "bf16" else 4
    lengths = _lengths(c)
    token = 2 * K * D * es   # a token's keys and values
    rows = 2 * B * n * H * D * es   # q and o
    if c["kind"] == "accept":
        moved = sum(p >= 0 and p != i for row in _branches(c, _parents(c, 1), 1) for i, p in enumerate(row))
        return {"bytes": float(max(1, moved) * token * 2 + B * n * 4 + B * 8), "flops": 0.0}
    if c["kind"] == "evict":
        kept = [min(x, c["keep"]) for x in lengths]
        moved = sum(m - min(m, c["sink"]) for m, x in zip(kept, lengths) if x > c["keep"])
        return {"bytes": float(sum(lengths) * K * 4 + sum(kept) * K * 8 + moved * token * 2 + B * 4), "flops": 0.0}
    if c["kind"] == "sparse":
        own_page = [[t // page for t in range(x - n, x)] for x in lengths]
        blocks = sum(max(p) + 1 for p in own_page)
        # a key head's chosen pages, each once for each new token, and the part of its own page that is held
        read = sum(min(c["count"], p + 1) * page for row in own_page for p in row)
        read -= sum(page - 1 - t % page for x in lengths for t in range(x - n, x))
        touched = sum((max(p) - min(p) + 1) * page for p in own_page)
        return {"bytes": float(read * token + touched * K * D * es + blocks * K * D * es + rows + B * n * K * c["count"] * 4),
                "flops": 4.0 * D * read * H + 2.0 * D * blocks * n * K}
    keys, pairs = sum(lengths), sum(sum(range(x - n + 1, x + 1)) for x in lengths)
    if c["kind"] == "tree":
        pairs = sum((x - n) * n + n for x in lengths)   # the tree's own pairs are few
        return {"bytes": float(keys * token + rows + B * n * 8), "flops": 4.0 * D * pairs * H}
    return {"bytes": float(keys * token + rows + keys * K * 8), "flops": 4.0 * D * pairs * H}


# -------------------------------------------------------------------- exact --

def _exact_rows(c, q, k, v, seen, slopes, away):
    """o [heads, rows, D] and the probabilities of one group of query heads [heads, rows, D] over keys [keys, D]."""
    z = q.double() @ k.double().t().contiguous() / math.sqrt(c["D"])
    if c["softcap"]:
        z = c["softcap"] * torch.tanh(z / c["softcap"])
    if slopes is not None:
        z = z - slopes.double()[:, None, None] * away
    some = seen.any(-1)[..., None]
    z = torch.where(seen | ~some, z, -math.inf)   # a row that sees nothing is taken out below
    p = torch.where(some, torch.exp(z - torch.logsumexp(z, -1, keepdim=True)), 0.0)
    return p @ v.double(), p


def _sequence(s, b, length, h):
    """Keys and values of one key head of one sequence."""
    pages = s["page_table"][b].long()
    return [s["cache"][pages, i, h].reshape(-1, s["case"]["D"])[:length] for i in (0, 1)]


def _exact_heads(s, b, h):
    c = s["case"]
    g, n = c["heads"] // c["kv_heads"], c["new"]
    rows, heads = slice(b * n, (b + 1) * n), slice(h * g, (h + 1) * g)
    slopes = None if s["slopes"] is None else s["slopes"][heads]
    return rows, heads, s["q"][rows, heads].transpose(0, 1), slopes


def _exact_tree(s, seed):
    c, n = s["case"], s["case"]["new"]
    o, positions = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), []
    for b, (length, parents) in enumerate(zip(_lengths(c), _parents(c, seed))):
        first = length - n
        lines = []
        for i, p in enumerate(parents):
            lines.append([] if p < -1 else [i] if p == -1 else lines[p] + [i])
        seen = torch.zeros(n, length, dtype=torch.bool)
        for i, line in enumerate(lines):
            seen[i, :first] = bool(line)
            seen[i, [first + x for x in line]] = True
        place = list(range(first)) + [first + max(len(line) - 1, 0) for line in lines]
        at = [first + len(line) - 1 for line in lines]
        positions.append([first + len(line) - 1 if line else 0 for line in lines])
        away = (torch.tensor(at)[:, None] - torch.tensor(place)).abs().cuda()
        seen = seen.cuda()
        for h in range(c["kv_heads"]):
            rows, heads, q, slopes = _exact_heads(s, b, h)
            oo, _ = _exact_rows(c, q, *_sequence(s, b, length, h), seen, slopes, away)
            o[rows, heads] = oo.transpose(0, 1)
    return {"o": o, "positions": _ints(positions)}


def _exact_sparse(s):
    c, n, page, K, D = s["case"], s["case"]["new"], s["case"]["page"], s["case"]["kv_heads"], s["case"]["D"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    means = s["means"].double()
    chosen = torch.full((c["B"] * n, K, c["count"]), -1, dtype=torch.int32)
    for b, length in enumerate(_lengths(c)):
        table = s["page_table"][b].long()
        for number in range((length - n) // page, (length - 1) // page + 1):
            held = min(page, length - number * page)
            means[table[number]] = s["cache"][table[number], 0, :, :held].double().sum(1) / held
        # the selection goes by the means as they are stored
        stored = means[table].to(s["means"].dtype).double()   # [blocks, K, D]
        scores = []
        for h in range(K):
            _, _, q, _ = _exact_heads(s, b, h)
            scores.append((q.double().sum(0)[:, None] * stored[None, :, h]).sum(-1).tolist())   # [n, blocks]
        for i in range(n):
            t = length - n + i
            last = t // page
            for h in range(K):
                must = set(range(min(c["sink"], last + 1))) | set(range(max(0, last - c["local"] + 1), last + 1))
                rest = sorted((x for x in range(last + 1) if x not in must), key=lambda x: (-scores[h][i][x], x))
                pick = sorted(must | set(rest[:max(0, c["count"] - len(must))]))
                chosen[b * n + i, h, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
                rows, heads, q, _ = _exact_heads(s, b, h)
                keys = (torch.tensor(pick, device="cuda")[:, None] * page + torch.arange(page, device="cuda")).view(-1)
                keys = keys[keys <= t]
                at = table[keys // page]
                k, v = (s["cache"][at, x, h, keys % page] for x in (0, 1))
                seen = torch.ones(1, keys.shape[0], dtype=torch.bool, device="cuda")
                o[b * n + i, heads] = _exact_rows(c, q[:, i:i + 1], k, v, seen, None, None)[0][:, 0]
    return {"o": o, "means": means, "chosen": chosen.cuda()}


def _exact_weigh(s):
    c, n = s["case"], s["case"]["new"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    weights = s["weighed"].double()
    for b, length in enumerate(_lengths(c)):
        j, at = torch.arange(length, device="cuda"), torch.arange(length - n, length, device="cuda")
        seen, away = j <= at[:, None], (at[:, None] - j).abs()
        for h in range(c["kv_heads"]):
            rows, heads, q, slopes = _exact_heads(s, b, h)
            oo, p = _exact_rows(c, q, *_sequence(s, b, length, h), seen, slopes, away)
            o[rows, heads] = oo.transpose(0, 1)
            weights[b, h, :length] = p.sum((0, 1))
            weights[b, h, :length - n] += s["weights"][b, h, :length - n].double()
    return {"o": o, "weights": weights}


def _exact_moves(s, b, heads, moves):
    """Token moves[i] of sequence b to place i of those heads, from a copy of what was there."""
    page, table = s["case"]["page"], s["page_table"][b].long()
    src, dst = (torch.tensor(x, device="cuda") for x in zip(*moves))
    held = s["cache"][table[src // page], :, heads, src % page].clone()
    s["cache"][table[dst // page], :, heads, dst % page] = held


def _exact_accept(s, seed):
    c = s["case"]
    for b, (length, row) in enumerate(zip(_lengths(c), _branches(c, _parents(c, seed), seed))):
        first = length - c["new"]
        moves = [(first + x, first + i) for i, x in enumerate(row) if x >= 0]
        for h in range(c["kv_heads"]):
            _exact_moves(s, b, h, moves)
    return {"cache": s["cache"].double()}


def _exact_evict(s):
    c = s["case"]
    kept = torch.full((c["B"], c["kv_heads"], c["keep"]), -1, dtype=torch.int32)
    weights = torch.zeros(kept.shape, dtype=torch.float64)
    for b, length in enumerate(_lengths(c)):
        for h in range(c["kv_heads"]):
            w = s["weights"][b, h, :length].tolist()
            if length <= c["keep"]:
                pick = list(range(length))
            else:
                old = range(c["sink"], length - c["recent"])
                heavy = sorted(old, key=lambda x: (-w[x], x))[:c["keep"] - c["sink"] - c["recent"]]
                pick = sorted([*range(c["sink"]), *heavy, *range(length - c["recent"], length)])
            kept[b, h, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
            weights[b, h, :len(pick)] = torch.tensor([w[x] for x in pick], dtype=torch.float64)
            _exact_moves(s, b, h, [(x, i) for i, x in enumerate(pick)])
    return {"kept": kept.cuda(), "weights": weights.cuda(), "cache": s["cache"].double()}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("tree", "accept"):
        return (_exact_tree if case["kind"] == "tree" else _exact_accept)(s, seed)
    return {"sparse": _exact_sparse, "weigh": _exact_weigh, "evict": _exact_evict}[case["kind"]](s)
