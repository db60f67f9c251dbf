"""Plain float64 forms of decoding over the paged cache, on the CPU, one sequence, head and token at a time.

How far an output may be off: as in _attention, an element of o is within u of itself (its own rounding) and within u sum p
|v| of the sum over unrounded probabilities, u = 2^-8 for bf16 (half a step is 2^-8 relative for eight significant bits);
in float32 the scores carry about sqrt(D) 2^-24 sum |q_d k_d| scale, which _attention takes as 2e-5 of the sums.  Weights
are float32 sums of probabilities of the scores as they are, bf16 inputs or not: the score of a row is off by at most (D + 3)
2^-24 of its sum of magnitudes, times its log2 e the exponential's argument, and maximum, sum and product add a few 2^-24."""

import math

import torch


def lines(parents):
    """Each node's line of nodes from the root, itself last; [] for no node."""
    out = []
    for i, p in enumerate(parents):
        if p == -1:
            out.append([i])
        elif 0 <= p < i and out[p]:
            out.append(out[p] + [i])
        else:
            out.append([])
    return out


def gather(cache, table, length):
    """Keys and values [tokens, K, D] of a sequence, and which tokens are there."""
    pages, _, K, page, D = cache.shape
    length = min(max(length, 0), len(table) * page)
    kv = torch.zeros(2, length, K, D, dtype=torch.float64)
    there = torch.zeros(length, dtype=torch.bool)
    for t in range(length):
        p = table[t // page]
        if 0 <= p < pages:
            kv[:, t] = cache[p, :, :, t % page].double()
            there[t] = True
    return kv[0], kv[1], there


def attend(q, k, v, seen, away, scale=None, softcap=0.0, slopes=None):
    """q [n, H, D] over k, v [L, K, D]; seen [n, K, L], away [n, L]: o, its magnitude sums, p [n, H, L], and the scores'
    sums of magnitudes."""
    n, H, D = q.shape
    L, K, _ = k.shape
    g = H // K
    q = q.double()
    o, mag = torch.zeros(n, H, D, dtype=torch.float64), torch.zeros(n, H, D, dtype=torch.float64)
    p, size = torch.zeros(n, H, L, dtype=torch.float64), torch.zeros(n, H, dtype=torch.float64)
    scale = D ** -0.5 if scale is None else scale
    for i in range(n):
        for h in range(H):
            s = seen[i, h // g]
            if not bool(s.any()):
                continue
            kk, vv = k[s, h // g], v[s, h // g]
            z = scale * kk @ q[i, h]
            size[i, h] = (scale * kk.abs() @ q[i, h].abs()).max()
            if softcap:
                z = softcap * torch.tanh(z / softcap)
            if slopes is not None:
                z = z - float(slopes[h]) * away[i, s]
                size[i, h] += float(slopes[h]) * away[i, s].max()
            w = torch.exp(z - torch.logsumexp(z, 0))
            p[i, h, s] = w
            o[i, h], mag[i, h] = w @ vv, w @ vv.abs()
    return o, mag, p, size


def tree(q, cache, table, length, parents, **how):
    """One sequence's tree: q [n, H, D]."""
    n = len(parents)
    k, v, there = gather(cache, table, length)
    L = k.shape[0]
    first, line = L - n, lines(parents)
    j = torch.arange(L)
    seen = torch.zeros(n, L, dtype=torch.bool)
    place = j.clone()
    at = torch.zeros(n, dtype=torch.int64)
    for i, x in enumerate(line):
        at[i] = first + len(x) - 1
        if first + i >= 0:
            place[first + i] = at[i]
        if x:
            seen[i] = (j < first) & there
            for c in x:
                if first + c >= 0:
                    seen[i, first + c] = there[first + c]
    K = cache.shape[2]
    return attend(q, k, v, seen[:, None].expand(n, K, L), (at[:, None] - place).abs(), **how)


def select(q, means, table, length, n, count, page, sink, local):
    """Chosen blocks [n, K, count] of one sequence's last n tokens, q [n, H, D]."""
    pages, K, D = means.shape
    g = q.shape[1] // K
    length = min(max(length, 0), len(table) * page)
    out = torch.full((n, K, count), -1, dtype=torch.int32)
    for i in range(n):
        t = length - n + i
        if t < 0:
            continue
        own = t // page
        always = set(range(min(sink, own + 1))) | set(range(max(0, own - local + 1), own + 1))
        ok = torch.tensor([0 <= table[c] < pages for c in range(own + 1)])
        at = torch.tensor([table[c] if ok[c] else 0 for c in range(own + 1)])
        for h in range(K):
            qs = q[i, h * g:(h + 1) * g].double().sum(0)
            score = torch.where(ok, (means[at, h].double() * qs).sum(-1), -math.inf).tolist()
            key = {c: (0 if math.isnan(score[c]) else 1, -score[c] if not math.isnan(score[c]) else 0, c) for c in range(own + 1)}
            rest = sorted((c for c in range(own + 1) if c not in always), key=key.get)
            pick = sorted(always | set(rest[:max(0, count - len(always))]))
            out[i, h, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
    return out


def blocks(q, cache, table, length, chosen, **how):
    """One sequence's last n tokens q [n, H, D] over chosen [n, K, count]."""
    n, page = q.shape[0], cache.shape[3]
    k, v, there = gather(cache, table, length)
    L, K = k.shape[0], cache.shape[2]
    seen = torch.zeros(n, K, L, dtype=torch.bool)
    at = torch.arange(L - n, L)
    for i in range(n):
        t = L - n + i
        for h in range(K):
            before = -1
            for c in chosen[i, h].tolist():
                if t < 0 or c <= before or c > t // page:
                    break
                before = c
                for x in range(c * page, min((c + 1) * page, t + 1)):
                    seen[i, h, x] = there[x]
    return attend(q, k, v, seen, (at[:, None] - torch.arange(L)).abs(), **how)


def weigh(q, cache, table, length, weights=None, **how):
    """One sequence's last n tokens: attend's results and the weights [K, tokens held]."""
    n, H, _ = q.shape
    k, v, there = gather(cache, table, length)
    L, K = k.shape[0], cache.shape[2]
    at = torch.arange(L - n, L)
    seen = ((torch.arange(L) <= at[:, None]) & there)[:, None].expand(n, K, L)
    o, mag, p, size = attend(q, k, v, seen, (at[:, None] - torch.arange(L)).abs(), **how)
    w = p.view(n, K, H // K, L).sum((0, 2))
    if weights is not None:
        old = max(L - n, 0)
        w[:, :old] += weights[:, :old].double()
    return o, mag, w, size


def evict(weights, length, keep, sink, recent):
    """Kept tokens of one row of weights."""
    n = min(max(length, 0), weights.shape[0])
    if n <= keep:
        pick = list(range(n))
    else:
        w = weights.tolist()
        key = lambda j: (0 if math.isnan(w[j]) else 1, 0 if math.isnan(w[j]) else -w[j], j)  # noqa: E731
        old = sorted(range(sink, n - recent), key=key)[:keep - sink - recent]
        pick = sorted([*range(sink), *old, *range(n - recent, n)])
    return pick


def keep(cache, table, kept, start):
    """The cache after one sequence's moves; kept [kept_heads, most], a list of lists."""
    pages, _, K, page, _ = cache.shape
    out = cache.clone()
    for h in range(K):
        for i, x in enumerate(kept[h if len(kept) > 1 else 0]):
            src, dst = start + x, start + i
            if x <= i or not 0 <= src < len(table) * page or not 0 <= dst < len(table) * page:
                continue
            ps, pd = table[src // page], table[dst // page]
            if 0 <= ps < pages and 0 <= pd < pages:
                out[pd, :, h, dst % page] = cache[ps, :, h, src % page]
    return out
