"""Trees of drafted tokens, selected pages, accumulated weights and eviction over the paged cache, against plain float64
forms."""

import math
import random

import pytest
import torch

import _decoding as ref
from _attention import U16, U32
from paper_2603_06492_amd import attention as na
from paper_2603_06492_amd import decoding as nd

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
IDS = {BF: "bf16", F32: "f32"}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _near(name, got, want, mag, u):
    """Infinities and NaN where the reference has them and nowhere else, everything else within its bound."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert bool((torch.isfinite(got) == fine).all()), f"{name}: infinities or NaN in other places"
    assert bool((torch.isnan(got) == torch.isnan(want)).all()), name
    inf = torch.isinf(want)
    assert bool((got[inf] == want[inf]).all()), name
    off = ((got - want).abs() - u * (want.abs() + mag))[fine]
    assert not off.numel() or float(off.max()) <= 1e-30, f"{name}: {float(off.max())} past its bound"


class Held:
    """A cache of random pages for sequences of the given lengths, some spare pages, and every slot past a sequence's tokens
    NaN: whoever reads one shows it."""

    def __init__(self, lengths, H, K, D, page, dt, seed, per=None):
        g = _gen(seed)
        B = len(lengths)
        self.lengths, self.page, self.dt = lengths, page, dt
        self.per = per or max(1, -(-max(lengths) // page) + 1)
        self.pages = B * self.per + 3
        self.cache = torch.randn((self.pages, 2, K, page, D), generator=g, device="cuda").to(dt)
        perm = torch.randperm(self.pages, generator=g, device="cuda")[:B * self.per]
        self.table = perm.view(B, self.per).to(torch.int32)
        rows = self.table.tolist()
        for b, n in enumerate(lengths):
            for t in range(max(0, min(n, self.per * page)), self.per * page):
                self.cache[rows[b][t // page], :, :, t % page] = math.nan
        self.len = _ints(lengths)
        self.H, self.K, self.D, self.g = H, K, D, g

    def q(self, n, std=1.0):
        return (torch.randn((len(self.lengths) * n, self.H, self.D), generator=self.g, device="cuda") * std).to(self.dt)

    def args(self):
        return self.cache, self.table, self.len

    def each(self):
        cache, table = self.cache.cpu(), self.table.tolist()
        return [(b, cache, table[b], n) for b, n in enumerate(self.lengths)]


def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda")


def _trees(rng, B, n, spoil=0.1):
    """Random trees: parents shortly before, now and then a node that is none, or a number that stands for nothing."""
    out = []
    for _ in range(B):
        row = [max(-1, i - 1 - int(rng.expovariate(0.5))) for i in range(n)]
        for i in range(n):
            if rng.random() < spoil:
                row[i] = rng.choice((-2, -7, i, i + 1, n, 2 ** 31 - 1, -2 ** 31))
        out.append(row)
    return out


# -------------------------------------------------------------------- tree --

@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 100, 255, 256])
def test_tree_rows(n):
    rng = random.Random(n)
    rows = _trees(rng, 4, n, 0.05) + [list(range(-1, n - 1)), [-1] * n, [-2] * n]
    lens = [5 * n, n, max(n - 3, 0), 0, 9 * n, n + 1, n]
    seen, depths, positions = (t.cpu() for t in nd.noble_tree_rows(_ints(rows), _ints(lens)))
    assert seen.shape == (7, n, (n + 31) // 32)
    for b, parents in enumerate(rows):
        for i, line in enumerate(ref.lines(parents)):
            words = [int(x) & 0xffffffff for x in seen[b, i]]
            bits = [c for c in range(32 * len(words)) if words[c // 32] >> (c % 32) & 1]
            assert bits == line, (b, i)
            assert int(depths[b, i]) == len(line) - 1
            assert int(positions[b, i]) == (max(lens[b] - n + len(line) - 1, 0) if line else 0)


TREES = [   # lengths, n, H, K, D, page, dtype, softcap, bias
    ([1000], 4, 16, 16, 128, 16, BF, 0.0, False),
    ([70, 33, 300, 9], 9, 4, 2, 64, 16, BF, 0.0, True),
    ([65, 64, 200], 33, 4, 4, 128, 8, BF, 30.0, False),
    ([40, 0, 5, 17, 131], 17, 8, 1, 80, 32, BF, 0.0, True),
    ([130, 64], 64, 2, 2, 32, 64, BF, 0.0, False),
    ([300, 256], 256, 1, 1, 8, 8, BF, 0.0, True),
    ([97, 30], 13, 4, 2, 64, 16, F32, 0.0, True),
    ([140, 21, 20], 20, 8, 2, 128, 16, F32, 20.0, False),
    ([50], 1, 12, 4, 96, 128, F32, 0.0, False),
    ([33], 7, 64, 2, 40, 8, BF, 0.0, False),
    ([2900, 1400], 6, 2, 1, 64, 16, BF, 0.0, True),
    ([2000, 65], 40, 8, 2, 128, 64, BF, 30.0, True),
    ([1800, 3], 3, 2, 1, 128, 8, F32, 0.0, True),
]


@pytest.mark.parametrize("lengths,n,H,K,D,page,dt,cap,bias", TREES,
                         ids=[f"{c[0]}-{c[1]}-{c[2]}over{c[3]}x{c[4]}-{IDS[c[6]]}" for c in TREES])
def test_attn_tree(lengths, n, H, K, D, page, dt, cap, bias):
    h = Held(lengths, H, K, D, page, dt, 3)
    q, parents = h.q(n), _trees(random.Random(5), len(lengths), n)
    sl = _slopes(H) if bias else None
    seen, depths, _ = nd.noble_tree_rows(_ints(parents), h.len)
    o = nd.noble_attn_tree(q, *h.args(), seen, depths, sl, softcap=cap)
    for b, cache, table, length in h.each():
        want, mag, _, _ = ref.tree(q[b * n:(b + 1) * n].cpu(), cache, table, length, parents[b], softcap=cap, slopes=sl)
        _near(f"o of {b}", o[b * n:(b + 1) * n], want, mag, U16 if dt == BF else U32)


def test_a_chain_is_the_paged_attention():
    """A tree that is one line sees what noble_attn_paged's rows see."""
    for dt, n in ((BF, 5), (F32, 3), (BF, 40)):
        h = Held([400, 77, 41], 4, 2, 64, 16, dt, 8)
        q = h.q(n)
        seen, depths, positions = nd.noble_tree_rows(_ints([list(range(-1, n - 1))] * 3), h.len)
        assert positions.tolist() == [list(range(x - n, x)) for x in h.lengths]
        o, p = nd.noble_attn_tree(q, *h.args(), seen, depths), na.noble_attn_paged(q, *h.args())
        torch.testing.assert_close(o.float(), p.float(), rtol=2 * U16 if dt == BF else 1e-5, atol=2 * U16 if dt == BF else 1e-5)


@pytest.mark.parametrize("dt", [BF, F32], ids=IDS.get)
@pytest.mark.parametrize("H,K,D", [(2, 2, 64), (8, 2, 128)])
def test_tree_infinite_and_nan_values_reach_who_sees_them(dt, H, K, D):
    n, lengths = 12, [90, 45, 12]
    h = Held(lengths, H, K, D, 16, dt, 4)
    rows = h.table.tolist()
    parents = [[-1, 0, 0, 1, 2, -1, 5, -2, 7, 5, 3, 4]] * 3
    for b, node, what, value in ((0, 1, 1, math.inf), (0, 5, 1, math.nan), (1, 2, 1, -math.inf), (2, 8, 1, math.nan),
                                 (2, 9, 0, math.nan)):
        t = lengths[b] - n + node
        h.cache[rows[b][t // 16], what, :, t % 16] = value
    q = h.q(n)
    seen, depths, _ = nd.noble_tree_rows(_ints(parents), h.len)
    o = nd.noble_attn_tree(q, *h.args(), seen, depths)
    for b, cache, table, length in h.each():
        want, mag, _, _ = ref.tree(q[b * n:(b + 1) * n].cpu(), cache, table, length, parents[b])
        _near(f"o of {b}", o[b * n:(b + 1) * n], want, mag, U16 if dt == BF else U32)
    # one in a token before the tree: every node has it, what is no node has not
    h.cache[rows[0][3], 1, :, 2] = math.nan
    o = nd.noble_attn_tree(q, *h.args(), seen, depths)[:n]
    node = torch.tensor([bool(x) for x in ref.lines(parents[0])])
    assert bool(torch.isnan(o[node.cuda()]).all()) and bool((o[~node.cuda()] == 0).all())


def test_tree_pages_outside_the_cache_are_not_there():
    n = 6
    h = Held([100, 60, 30], 4, 2, 64, 8, BF, 6)
    h.table[0, 2], h.table[0, 12], h.table[1, 7] = -1, h.pages, 2 ** 31 - 1
    h.table[2] = -5
    q, parents = h.q(n), _trees(random.Random(1), 3, n, 0.0)
    seen, depths, _ = nd.noble_tree_rows(_ints(parents), h.len)
    o = nd.noble_attn_tree(q, *h.args(), seen, depths)
    for b, cache, table, length in h.each():
        want, mag, _, _ = ref.tree(q[b * n:(b + 1) * n].cpu(), cache, table, length, parents[b])
        _near(f"o of {b}", o[b * n:(b + 1) * n], want, mag, U16)
    assert bool((o[2 * n:] == 0).all())


# -------------------------------------------------------------------- keep --

def _numbered(h):
    """The cache with a number of its own in every element: moves are checked bit for bit."""
    h.cache = torch.arange(h.cache.numel(), device="cuda", dtype=torch.float32).view(h.cache.shape)
    if h.dt == BF:   # any bits that are no NaN: a move keeps them
        h.cache = (h.cache.long() % 32000).to(torch.int16).view(BF)
    return h


def _same(a, b):
    return bool((a.contiguous().view(torch.int16) == b.contiguous().view(torch.int16)).all())


KEEPS = [(8, 64, 16, BF), (1, 128, 8, BF), (4, 80, 32, BF), (2, 8, 16, BF), (2, 128, 64, F32), (3, 40, 8, F32)]


@pytest.mark.parametrize("K,D,page,dt", KEEPS, ids=[f"{c[0]}x{c[1]}-{c[2]}-{IDS[c[3]]}" for c in KEEPS])
def test_cache_keep(K, D, page, dt):
    lengths = [700, 333, 40, 0]
    rng = random.Random(K)
    for heads in {1, K}:
        h = _numbered(Held(lengths, K, K, D, page, dt, 11))
        most = 500
        kept = [[sorted(rng.sample(range(n), min(most, n * 2 // 3))) for _ in range(heads)] for n in lengths]
        kept = [[x + [-1] * (most - len(x)) for x in row] for row in kept]
        before = h.cache.clone()
        out = nd.noble_cache_keep(h.cache, h.table, _ints(kept))
        assert out is h.cache
        want = before.cpu()
        for b, _, table, _ in h.each():
            moved = ref.keep(before.cpu(), table, kept[b], 0)
            mine = [p for p in table if 0 <= p < h.pages]
            want[mine] = moved[mine]
        assert _same(h.cache.cpu(), want)


def test_cache_keep_of_an_accepted_branch():
    n, lengths = 9, [100, 33, 9, 4]
    h = _numbered(Held(lengths, 2, 2, 64, 8, BF, 12))
    kept = [[[0, 2, 3, 7, 8, -1, -1, -1, -1]], [[4] + [-1] * 8], [[0, 1, 2, 3, 4, 5, 6, 7, 8]], [[1, 6, -1, -1, -1, -1, -1, -1, -1]]]
    start = [x - n for x in lengths]
    before = h.cache.clone()
    nd.noble_cache_keep(h.cache, h.table, _ints(kept), _ints(start))
    want = before.cpu()
    for b, _, table, _ in h.each():
        moved = ref.keep(before.cpu(), table, kept[b], start[b])
        want[table] = moved[table]
    assert _same(h.cache.cpu(), want)


def test_cache_keep_skips_what_is_not_there():
    h = _numbered(Held([64, 64, 64], 2, 2, 16, 8, BF, 13, per=8))
    h.table[0, 3], h.table[1, 0], h.table[2, 1] = -1, h.pages, 2 ** 31 - 1
    kept = [[list(range(8, 40))], [[5, 0, 9, 3, 2 ** 31 - 1, -2 ** 31, 63, 64] + [-1] * 24], [list(range(20, 52))]]
    start = [0, 3, 2 ** 31 - 1]
    before = h.cache.clone()
    nd.noble_cache_keep(h.cache, h.table, _ints(kept), _ints(start))
    want = before.cpu()
    for b, _, table, _ in h.each():
        moved = ref.keep(before.cpu(), table, kept[b], start[b])
        mine = [p for p in table if 0 <= p < h.pages]
        want[mine] = moved[mine]
    assert _same(h.cache.cpu(), want)


def test_lists_longer_than_the_sequences_may_be():
    """Room for more tokens than the page table holds: the rest of the list is -1, and nothing moves there."""
    h = _numbered(Held([40, 17], 2, 2, 64, 8, BF, 14, per=5))
    w = torch.rand((2, 2, 40), generator=h.g, device="cuda")
    before = h.cache.clone()
    for keep, sink, recent in ((69, 4, 64), (300, 0, 0)):
        kept, left = nd.noble_evict_select(w, h.len, keep, sink=sink, recent=recent)
        for b, n in enumerate(h.lengths):
            assert kept[b].tolist() == [list(range(n)) + [-1] * (keep - n)] * 2
        nd.noble_cache_keep(h.cache, h.table, kept)
        assert _same(h.cache, before)
    kept[0, :, 3:40] = torch.arange(3, 40, device="cuda") + 20   # past the table from 40 on
    nd.noble_cache_keep(h.cache, h.table, kept)
    want = before.cpu()
    table = h.table[0].tolist()
    want[table] = ref.keep(before.cpu(), table, kept[0].tolist(), 0)[table]
    assert _same(h.cache.cpu(), want)


# ---------------------------------------------------------- selected pages --

@pytest.mark.parametrize("K,D,page,dt", [(2, 128, 16, BF), (4, 80, 8, BF), (1, 8, 32, F32), (3, 64, 64, F32)])
@pytest.mark.parametrize("new", [1, 3, 40, 10 ** 9])
def test_page_means(K, D, page, dt, new):
    lengths = [300, 1, 0, page, 2 * page + 1, 77]
    h = Held(lengths, K, K, D, page, dt, 21)
    h.table[0, 1] = -1
    means = torch.full((h.pages, K, D), 7.0, dtype=dt, device="cuda")
    assert nd.noble_page_means(*h.args(), new, means) is means
    want = torch.full((h.pages, K, D), 7.0, dtype=torch.float64)
    for b, cache, table, n in h.each():
        for c in range(max(0, n - new) // page, -(-n // page)):
            if 0 <= table[c] < h.pages:
                want[table[c]] = cache[table[c], 0, :, :min(page, n - c * page)].double().mean(1)
    got = means.double().cpu()
    # one rounding: half a step, which is eps / 2 of the value at most (the steps between 1 and 2 are eps)
    off = float(((got - want).abs() - want.abs() * (torch.finfo(dt).eps / 2)).max())
    assert off <= 1e-12, off
    fresh = nd.noble_page_means(*h.args(), new)
    assert bool((fresh.double().cpu() == torch.where(want == 7.0, 0.0, got)).all())


SELECTS = [   # lengths, n, H, K, D, page, dtype, count, sink, local
    ([1000, 30, 0, 517], 1, 8, 2, 128, 8, BF, 20, 1, 2),
    ([700, 64, 3], 5, 4, 4, 64, 16, BF, 9, 2, 1),
    ([400], 2, 16, 1, 80, 8, F32, 33, 0, 4),
    ([300, 299], 1, 2, 2, 8, 8, BF, 1, 0, 1),
    ([256, 255, 100], 3, 3, 3, 40, 32, F32, 5, 2, 3),
    ([2048], 1, 4, 1, 32, 8, BF, 200, 1, 1),
]


@pytest.mark.parametrize("lengths,n,H,K,D,page,dt,count,sink,local", SELECTS, ids=[f"{c[0]}-{c[1]}-{c[7]}" for c in SELECTS])
def test_block_select(lengths, n, H, K, D, page, dt, count, sink, local):
    h = Held(lengths, H, K, D, page, dt, 22)
    means = torch.randn((h.pages, K, D), generator=h.g, device="cuda").to(dt)
    means[5] = means[9] = means[h.pages // 2]   # ties
    if h.per > 12:
        h.table[0, 7] = -1
    q = h.q(n)
    got = nd.noble_block_select(q, means, h.table, h.len, count, page=page, sink=sink, local=local)
    assert got.shape == (len(lengths) * n, K, count) and got.dtype == torch.int32
    for b, _, table, length in h.each():
        want = ref.select(q[b * n:(b + 1) * n].cpu(), means.cpu(), table, length, n, count, page, sink, local)
        assert got[b * n:(b + 1) * n].cpu().tolist() == want.tolist(), b


def test_block_select_ties_zeros_infinities_and_nan():
    page, K, D, count = 8, 1, 16, 6
    h = Held([8 * 30], 2, K, D, page, F32, 23)
    means = torch.zeros((h.pages, K, D), device="cuda")
    table = h.table[0].tolist()
    q = torch.ones((1, 2, D), device="cuda")
    pick = lambda: nd.noble_block_select(q, means, h.table, h.len, count, page=page, sink=1, local=2)[0, 0].tolist()  # noqa: E731
    assert pick() == [0, 1, 2, 3, 28, 29]                # all equal: the first
    means[table[4]] = -0.0
    assert pick() == [0, 1, 2, 3, 28, 29]                # -0 is no less than 0
    means[table[20]], means[table[9]] = math.nan, math.inf
    means[table[2]] = -math.inf
    assert pick() == [0, 1, 9, 20, 28, 29]
    means[table[17]], means[table[11]], means[table[10]] = math.nan, math.nan, 1e30
    assert pick() == [0, 11, 17, 20, 28, 29]
    means[table[25]] = math.nan
    assert pick() == [0, 11, 17, 20, 28, 29]             # four NaN: the first three


@pytest.mark.parametrize("blocks", [2047, 2500, 16385, 20000])
def test_block_select_of_long_sequences(blocks):
    """More blocks than the small and the large form keep in LDS."""
    page, D, count = 8, 8, 40
    g = _gen(blocks)
    table = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)[None]
    means = torch.randn((blocks, 1, D), generator=g, device="cuda").to(BF)
    q = torch.randn((2, 2, D), generator=g, device="cuda").to(BF)
    length = blocks * page - 3
    got = nd.noble_block_select(q, means, table, _ints([length]), count, page=page, sink=2, local=3)
    want = ref.select(q.cpu(), means.cpu(), table[0].tolist(), length, 2, count, page, 2, 3)
    assert got.cpu().tolist() == want.tolist()


@pytest.mark.parametrize("B,n,H,K,D,dt,count,sink,local", [
    (3, 2, 4, 2, 128, BF, 40, 2, 3), (20, 2, 4, 2, 128, BF, 40, 2, 3), (3, 1, 2, 1, 40, F32, 300, 0, 1), (45, 1, 2, 1, 64, F32, 6, 5, 1),
    (2, 3, 6, 3, 72, BF, 130, 127, 2)], ids=str)
def test_block_select_by_one_workgroup_or_several(B, n, H, K, D, dt, count, sink, local):
    """Rows over hundreds of blocks, few and many; equal blocks far apart, pages that are none, shorter sequences."""
    page, per = 8, 640
    g = _gen(B + D)
    lengths = [(per * page, per * page - 5, 300 * page + 1, count * page, 1023, 1)[b % 6] for b in range(B)]
    table = torch.randperm(B * per, generator=g, device="cuda").view(B, per).to(torch.int32)
    table[:, 30:600:7] = table[:, 20:21]           # one page many times: the first of them are taken
    table[:, 33] = -1
    table[:, 450] = B * per
    means = torch.randn((B * per, K, D), generator=g, device="cuda").to(dt)
    means[table[:, 20].long()] = means[table[:, 20].long()].abs() * 3
    q = torch.randn((B * n, H, D), generator=g, device="cuda").abs().to(dt)
    got = nd.noble_block_select(q, means, table, _ints(lengths), count, page=page, sink=sink, local=local).cpu()
    rows = table.tolist()
    for b in list(range(min(B, 6))) + [B - 1]:
        mine = slice(b * n, (b + 1) * n)
        want = ref.select(q[mine].cpu(), means.cpu(), rows[b], lengths[b], n, count, page, sink, local)
        assert got[mine].tolist() == want.tolist(), b


BLOCKS = [   # lengths, n, H, K, D, page, dtype, count, softcap, bias
    ([1000, 30, 0, 517], 1, 8, 2, 128, 8, BF, 20, 0.0, False),
    ([300, 64, 2], 5, 4, 4, 64, 16, BF, 9, 0.0, True),
    ([400], 2, 16, 1, 80, 8, F32, 33, 20.0, True),
    ([256, 255, 100], 3, 40, 2, 40, 32, BF, 5, 30.0, False),
    ([700], 1, 4, 2, 128, 64, F32, 7, 0.0, False),
    ([500, 129], 1, 2, 1, 96, 128, BF, 3, 0.0, True),
    ([2000, 900], 2, 40, 2, 64, 32, BF, 45, 0.0, False),
    ([1500], 1, 2, 1, 128, 16, BF, 80, 0.0, True),
]


@pytest.mark.parametrize("lengths,n,H,K,D,page,dt,count,cap,bias", BLOCKS, ids=[f"{c[0]}-{c[1]}-{c[7]}" for c in BLOCKS])
def test_attn_blocks(lengths, n, H, K, D, page, dt, count, cap, bias):
    h = Held(lengths, H, K, D, page, dt, 24)
    rng = random.Random(2)
    chosen = []
    for length in lengths:
        for i in range(n):
            own = (length - n + i) // page
            for _ in range(K):
                pick = sorted(rng.sample(range(own + 1), min(own + 1, rng.randint(0, count)))) if own >= 0 else []
                if pick and rng.random() < 0.5 and own not in pick:
                    pick[-1] = own
                chosen.append((pick + [-1] * count)[:count])
    chosen = torch.tensor(chosen, dtype=torch.int32).view(-1, K, count)
    q, sl = h.q(n), _slopes(H) if bias else None
    o = nd.noble_attn_blocks(q, *h.args(), chosen.cuda(), sl, softcap=cap)
    for b, cache, table, length in h.each():
        want, mag, _, _ = ref.blocks(q[b * n:(b + 1) * n].cpu(), cache, table, length, chosen[b * n:(b + 1) * n], softcap=cap,
                                     slopes=sl)
        _near(f"o of {b}", o[b * n:(b + 1) * n], want, mag, U16 if dt == BF else U32)


def test_attn_blocks_lists_end_at_what_is_no_block():
    """Numbers out of order, twice, past the row's own block or negative end a list; pages outside the cache are skipped."""
    h = Held([90, 90], 2, 1, 32, 8, F32, 25)
    h.table[1, 4] = -1
    lists = [[[0, 3, 3, 5, 6]], [[2, 1, 0, 4, 5]], [[1, 12, 3, 4, 5]], [[-1, 0, 1, 2, 3]], [[0, 4, 10, 11, 2 ** 31 - 1]],
             [[4, 5, -2 ** 31, 6, 7]], [[4, -1, -1, -1, -1]], [[0, 1, 2, 3, 4]]]
    q, chosen = h.q(4), torch.tensor(lists, dtype=torch.int32)
    o = nd.noble_attn_blocks(q, *h.args(), chosen.cuda())
    for b, cache, table, length in h.each():
        want, mag, _, _ = ref.blocks(q[b * 4:b * 4 + 4].cpu(), cache, table, length, chosen[b * 4:b * 4 + 4])
        _near(f"o of {b}", o[b * 4:b * 4 + 4], want, mag, U32)
    assert bool((o[3] == 0).all()) and bool((o[6] == 0).all())


def test_all_blocks_are_the_paged_attention():
    for dt in (BF, F32):
        h = Held([400, 77, 3], 4, 2, 64, 16, dt, 26)
        q = h.q(2)
        means = nd.noble_page_means(*h.args(), 400)
        chosen = nd.noble_block_select(q, means, h.table, h.len, 25, page=16)
        assert chosen[0, 0].tolist() == list(range(25)) and chosen[2, 0].tolist() == list(range(5)) + [-1] * 20
        o, p = nd.noble_attn_blocks(q, *h.args(), chosen), na.noble_attn_paged(q, *h.args())
        torch.testing.assert_close(o.float(), p.float(), rtol=2 * U16 if dt == BF else 1e-5, atol=2 * U16 if dt == BF else 1e-5)


# ------------------------------------------------------ weights, eviction --

WEIGHS = [   # lengths, n, H, K, D, page, dtype, softcap, bias
    ([1000], 1, 16, 16, 128, 16, BF, 0.0, False),
    ([70, 33, 1300, 9], 1, 4, 2, 64, 16, BF, 0.0, True),
    ([65, 64, 200], 33, 4, 4, 128, 8, BF, 30.0, False),
    ([40, 0, 5, 17, 131], 17, 8, 1, 80, 32, BF, 0.0, True),
    ([97, 30], 13, 4, 2, 64, 16, F32, 0.0, True),
    ([140, 21, 20], 5, 8, 2, 128, 16, F32, 20.0, False),
    ([333], 333, 2, 1, 32, 64, F32, 0.0, False),
    ([300, 150], 150, 2, 1, 64, 16, BF, 20.0, True),
    ([2500, 1300], 1, 4, 1, 128, 16, BF, 0.0, True),
]


@pytest.mark.parametrize("lengths,n,H,K,D,page,dt,cap,bias", WEIGHS,
                         ids=[f"{c[0]}-{c[1]}-{c[2]}over{c[3]}x{c[4]}-{IDS[c[6]]}" for c in WEIGHS])
def test_attn_weigh(lengths, n, H, K, D, page, dt, cap, bias):
    h = Held(lengths, H, K, D, page, dt, 31)
    q, sl = h.q(n), _slopes(H) if bias else None
    old = torch.rand((len(lengths), K, h.per * page), generator=h.g, device="cuda")
    for b, x in enumerate(lengths):
        old[b, :, max(0, x - n):] = math.nan   # nothing yet, whatever it holds
    o, new = nd.noble_attn_weigh(q, *h.args(), old, sl, softcap=cap)
    o2, none = nd.noble_attn_weigh(q, *h.args(), None, sl, softcap=cap)
    same = old.clone()
    o3, into = nd.noble_attn_weigh(q, *h.args(), same, sl, softcap=cap, out=same)
    assert into is same and bool((o == o2).all()) and bool((o == o3).all())
    for b, cache, table, length in h.each():
        rows = q[b * n:(b + 1) * n].cpu()
        want, mag, w, size = ref.weigh(rows, cache, table, length, old[b].cpu(), softcap=cap, slopes=sl)
        _near(f"o of {b}", o[b * n:(b + 1) * n], want, mag, U16 if dt == BF else U32)
        # the largest score's rounding, (D + 3) 2^-24 of its sum of magnitudes, is the relative error of a probability and, by
        # the sum, of all of a row; a sum of n H / K + 1 terms adds as many 2^-24 at most
        u = (2 * (D + 3) * float(size.max() if size.numel() else 0) + 16 + n * H // K) * 2.0 ** -24
        held = w.shape[1]
        _near(f"weights of {b}", new[b, :, :held], w, torch.zeros_like(w), u)
        _near(f"weights of {b} from nothing", none[b, :, :held], ref.weigh(rows, cache, table, length, softcap=cap, slopes=sl)[2],
              torch.zeros_like(w), u)
        assert bool((new[b, :, held:] == 0).all()) and bool((same[b, :, :held] == new[b, :, :held]).all())
        assert bool(torch.isnan(same[b, :, held:]).all())   # left as they were


def test_weights_add_up_over_steps():
    """Three calls of one token each, and one of three: the same weights."""
    h = Held([120, 64], 4, 2, 64, 16, F32, 32)
    q = h.q(3).view(2, 3, 4, 64)
    steps = None
    for i in range(3):
        lens = h.len - 2 + i
        _, steps = nd.noble_attn_weigh(q[:, i].contiguous(), h.cache, h.table, lens, steps, out=steps)
    _, once = nd.noble_attn_weigh(q.reshape(6, 4, 64), *h.args())
    for b, n in enumerate(h.lengths):
        _, lone = nd.noble_attn_weigh(q[:, 0].contiguous(), h.cache, h.table, h.len - 2)
        assert bool((lone[b, :, n - 2:] == 0).all())
        torch.testing.assert_close(steps[b, :, :n], once[b, :, :n], rtol=2e-5, atol=1e-9)
        torch.testing.assert_close(once[b, :, :n].sum(1), torch.full((2,), 6.0, device="cuda"), rtol=1e-5, atol=0)


@pytest.mark.parametrize("dt", [BF, F32], ids=IDS.get)
def test_weigh_infinities_nan_and_missing_pages(dt):
    n = 4
    h = Held([70, 70, 40, 2], 2, 1, 64, 8, dt, 33)
    rows = h.table.tolist()
    h.cache[rows[0][8], 1, :, 5] = math.inf       # token 69, the last: seen by its own row alone
    h.cache[rows[1][8], 0, :, 4] = math.nan       # token 68's key: rows 2 and 3
    h.table[1, 2] = -1
    h.table[2] = h.pages
    q = h.q(n)
    old = torch.ones((4, 1, h.per * 8), device="cuda")
    o, w = nd.noble_attn_weigh(q, *h.args(), old)
    for b, cache, table, length in h.each():
        want, mag, ww, size = ref.weigh(q[b * n:(b + 1) * n].cpu(), cache, table, length, old[b].cpu())
        _near(f"o of {b}", o[b * n:(b + 1) * n], want, mag, U16 if dt == BF else U32)
        _near(f"weights of {b}", w[b, :, :ww.shape[1]], ww, torch.zeros_like(ww), 1e-5)


EVICTS = [   # row, lengths, heads, keep, sink, recent
    (100, [100, 50, 0, 99, 100], 3, 40, 4, 8),
    (100, [100, 41, 40, 39, 1], 2, 40, 0, 0),
    (64, [64, 64], 1, 10, 10, 0),
    (64, [64, 64], 1, 10, 0, 10),
    (64, [64, 64], 1, 10, 4, 6),
    (64, [64, 1000, -3], 1, 1, 0, 0),
    (3000, [3000, 2999, 1025], 2, 1024, 4, 64),
    (9000, [9000, 8192, 8193], 2, 777, 1, 1),
    (32768, [32768], 1, 20000, 4, 1000),
    (40000, [40000, 32769], 1, 30000, 4, 1000),
    (40000, [40000], 2, 5, 1, 2),
    (50, [50], 1, 200, 30, 100),
]


@pytest.mark.parametrize("row,lengths,heads,keep,sink,recent", EVICTS, ids=str)
@pytest.mark.parametrize("kind", ["spread", "zeros", "few", "odd"])
def test_evict_select(row, lengths, heads, keep, sink, recent, kind):
    g = _gen(row + keep)
    w = torch.rand((len(lengths), heads, row), generator=g, device="cuda")
    if kind == "zeros":
        w = (w - 0.6).clamp(min=0.0)
    elif kind == "few":
        w = (w * 5).floor() / 8
    elif kind == "odd":
        x = torch.rand(w.shape, generator=g, device="cuda")
        w = torch.where(x < 0.1, math.nan, torch.where(x < 0.2, math.inf, torch.where(x < 0.3, -math.inf, w - 0.5)))
        w = torch.where((x > 0.3) & (x < 0.5), -0.0, torch.where((x > 0.5) & (x < 0.7), 0.0, w))
    kept, kw = nd.noble_evict_select(w, _ints(lengths), keep, sink=sink, recent=recent)
    for b, n in enumerate(lengths):
        for h in range(heads):
            pick = ref.evict(w[b, h].cpu(), n, keep, sink, recent)
            assert kept[b, h].tolist() == pick + [-1] * (keep - len(pick)), (b, h)
            assert bool((kw[b, h, :len(pick)].view(torch.int32) == w[b, h, pick].view(torch.int32)).all())
            assert bool((kw[b, h, len(pick):] == 0).all())
