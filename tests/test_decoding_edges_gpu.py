"""The decoding operators at the edges of their calls: native and Python paths, strides, other streams, graphs, caches past
4 GiB, page tables that sequences share, nothing to do."""

import math
import random

import pytest
import torch

import _decoding as ref
from _attention import U16, U32
from paper_2603_06492_amd import attention as na
from paper_2603_06492_amd import decoding as nd
from test_decoding_gpu import BF, F32, TREES, WEIGHS, Held, _gen, _ints, _near, _slopes, _trees

pytestmark = pytest.mark.gpu


class Calls:
    """Every call over one set of inputs."""

    def __init__(self, dt, n=3, lengths=(150, 64, 5, 0), H=4, K=2, D=64, page=16, seed=41):
        self.h = h = Held(list(lengths), H, K, D, page, dt, seed)
        self.n, self.count = n, 4
        self.q, self.slopes = h.q(n), _slopes(H)
        self.parents = _ints(_trees(random.Random(2), len(lengths), n, 0.1))
        self.means = torch.randn((h.pages, K, D), generator=h.g, device="cuda").to(dt)
        self.weights = torch.rand((len(lengths), K, h.per * page), generator=h.g, device="cuda")

    def run(self, **on):
        """All results, over copies of what is written."""
        h, q = self.h, self.q
        cache, means, weights = h.cache.clone(), self.means.clone(), self.weights.clone()
        torch.cuda.synchronize()   # the copies are made on the current stream
        return self.over(cache, means, weights, **on)

    def over(self, cache, means, weights, **on):
        h, q, held = self.h, self.q, (cache, self.h.table, self.h.len)
        seen, depths, positions = nd.noble_tree_rows(self.parents, h.len, **on)
        tree = nd.noble_attn_tree(q, *held, seen, depths, self.slopes, softcap=20.0, **on)
        nd.noble_page_means(*held, self.n, means, **on)
        chosen = nd.noble_block_select(q, means, h.table, h.len, self.count, page=h.page, sink=1, local=1, **on)
        blocks = nd.noble_attn_blocks(q, *held, chosen, **on)
        o, _ = nd.noble_attn_weigh(q, *held, weights, out=weights, scale=0.2, **on)
        kept, left = nd.noble_evict_select(weights, h.len, 40, sink=2, recent=8, **on)
        nd.noble_cache_keep(cache, h.table, kept, **on)
        return [seen, depths, positions, tree, means, chosen, blocks, o, weights, kept, left, cache]


def _bits(x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


def _same(a, b):
    assert len(a) == len(b)
    for i, (x, y) in enumerate(zip(a, b)):
        assert bool((_bits(x) == _bits(y)).all()), i


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_native_and_python_calls(dt, monkeypatch):
    """The native code serves every ordinary call, and gives what the Python path does."""
    c = Calls(dt)
    served = []
    native = nd._native()

    class Watch:
        def __getattr__(self, name):
            f = getattr(native, name)

            def call(*a):
                out = f(*a)
                served.append((name, out is not None))
                return out
            return call

    monkeypatch.setattr(nd, "_native", lambda: Watch())
    fast = c.run()
    assert len(served) == 8 and all(ok for _, ok in served), served
    _same(fast, c.run(stream=torch.cuda.current_stream()))


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_calls_on_another_stream_while_the_current_one_is_busy(dt):
    c = Calls(dt)
    want = c.run()
    torch.cuda.synchronize()
    given = [t.clone() for t in (c.h.cache, c.means, c.weights)]
    torch.cuda.synchronize()
    side, big = torch.cuda.Stream(), torch.randn(2048, 2048, device="cuda")
    for _ in range(30):
        big = big @ big * 1e-3
    got = c.over(*given, stream=side)
    torch.cuda.synchronize()
    _same(got, want)


@pytest.mark.parametrize("dt,n", [(BF, 1), (BF, 5), (BF, 40), (F32, 3)], ids=["bf16-1", "bf16-5", "bf16-40", "f32-3"])
def test_captured_and_replayed(dt, n):
    """The calls of a step in a graph, beside another graph of the same, replayed over new inputs with eager work between."""
    lengths = (150, 64, 45, 41)
    cs = [Calls(dt, n, lengths, seed=s) for s in (51, 52, 53)]
    eager = [c.run() for c in cs]
    live = Calls(dt, n, lengths, seed=54)
    state = [t.clone() for t in (live.h.cache, live.means, live.weights)]
    live.over(*state)
    graphs = []
    for _ in range(2):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = live.over(*state)
        graphs.append((g, out))
    for turn in range(3):
        for (g, out), c, want in zip(graphs, cs[turn % 2:], eager[turn % 2:]):
            live.q.copy_(c.q)
            live.parents.copy_(c.parents)
            live.h.table.copy_(c.h.table)
            live.h.len.copy_(c.h.len)
            for dst, src in zip(state, (c.h.cache, c.means, c.weights)):
                dst.copy_(src)
            g.replay()
            cs[2].run()
            torch.cuda.synchronize()
            _same(out, want)


@pytest.mark.parametrize("dt,n", [(BF, 2), (BF, 20), (BF, 70), (F32, 4)])
def test_strided_queries_and_outputs(dt, n):
    """Queries that are columns of wider rows, outputs into such, broadcast queries: as dense ones."""
    h = Held([100, 80], 4, 2, 64, 16, dt, 61)
    wide = torch.randn((2 * n, 4 * 64 + 128), generator=h.g, device="cuda").to(dt)
    q = wide[:, 64:64 + 256].view(2 * n, 4, 64)
    seen, depths, _ = nd.noble_tree_rows(_ints(_trees(random.Random(1), 2, n)), h.len)
    means = nd.noble_page_means(*h.args(), 100)
    chosen = nd.noble_block_select(q, means, h.table, h.len, 3, page=16)
    assert bool((chosen == nd.noble_block_select(q.contiguous(), means, h.table, h.len, 3, page=16)).all())
    one = q[:1, :1].expand(2 * n, 4, 64)
    for call in (lambda q, **kw: nd.noble_attn_tree(q, *h.args(), seen, depths, **kw),
                 lambda q, **kw: nd.noble_attn_blocks(q, *h.args(), chosen, **kw),
                 lambda q, **kw: nd.noble_attn_weigh(q, *h.args(), **kw)[0]):
        _same([call(q)], [call(q.contiguous())])
        _same([call(one)], [call(one.contiguous())])
        into = torch.full((2 * n, 4 * 64 + 64), 3.0, dtype=dt, device="cuda")
        o = into[:, :256].view(2 * n, 4, 64)
        assert call(q, o=o).data_ptr() == o.data_ptr()
        _same([o], [call(q)])
        assert bool((into[:, 256:] == 3.0).all())
        swapped = torch.empty((4, 2 * n, 64), dtype=dt, device="cuda").transpose(0, 1)   # heads outermost
        _same([call(q, o=swapped)], [call(q)])


def test_caches_past_4_gib():
    """Pages whose places need more than 32 bits, at the end of a cache of 6.4 GB."""
    page, K, D, H, n = 4096, 1, 128, 2, 3
    pages = 3050
    cache = torch.empty((pages, 2, K, page, D), dtype=BF, device="cuda")
    assert cache.numel() * 2 > 2 ** 32 * 1.4
    g = _gen(71)
    table = _ints([[pages - 1, 5], [pages - 2, 2100]])
    lens = [4100, 40]
    for b in range(2):
        for p in table[b].tolist():
            cache[p, :, :, :64].normal_(generator=g)
            cache[p, :, :, 64:] = 0.25
    q = torch.randn((2 * n, H, D), generator=g, device="cuda").to(BF)
    lengths = _ints(lens)
    parents = [[-1, 0, -1]] * 2
    seen, depths, _ = nd.noble_tree_rows(_ints(parents), lengths)
    o = nd.noble_attn_tree(q, cache, table, lengths, seen, depths)
    ow, w = nd.noble_attn_weigh(q, cache, table, lengths)
    means = nd.noble_page_means(cache, table, lengths, 5000)
    chosen = nd.noble_block_select(q, means, table, lengths, 2, page=page)
    ob = nd.noble_attn_blocks(q, cache, table, lengths, chosen)
    small = {p: cache[p:p + 1].cpu() for p in (pages - 1, 5, pages - 2, 2100)}
    for b in range(2):
        own = torch.cat([small[p] for p in table[b].tolist()])
        rows = slice(b * n, (b + 1) * n)
        want, mag, _, _ = ref.tree(q[rows].cpu(), own, [0, 1], lens[b], parents[b])
        _near("tree", o[rows], want, mag, U16)
        want, mag, ww, size = ref.weigh(q[rows].cpu(), own, [0, 1], lens[b])
        _near("weigh", ow[rows], want, mag, U16)
        _near("weights", w[b, :, :lens[b]], ww, torch.zeros_like(ww), (2 * (D + 3) * float(size.max()) + 20) * 2.0 ** -24)
        _near("blocks", ob[rows], want, mag, U16)
        mean = own[0, 0, :, :min(page, lens[b])].double().mean(1)
        assert float(((means[table[b, 0]].double().cpu() - mean).abs() - mean.abs() * 2.0 ** -8).max()) <= 1e-12
    before = cache[pages - 1].clone()
    nd.noble_cache_keep(cache, table, _ints([[[10, 4097]], [[1, 39]]]))
    assert bool((cache[pages - 1, :, :, 0] == before[:, :, 10]).all())
    assert bool((cache[pages - 1, :, :, 1].cpu() == small[5][0, :, :, 1]).all())
    assert bool((cache[pages - 2, :, :, 1].cpu() == small[pages - 2][0, :, :, 39]).all())


def test_sequences_may_share_pages_that_are_read():
    """A common prefix in the same pages: attention of every form, and weights of each sequence."""
    h = Held([70, 70, 70], 4, 2, 64, 8, F32, 81)
    h.table[1, :8] = h.table[2, :8] = h.table[0, :8]
    q = h.q(2)
    o, w = nd.noble_attn_weigh(q, *h.args())
    seen, depths, _ = nd.noble_tree_rows(_ints([[-1, 0]] * 3), h.len)
    t = nd.noble_attn_tree(q, *h.args(), seen, depths)
    for b, cache, table, length in h.each():
        want, mag, ww, _ = ref.weigh(q[2 * b:2 * b + 2].cpu(), cache, h.table[b].tolist(), length)
        _near("o", o[2 * b:2 * b + 2], want, mag, U32)
        _near("tree", t[2 * b:2 * b + 2], want, mag, U32)
        _near("weights", w[b, :, :length], ww, torch.zeros_like(ww), 2e-5)


def test_more_sequences_than_slots_and_lanes():
    """Workgroups that go through several sequences, more of them than a wave has lanes."""
    rng = random.Random(3)
    for K, n, H in ((1, 1, 1), (2, 3, 4), (1, 40, 2)):
        lengths = [rng.choice((0, 1, n, 17, 40, 41, 130)) for _ in range(150)]
        h = Held(lengths, H, K, 32, 8, BF, 91 + n)
        q = h.q(n)
        o, w = nd.noble_attn_weigh(q, *h.args())
        parents = _trees(rng, 150, n)
        seen, depths, _ = nd.noble_tree_rows(_ints(parents), h.len)
        t = nd.noble_attn_tree(q, *h.args(), seen, depths)
        p = na.noble_attn_paged(q, *h.args())
        torch.testing.assert_close(o.float(), p.float(), rtol=2 * U16, atol=2 * U16)
        for b, cache, table, length in list(h.each())[::7 if n < 40 else 40]:
            rows = slice(b * n, (b + 1) * n)
            want, mag, _, _ = ref.tree(q[rows].cpu(), cache, table, length, parents[b])
            _near("tree", t[rows], want, mag, U16)
        # every row that sees a token gives a weight of one for each query head
        total = sum(min(max(x, 0), n) for x in lengths) * H
        assert abs(float(w.double().sum()) - total) < 1e-4 * total


@pytest.mark.parametrize("lengths,n,H,K,D,dt", [([9001], 1, 4, 4, 128, BF), ([8200, 300], 3, 4, 2, 64, BF), ([5000], 2, 3, 1, 80, F32),
                                                ([4100, 0], 5, 1, 1, 64, F32), ([6500], 12, 4, 1, 128, BF), ([7000], 70, 2, 1, 64, BF)],
                         ids=["9001-1", "8200-3", "5000-2-f32", "4100-5-f32", "6500-48rows", "7000-140rows"])
def test_rows_of_many_pieces(lengths, n, H, K, D, dt):
    """Few long sequences, whose rows are put together from dozens of pieces: pieces without a page, and values that are no
    numbers in the first, in one between and in the last, for the rows that see them."""
    u = U16 if dt == BF else U32
    for spoiled in (False, True):
        h = Held(lengths, H, K, D, 16, dt, 97 + n)
        rows = h.table.tolist()
        if spoiled:
            h.table[0, 20:200] = -1
            h.cache[rows[0][0], 1, 0, 3, 1] = math.inf
            h.cache[rows[0][-40], 1, K - 1, 7, 5] = math.nan
            h.cache[rows[0][(lengths[0] - 1) // 16], 1, 0, (lengths[0] - 1) % 16, 0] = -math.inf   # its own row's alone
        q, parents = h.q(n), _trees(random.Random(n), len(lengths), n, 0.0)
        seen, depths, _ = nd.noble_tree_rows(_ints(parents), h.len)
        t = nd.noble_attn_tree(q, *h.args(), seen, depths)
        o, w = nd.noble_attn_weigh(q, *h.args())
        blocks = max(lengths) // 16
        lists = [[[j for j in range(max(0, x - n + i) // 16 + 1) if j % 3] for _ in range(K)] if x else [[]] * K
                 for x in lengths for i in range(n)]
        chosen = torch.tensor([[(x + [-1] * blocks)[:blocks] for x in y] for y in lists], dtype=torch.int32)
        s = nd.noble_attn_blocks(q, *h.args(), chosen.cuda())
        for b, cache, table, length in h.each():
            mine = slice(b * n, (b + 1) * n)
            want, mag, _, _ = ref.tree(q[mine].cpu(), cache, table, length, parents[b])
            _near("tree", t[mine], want, mag, u)
            want, mag, ww, size = ref.weigh(q[mine].cpu(), cache, table, length)
            _near("o", o[mine], want, mag, u)
            # as for the weights of shorter sequences: two scores' roundings, and one for every term of the sum
            terms = (2 * (D + 3) * float(size.max() if size.numel() else 0) + 16 + n * H // K) * 2.0 ** -24
            _near("weights", w[b, :, :ww.shape[1]], ww, torch.zeros_like(ww), terms)
            want, mag, _, _ = ref.blocks(q[mine].cpu(), cache, table, length, chosen[mine])
            _near("blocks", s[mine], want, mag, u)


def _roomy(h, n):
    """Room for sequences so long that the calls take more than one group of 16 rows to a workgroup."""
    tiles = -(-n * h.H // h.K // 16)
    room = 8192 * 32 // (len(h.lengths) * h.K * tiles * h.page) + 1
    h.table = torch.cat([h.table, torch.full((len(h.lengths), room), -1, dtype=torch.int32, device="cuda")], 1)
    return h


@pytest.mark.parametrize("case", [c for c in TREES if c[1] * c[2] > 16 * c[3]], ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}over{c[3]}")
def test_trees_in_tables_with_room(case):
    lengths, n, H, K, D, page, dt, cap, bias = case
    h = _roomy(Held(lengths, H, K, D, page, dt, 3), n)
    for b in range(1, len(lengths)):               # values that are no numbers, the last one seen by its own row alone
        if lengths[b] > n:
            h.cache[int(h.table[b, 0]), 1, 0, 1, 2] = math.inf
            h.cache[int(h.table[b, (lengths[b] - 1) // page]), 1, K - 1, (lengths[b] - 1) % page, 3] = math.nan
    q, parents, sl = h.q(n), _trees(random.Random(5), len(lengths), n), _slopes(H) if bias else None
    seen, depths, _ = nd.noble_tree_rows(_ints(parents), h.len)
    o = nd.noble_attn_tree(q, *h.args(), seen, depths, sl, softcap=cap)
    for b, cache, table, length in h.each():
        want, mag, _, _ = ref.tree(q[b * n:(b + 1) * n].cpu(), cache, table, length, parents[b], softcap=cap, slopes=sl)
        _near(f"o of {b}", o[b * n:(b + 1) * n], want, mag, U16 if dt == BF else U32)


@pytest.mark.parametrize("case", [c for c in WEIGHS if c[1] * c[2] > 16 * c[3]], ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}over{c[3]}")
def test_weights_in_tables_with_room(case):
    lengths, n, H, K, D, page, dt, cap, bias = case
    h = _roomy(Held(lengths, H, K, D, page, dt, 31), n)
    q, sl = h.q(n), _slopes(H) if bias else None
    o, w = nd.noble_attn_weigh(q, *h.args(), None, sl, softcap=cap)
    for b, cache, table, length in h.each():
        want, mag, ww, size = ref.weigh(q[b * n:(b + 1) * n].cpu(), cache, table, length, softcap=cap, slopes=sl)
        _near(f"o of {b}", o[b * n:(b + 1) * n], want, mag, U16 if dt == BF else U32)
        u = (2 * (D + 3) * float(size.max() if size.numel() else 0) + 16 + n * H // K) * 2.0 ** -24   # see test_attn_weigh
        _near(f"weights of {b}", w[b, :, :ww.shape[1]], ww, torch.zeros_like(ww), u)


def test_rows_of_minus_infinity_and_large_scores():
    """Scores that are all minus infinity give NaN, as the formula does; scores of thousands neither overflow nor lose the
    largest."""
    h = Held([40, 40], 2, 1, 64, 8, F32, 95)
    h.cache[:, 0] = h.cache[:, 0].abs()
    q = h.q(1, std=300.0)
    q[0] = -math.inf
    o, w = nd.noble_attn_weigh(q, *h.args())
    assert bool(torch.isnan(o[0]).all()) and bool(torch.isnan(w[0, :, :40]).all())
    want, mag, ww, size = ref.weigh(q[1:].cpu(), h.cache.cpu(), h.table[1].tolist(), 40)
    u = 2 * 67 * float(size.max()) * 2.0 ** -24
    _near("o", o[1:], want, mag, max(u, U32))
    assert float((w[1, :, :40].double().cpu() - ww).abs().max()) <= u


def test_nothing_to_do():
    """No sequences' tokens, empty tables, no pages: zeros and nothing written."""
    z = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    q, cache = torch.ones(4, 2, 16, device="cuda"), torch.ones(3, 2, 1, 8, 16, device="cuda")
    for table in (z(2, 0), z(2, 3)):
        lens = z(2)
        seen, depths, positions = nd.noble_tree_rows(_ints([[-1, 0]] * 2), lens)
        assert positions.tolist() == [[0, 0]] * 2
        assert bool((nd.noble_attn_tree(q, cache, table, lens, seen, depths) == 0).all())
        o, w = nd.noble_attn_weigh(q, cache, table, lens)
        assert bool((o == 0).all()) and bool((w == 0).all()) and w.shape == (2, 1, 8 * table.shape[1])
        means = torch.ones(3, 1, 16, device="cuda")
        nd.noble_page_means(cache, table, lens, 2, means)
        chosen = nd.noble_block_select(q, means, table, lens, 3, page=8)
        assert bool((chosen == -1).all()) and bool((means == 1).all())
        assert bool((nd.noble_attn_blocks(q, cache, table, lens, chosen) == 0).all())
        kept, left = nd.noble_evict_select(w, lens, 4)
        assert bool((kept == -1).all()) and bool((left == 0).all())
        if table.shape[1]:
            nd.noble_cache_keep(cache, table, kept)
        nd.noble_cache_keep(cache, table, kept[:, :, :0].contiguous())
        assert bool((cache == 1).all())
    empty = torch.empty(0, 2, 1, 8, 16, device="cuda")
    assert bool((nd.noble_attn_tree(q, empty, z(2, 3), _ints([9, 20]), seen, depths) == 0).all())
    assert nd.noble_cache_keep(empty, z(2, 3), _ints([[[4]], [[9]]])) is empty


def test_refusals_on_the_gpu():
    c = Calls(BF)
    h, q = c.h, c.q
    seen, depths, _ = nd.noble_tree_rows(c.parents, h.len)
    for bad in (lambda: nd.noble_attn_tree(q, *h.args(), seen[:, :1], depths),
                lambda: nd.noble_attn_tree(q, *h.args(), seen, depths[:1]),
                lambda: nd.noble_attn_tree(q[:-1], *h.args(), seen, depths),
                lambda: nd.noble_attn_tree(q, h.cache[:, :1], h.table, h.len, seen, depths),
                lambda: nd.noble_attn_blocks(q, *h.args(), torch.zeros(3, 2, 4, dtype=torch.int32, device="cuda")),
                lambda: nd.noble_attn_weigh(q, *h.args(), c.weights[:, :, :-8].contiguous()),
                lambda: nd.noble_attn_weigh(q, *h.args(), out=c.weights[:, :1].contiguous()),
                lambda: nd.noble_block_select(q, c.means, h.table, h.len, -1, page=16),
                lambda: nd.noble_block_select(q, c.means, h.table, h.len, 2 ** 32 + 5, page=16),
                lambda: nd.noble_page_means(*h.args(), -1, c.means),
                lambda: nd.noble_page_means(*h.args(), 2 ** 31, c.means),
                lambda: nd.noble_evict_select(c.weights, h.len, 2 ** 31),
                lambda: nd.noble_cache_keep(h.cache, h.table, torch.zeros(4, 3, 5, dtype=torch.int32, device="cuda")),
                lambda: nd.noble_tree_rows(c.parents[0], h.len)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: nd.noble_attn_tree(q.float(), *h.args(), seen, depths),
                lambda: nd.noble_attn_tree(q, h.cache, h.table.long(), h.len, seen, depths),
                lambda: nd.noble_attn_tree(q, h.cache, h.table, None, seen, depths),
                lambda: nd.noble_attn_tree(q, *h.args(), None, depths),
                lambda: nd.noble_attn_weigh(q, *h.args(), c.weights.bfloat16()),
                lambda: nd.noble_page_means(*h.args(), 1, c.means.float()),
                lambda: nd.noble_tree_rows(c.parents, None)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: nd.noble_block_select(q, c.means, h.table, h.len, 2, page=16, sink=2, local=1),
                lambda: nd.noble_block_select(q, c.means, h.table, h.len, 2, page=17),
                lambda: nd.noble_evict_select(c.weights, h.len, 3, sink=2, recent=2),
                lambda: nd.noble_evict_select(c.weights, h.len, 0),
                lambda: nd.noble_page_means(*h.args(), 0, c.means),
                lambda: nd.noble_attn_weigh(q, *h.args(), softcap=-1.0)):
        with pytest.raises(nd.NobleError):
            bad()
