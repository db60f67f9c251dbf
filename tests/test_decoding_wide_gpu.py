"""The kernels of many rows to a key head, attn_wide_kernel and attn_decode_kernel with two groups of rows, at the edges of their
calls: page tables with so much room that the calls take them (test_decoding_launches holds that they do), pages that are none,
values that are no numbers, rows of many pieces, many sequences, strides, graphs, caches past 4 GiB; and prompts through the
calls that are for few tokens."""

import math
import random

import pytest
import torch

import _decoding as ref
import test_decoding_edges_gpu as edges
from _attention import U16, U32
from paper_2603_06492_amd import attention as na
from paper_2603_06492_amd import decoding as nd
from paper_2603_06492_amd.attention import NobleSelfAttention, PagedCache
from test_decoding_gpu import BF, F32, Held, _gen, _ints, _near, _slopes, _trees

pytestmark = pytest.mark.gpu


def table_pages(lengths, n, H, K, page):
    """Columns of a page table with room for so many chunks of 32 tokens that the calls take more than one group of 16 rows to a
    workgroup, behind those of the longest sequence."""
    tiles = -(-n * H // K // 16)
    return max(1, -(-max(lengths) // page) + 1) + 8192 * 32 // (len(lengths) * K * tiles * page) + 1


class Roomy(Held):
    def __init__(self, lengths, n, H, K, D, page, dt, seed):
        super().__init__(lengths, H, K, D, page, dt, seed)
        more = table_pages(lengths, n, H, K, page) - self.per
        self.table = torch.cat([self.table, torch.full((len(lengths), more), -1, dtype=torch.int32, device="cuda")], 1)
        self.per = self.table.shape[1]


def _terms(n, H, K, D, size):
    """A weight's error by its roundings: two scores', and one for every term of the sum (see test_attn_weigh)."""
    size = size[torch.isfinite(size)]   # of the rows that have numbers
    return (2 * (D + 3) * float(size.max() if size.numel() else 0) + 16 + n * H // K) * 2.0 ** -24


def _infinite(got, want, p, cache, table, length):
    """What is wanted of o, with NaN for infinity where got has it and 32 bits cannot hold p [n, H, tokens], the infinite value's
    probability: it is the product of three factors (the score's, its wave's, its piece's, exp2 of a difference each) over their
    sum, of which one that is below float32's normal numbers, 2^-126, is zero, and 0 times infinity is NaN.  From 2^-100 on none
    is: each is at most 2^8, by which a running maximum may be short, the sum at least 2^-8, and 2^-100 2^-8 / 2^16 = 2^-124."""
    v, H = ref.gather(cache, table, length)[1], p.shape[1]
    largest = torch.zeros(want.shape, dtype=torch.float64)
    for t in torch.isinf(v).flatten(1).any(1).nonzero()[:, 0].tolist():
        largest = torch.maximum(largest, p[:, :, t, None] * torch.isinf(v[t]).repeat_interleave(H // v.shape[1], 0))
    either = torch.isinf(want) & (largest < 2.0 ** -100)
    return torch.where(either & torch.isnan(got.double().cpu()), math.nan, want)


def _against_reference(h, n, cap=0.0, sl=None, sequences=None, parents=None):
    """Tree and weighed attention of one set of inputs, every sequence or some, against the plain forms."""
    u = U16 if h.dt == BF else U32
    q = h.q(n)
    parents = _trees(random.Random(n), len(h.lengths), n) if parents is None else parents
    seen, depths, _ = nd.noble_tree_rows(_ints(parents), h.len)
    t = nd.noble_attn_tree(q, *h.args(), seen, depths, sl, softcap=cap)
    old = torch.rand((len(h.lengths), h.K, h.per * h.page), generator=h.g, device="cuda")
    o, w = nd.noble_attn_weigh(q, *h.args(), old, sl, softcap=cap)
    for b, cache, table, length in h.each():
        if sequences is not None and b not in sequences:
            continue
        mine = slice(b * n, (b + 1) * n)
        rows, how = q[mine].cpu(), dict(softcap=cap, slopes=sl)
        want, mag, p, _ = ref.tree(rows, cache, table, length, parents[b], **how)
        _near(f"tree {b}", t[mine], _infinite(t[mine], want, p, cache, table, length), mag, u)
        want, mag, ww, size = ref.weigh(rows, cache, table, length, old[b].cpu(), **how)
        if bool(torch.isinf(want).any()):   # a line of nodes sees what a row of new tokens does: its probabilities
            p = ref.tree(rows, cache, table, length, list(range(-1, n - 1)), **how)[2]
            want = _infinite(o[mine], want, p, cache, table, length)
        _near(f"o of {b}", o[mine], want, mag, u)
        _near(f"weights of {b}", w[b, :, :ww.shape[1]], ww, torch.zeros_like(ww), _terms(n, h.H, h.K, h.D, size))
        assert bool((w[b, :, ww.shape[1]:] == 0).all())
    return q, o, w


PIECES = [   # lengths, n, H, K, D, page, dtype, softcap, bias
    ([7000, 300], 70, 2, 1, 64, 16, BF, 0.0, False),      # eight waves, pages smaller than a tile
    ([5000, 64, 70], 64, 4, 1, 128, 128, BF, 0.0, True),  # one row tile to the last row, pages of two tiles
    ([4200, 40], 33, 16, 2, 40, 64, BF, 30.0, False),     # two row tiles, the second of eight rows, a page a tile
    ([2600, 150], 43, 12, 4, 80, 32, BF, 20.0, True),     # 129 rows: a wave with one
    ([6500, 900], 12, 4, 1, 128, 8, BF, 0.0, False),      # four waves, two workgroups a CU
    ([3000, 33, 34], 33, 1, 1, 64, 64, BF, 0.0, True),    # a row more than two groups
    ([2100, 130], 100, 1, 1, 32, 8, BF, 50.0, False),
    ([1900, 65], 32, 4, 1, 96, 16, BF, 30.0, False),      # 128 rows
    ([3900, 20], 24, 1, 1, 64, 8, BF, 0.0, False),        # two groups of rows
    ([2200, 70], 5, 16, 4, 128, 32, BF, 0.0, True),
    ([3300, 150], 20, 2, 1, 128, 16, F32, 0.0, False),    # float32: two groups, several row tiles
    ([1700, 41], 17, 1, 1, 40, 8, F32, 20.0, True),
]


@pytest.mark.parametrize("case", PIECES, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}over{c[3]}x{c[4]}-{c[5]}-{'bf16' if c[6] == BF else 'f32'}")
def test_pieces_missing_pages_and_what_is_no_number(case):
    """Rows of many pieces; and with pages that are none, a run of them and single ones, among the tokens that all rows see and
    among the new ones, with values and a key that are no numbers, in the first page, between and in the last, for who sees them."""
    lengths, n, H, K, D, page, dt, cap, bias = case
    sl = _slopes(H) if bias else None
    for spoiled in (False, True):
        h = Roomy(lengths, n, H, K, D, page, dt, 97 + n)
        rows = h.table.tolist()
        last = (lengths[0] - 1) // page
        if spoiled:
            h.cache[rows[0][0], 1, 0, 3, 1] = math.inf
            h.cache[rows[0][last // 2], 1, K - 1, 7, 5] = math.nan
            h.cache[rows[0][last], 1, 0, (lengths[0] - 1) % page, 0] = -math.inf      # its own row's alone
            h.cache[rows[1][(lengths[1] - 2) // page], 0, K - 1, (lengths[1] - 2) % page, 2] = math.nan   # a new token's key
            h.table[0, 2:max(3, last // 3)] = -1
            h.table[0, last // 2 + 1], h.table[0, last // 2 + 3] = h.pages, 2 ** 31 - 1
            if n > page:
                h.table[0, (lengths[0] - n) // page + 1] = -7                         # among the new tokens
            if len(lengths) > 2:
                h.table[2] = -1                                                       # nothing at all
        _against_reference(h, n, cap, sl)


MANY = [   # 150 sequences each, see test_many_sequences
    ([0] * 149 + [190], 40, 2, 1, 32, 8, BF, 0.0, False),
    ([0] * 149 + [300], 150, 1, 1, 64, 16, BF, 0.0, False),
    ([0] * 149 + [170], 20, 1, 1, 32, 8, BF, 0.0, False),
    ([0] * 149 + [170], 20, 2, 1, 32, 8, F32, 0.0, False),
    ([0] * 149 + [200], 70, 4, 2, 128, 64, BF, 30.0, False),
]


@pytest.mark.parametrize("case", MANY, ids=lambda c: f"{c[1]}-{c[2]}over{c[3]}x{c[4]}-{'bf16' if c[6] == BF else 'f32'}")
def test_many_sequences(case):
    """More of them than a wave has lanes, of no tokens, fewer than the new ones, as many, and more: workgroups go through
    several."""
    most, n, H, K, D, page, dt, cap, _ = case
    rng = random.Random(3)
    lengths = [rng.choice((0, 1, n, 17, n + 1, n + 20, max(most))) for _ in range(149)] + [max(most)]
    h = Roomy(lengths, n, H, K, D, page, dt, 91 + n)
    q, o, w = _against_reference(h, n, cap, sequences=set(range(0, 150, 29)) | {149})
    # every sequence: the paged attention's rows, either side off by u of itself and of sum p |v| at most
    p = na.noble_attn_paged(q, *h.args(), softcap=cap)
    u = 2 * (U16 if dt == BF else U32)
    v = h.cache[:, 1].float()
    torch.testing.assert_close(o.float(), p.float(), rtol=u, atol=u * float(v[torch.isfinite(v)].abs().max()))


CALLS = [   # of edges.Calls: four sequences of up to 150 tokens
    ([150, 64, 45, 41], n, 4, 2, 64, 16, dt, 0.0, False) for n, dt in ((12, BF), (20, BF), (40, BF), (70, BF), (12, F32), (20, F32))]


@pytest.fixture
def roomy(monkeypatch):
    """Lets the tests of edges make tables with room for calls of n new tokens."""
    def use(n):
        monkeypatch.setattr(edges, "Held", lambda lengths, H, K, D, page, dt, seed: Roomy(lengths, n, H, K, D, page, dt, seed))
    return use


@pytest.mark.parametrize("dt,n", [(c[6], c[1]) for c in CALLS], ids=lambda x: str(x).replace("torch.", ""))
def test_captured_and_replayed(dt, n, roomy):
    roomy(n)
    edges.test_captured_and_replayed(dt, n)


@pytest.mark.parametrize("dt,n", [(c[6], c[1]) for c in CALLS], ids=lambda x: str(x).replace("torch.", ""))
def test_strided_queries_and_outputs(dt, n, roomy):
    roomy(n)
    edges.test_strided_queries_and_outputs(dt, n)


@pytest.mark.parametrize("dt,n", [(BF, 20), (BF, 70), (F32, 12)], ids=lambda x: str(x).replace("torch.", ""))
def test_another_stream_and_the_python_calls(dt, n, roomy):
    roomy(n)
    c = edges.Calls(dt, n, (150, 64, 45, 41))
    want = c.run()
    edges._same(c.run(), want)
    edges._same(c.run(stream=torch.cuda.current_stream()), want)
    given = [t.clone() for t in (c.h.cache, c.means, c.weights)]
    torch.cuda.synchronize()
    side, big = torch.cuda.Stream(), torch.randn(2048, 2048, device="cuda")
    for _ in range(30):
        big = big @ big * 1e-3
    got = c.over(*given, stream=side)
    torch.cuda.synchronize()
    edges._same(got, want)


LARGE = [([4100, 100], n, 2, 1, 128, 4096, dt, 0.0, False) for n, dt in ((40, BF), (70, BF), (12, BF), (12, F32))]


@pytest.mark.parametrize("dt,n", [(c[6], c[1]) for c in LARGE], ids=lambda x: str(x).replace("torch.", ""))
def test_caches_past_4_gib(dt, n):
    """Pages whose places need more than 32 bits, at the end of a cache of 6.4 GB or more."""
    page, K, D, H, pages, lens = 4096, 1, 128, 2, 3050, LARGE[0][0]
    cache = torch.empty((pages, 2, K, page, D), dtype=dt, device="cuda")
    assert cache.numel() * cache.element_size() > 2 ** 32 * 1.4
    g = _gen(71)
    table = torch.full((2, table_pages(lens, n, H, K, page)), -1, dtype=torch.int32, device="cuda")
    own = [[pages - 1, 5], [pages - 2, 2100]]
    for b in range(2):
        table[b, :2] = _ints(own[b])
        for p in own[b]:
            cache[p, :, :, :128].normal_(generator=g)
            cache[p, :, :, 128:] = 0.25
    q = torch.randn((2 * n, H, D), generator=g, device="cuda").to(dt)
    lengths, parents = _ints(lens), _trees(random.Random(n), 2, n)
    seen, depths, _ = nd.noble_tree_rows(_ints(parents), lengths)
    t = nd.noble_attn_tree(q, cache, table, lengths, seen, depths)
    o, w = nd.noble_attn_weigh(q, cache, table, lengths)
    u = U16 if dt == BF else U32
    for b in range(2):
        mine = slice(b * n, (b + 1) * n)
        small = torch.cat([cache[p:p + 1].cpu() for p in own[b]])
        want, mag, _, _ = ref.tree(q[mine].cpu(), small, [0, 1], lens[b], parents[b])
        _near("tree", t[mine], want, mag, u)
        want, mag, ww, size = ref.weigh(q[mine].cpu(), small, [0, 1], lens[b])
        _near("o", o[mine], want, mag, u)
        _near("weights", w[b, :, :lens[b]], ww, torch.zeros_like(ww), _terms(n, H, K, D, size))


@pytest.mark.parametrize("n,dt", [(20, BF), (70, BF), (24, F32)], ids=lambda x: str(x).replace("torch.", ""))
def test_rows_of_minus_infinity_and_large_scores(n, dt):
    """Scores that are all minus infinity give NaN, as the formula does; scores of thousands neither overflow nor lose the
    largest."""
    D, lens = 64, [200, 90]
    h = Roomy(lens, n, 2, 1, D, 8, dt, 95)
    h.cache[:, 0] = h.cache[:, 0].abs()
    q = h.q(n, std=300.0)
    q[0] = -math.inf
    o, w = nd.noble_attn_weigh(q, *h.args())
    assert bool(torch.isnan(o[0]).all()) and bool(torch.isnan(w[0, :, :lens[0] - n + 1]).all())
    assert bool(torch.isfinite(w[0, :, lens[0] - n + 1:]).all())   # which that row does not see
    for b, first in ((0, 1), (1, 0)):
        rows = q[b * n:(b + 1) * n].cpu()
        want, mag, ww, size = ref.weigh(rows, h.cache.cpu(), h.table[b].tolist(), lens[b])
        # a score is off by at most (D + 3) 2^-24 of its sum of magnitudes, and so is its probability, twice with the sum's
        off = 2 * (D + 3) * float(size[first:].max()) * 2.0 ** -24
        _near("o", o[b * n + first:(b + 1) * n], want[first:], mag[first:], off + (U16 if dt == BF else U32))
        if b:
            # a row's probabilities are off by `off` of themselves: their sum by as much of itself
            _near("weights", w[b, :, :lens[b]], ww, torch.zeros_like(ww), off + (16 + 2 * n) * 2.0 ** -24)


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H,K,D,page,count", [(4, 2, 64, 8, 9), (2, 1, 128, 64, 2)])
def test_prompts_over_selected_pages(dt, H, K, D, page, count):
    """Hundreds of new tokens, the first of them over one page, the last over many, and a sequence shorter than the prompt."""
    n, lengths = 150, [150, 260, 90]
    h = Held(lengths, H, K, D, page, dt, 29)
    q = h.q(n)
    means = nd.noble_page_means(*h.args(), n + 200)
    chosen = nd.noble_block_select(q, means, h.table, h.len, count, page=page, sink=1, local=1)
    o = nd.noble_attn_blocks(q, *h.args(), chosen)
    for b, cache, table, length in h.each():
        mine = slice(b * n, (b + 1) * n)
        picks = ref.select(q[mine].cpu(), means.cpu(), table, length, n, count, page, 1, 1)
        assert chosen[mine].cpu().tolist() == picks.tolist(), b
        want, mag, _, _ = ref.blocks(q[mine].cpu(), cache, table, length, picks)
        _near(f"o of {b}", o[mine], want, mag, U16 if dt == BF else U32)


def test_prompts_through_the_block():
    """A prompt's step over all of its pages by selection, and into a cache that keeps weights and has room for long sequences:
    the plain step's rows, and weights of one for each row and head."""
    block, B, n = NobleSelfAttention(128, 4, 16, kv_heads=2, longest=4096), 2, 90
    x = torch.randn(B * n, 128, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(BF)
    make = lambda longest, **kw: PagedCache(B, longest, 64, kv_heads=2, head_dim=32, page=8, **kw)  # noqa: E731
    plain, picked, weighed = make(200), make(200, means=True), make(60000, weights=True)
    want = block.step(x, plain, *plain.extend(n))
    got = block.step(x, picked, *picked.extend(n), blocks=12)
    # roundings to bf16 of the probabilities, the attention's output and the O layer's on either side: half a step, 2^-8, each
    close = lambda a, b: float((a.float() - b.float()).norm() / b.float().norm()) < 6 * 2.0 ** -8  # noqa: E731
    assert close(got, want)
    few = make(200, means=True)
    assert not close(block.step(x, few, *few.extend(n), blocks=2), want)
    assert close(block.step(x, weighed, *weighed.extend(n)), want)
    total = weighed.weights[0].double().sum(2)
    assert float((total - 2 * n).abs().max()) < 1e-4 * 2 * n
    weighed.evict(40, sink=2, recent=8)
    assert weighed.held == 40 and weighed.seen == n
