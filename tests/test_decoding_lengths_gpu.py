"""Lengths that the page table does not hold, negative ones, and the outputs that a caller of the C ABI may leave out."""

import ctypes
import random

import pytest
import torch

import _decoding as ref
from _attention import U16, U32
from paper_2603_06492_amd import decoding as nd
from test_decoding_gpu import BF, F32, Held, _ints, _near, _numbered, _same, _trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 3, 20])
def test_lengths_are_cut_to_the_page_table_and_to_zero(dt, n):
    page, K, per = 8, 2, 9
    lengths = [per * page, per * page + 1, 1000, 2 ** 31 - 1, -1, -2 ** 31, 33]
    h = Held(lengths, 4, K, 64, page, dt, 101, per=per)
    q, u, rows = h.q(n), U16 if dt == BF else U32, h.table.tolist()
    parents = _trees(random.Random(4), len(lengths), n, 0.0)
    seen, depths, _ = nd.noble_tree_rows(_ints(parents), h.len)
    t = nd.noble_attn_tree(q, *h.args(), seen, depths)
    o, w = nd.noble_attn_weigh(q, *h.args())
    means = torch.full((h.pages, K, 64), 7.0, dtype=dt, device="cuda")
    nd.noble_page_means(*h.args(), n, means)
    every = nd.noble_page_means(*h.args(), 2 ** 31 - 4096)
    chosen = nd.noble_block_select(q, every, h.table, h.len, 5, page=page, sink=1, local=1)
    s = nd.noble_attn_blocks(q, *h.args(), chosen)
    for b, cache, table, length in h.each():
        mine, held = slice(b * n, (b + 1) * n), min(max(length, 0), per * page)
        want, mag, _, _ = ref.tree(q[mine].cpu(), cache, table, length, parents[b])
        _near("tree", t[mine], want, mag, u)
        want, mag, ww, size = ref.weigh(q[mine].cpu(), cache, table, length)
        _near("o", o[mine], want, mag, u)
        terms = (2 * 67 * float(size.max()) + 16 + 2 * n) * 2.0 ** -24   # see test_attn_weigh
        _near("weights", w[b, :, :held], ww, torch.zeros_like(ww), terms)
        assert bool((w[b, :, held:] == 0).all())
        picks = ref.select(q[mine].cpu(), every.cpu(), table, length, n, 5, page, 1, 1)
        assert chosen[mine].cpu().tolist() == picks.tolist(), b
        want, mag, _, _ = ref.blocks(q[mine].cpu(), cache, table, length, picks)
        _near("blocks", s[mine], want, mag, u)
        for c in range(per):
            got = means[rows[b][c]].double().cpu()
            if c in range(max(0, held - n) // page, -(-held // page)):
                mean = cache[rows[b][c], 0, :, :min(page, held - c * page)].double().mean(1)
                assert float(((got - mean).abs() - mean.abs() * (torch.finfo(dt).eps / 2)).max()) <= 1e-12, (b, c)
            else:
                assert bool((got == 7.0).all()), (b, c)


def test_outputs_that_are_left_out():
    """No positions (and then no lengths), no kept weights: the others as they are with them."""
    L, st = nd.lib(), torch.cuda.current_stream().cuda_stream
    for n in (7, 100):
        parents = _ints(_trees(random.Random(n), 5, n))
        seen, depths, _ = nd.noble_tree_rows(parents, _ints([200] * 5))
        s2, d2 = torch.full_like(seen, 3), torch.full_like(depths, 3)
        assert L.noble_tree_rows(5, n, parents.data_ptr(), None, s2.data_ptr(), d2.data_ptr(), None, st) == 0
        assert bool((s2 == seen).all()) and bool((d2 == depths).all())
    for row in (100, 9000, 40000):
        w, lens = torch.rand(3, 2, row, device="cuda"), _ints([row, 10, row - 1])
        kept, _ = nd.noble_evict_select(w, lens, 40, sink=3, recent=5)
        k2 = torch.full_like(kept, 9)
        d = nd.noble_evict_desc(3, row, 2, 40, 3, 5)
        assert L.noble_evict_select(ctypes.byref(d), w.data_ptr(), lens.data_ptr(), k2.data_ptr(), None, st) == 0
        assert bool((k2 == kept).all())


@pytest.mark.parametrize("most", [40, 300])
def test_lists_of_each_head_from_a_start_of_each_sequence(most):
    """Each key head its own list, behind tokens that stay where they are."""
    rng, lengths, start = random.Random(most), [700, 400, 350], [13, 0, 40]
    h = _numbered(Held(lengths, 3, 3, 40, 16, BF, 103))
    kept = [[sorted(rng.sample(range(x - s), min(most, x - s))) for _ in range(3)] for x, s in zip(lengths, start)]
    kept = [[x + [-1] * (most - len(x)) for x in row] for row in kept]
    before = h.cache.clone()
    nd.noble_cache_keep(h.cache, h.table, _ints(kept), _ints(start))
    want = before.cpu()
    for b, _, table, _ in h.each():
        want[table] = ref.keep(before.cpu(), table, kept[b], start[b])[table]
    assert _same(h.cache.cpu(), want)
