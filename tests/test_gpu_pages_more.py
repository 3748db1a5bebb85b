"""Moves, copies and page lists beyond test_gpu_pages: fewer units than entries, long lists, many sequences that grow at once, what a call lacks.
Needs an MI355X.  Everything here is exact."""
import numpy as np
import pytest
import torch

import paper_2411_03786_amd as ngg
from test_gpu_operators import ints
from test_gpu_pages import CACHES, Lists, Pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_moves_of_more_entries_than_units(cache, hd):
    """One key head has as few as one unit of a kind: the lanes that have none still hold entries."""
    p = Pool(cache, 2, 3, 32, 1, hd)
    rng = np.random.default_rng(hd)
    for n in range(1, 17):
        mine = rng.permutation(p.n)
        src, dst = mine[:n], rng.permutation(mine[:2 * n])[:n]
        src[rng.random(n) < 0.2] = -1
        p.kv.move(ints(src), ints(dst))
        p.move([src], [dst])
        p.check()


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("n", [64, 65, 128, 129, 200, 256, 257, 500, 512, 513, 1023])
def test_long_moves(cache, n):
    """Lists that wait in LDS, by workgroups of 64 threads down to 4."""
    for layers, Hkv, hd, page in ((2, 3, 64, 96), (1, 1, 32, 32), (1, 2, 128, 160)):
        p = Pool(cache, layers, -(-4 * n // page) + 1, page, Hkv, hd, seed=n)
        rng = np.random.default_rng(n)
        mine = rng.permutation(p.n)[:4 * n].reshape(2, 2 * n)
        src, dst = (np.stack([rng.permutation(m)[:n] for m in mine]) for _ in range(2))
        src[:, ::7], dst[0, n // 2], src[1, -1] = -1, p.n, 2 ** 31 - 1
        p.kv.move(ints(src), ints(dst))
        p.move(src, dst)
        p.check()


@pytest.mark.parametrize("n_seqs,max_pages,page", [(1024, 12, 32), (700, 40, 64), (1024, 9, 160)])
def test_many_sequences_grow_by_many_pages(n_seqs, max_pages, page):
    """All threads count the entries of all sequences, and there are pages for them; forks among them go on in shared pages."""
    n_pages = n_seqs * max_pages + 3
    table, lists = ngg.PageTable(n_seqs, max_pages, n_pages, page), Lists(n_seqs, max_pages, n_pages, page)
    rng = np.random.default_rng(page)
    half = max_pages // 2 * page
    for step in range(4):
        new = rng.integers(0, half, n_seqs)
        new[rng.random(n_seqs) < 0.2] = 0
        new = np.minimum(new, max_pages * page - np.array(lists.lens))
        new[5] = min(5 * page, max_pages * page - lists.lens[5])
        r, want = table.reserve(ints(new)), lists.reserve(new.tolist())
        assert want[3] == [0] and [t.tolist() for t in r] == [list(w) for w in want]
        assert step or (new > 4 * page).any()
        lists.lens = [a + int(b) for a, b in zip(lists.lens, new)]
        table.lens += ints(new)
        lists.check(table)
        order = rng.permutation(n_seqs)
        sources, targets = order[:n_seqs // 4].repeat(2), order[n_seqs // 4:][:n_seqs // 4 * 2]
        table.fork(ints(sources), ints(targets))
        lists.fork(sources.tolist(), targets.tolist())
        keep = np.where(rng.random(n_seqs) < 0.5, rng.integers(0, half, n_seqs), -1)
        table.release(ints(keep))
        lists.release(keep.tolist())
        lists.check(table)


@pytest.mark.parametrize("new,lacks", [([65, 1, 32], 3), ([10 ** 9, 0, 0], 31250002 - 5 + 1), ([2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], None), ([0, 0, 130], 3), ([1, 1, 1], 0), ([33, 1, 0], 1)])
def test_how_many_pages_a_call_lacks(new, lacks):
    """Three sequences of 64, 33 and (forked from the second) 33 positions in six pages of 32, of which two are free, lists of five.  [65, 1, 32]: three pages, a copy
    for the second, of which the third keeps the page, and one more for the third.  10^9: 31250002 pages in all, of which five fit the
    list, two are there and two are free: one lacks beside those beyond the list.  [33, 1, 0]: two and a copy."""
    t, lists = ngg.PageTable(3, 5, 6, 32), Lists(3, 5, 6, 32)
    for x in (t, lists):
        x.reserve(ints([64, 33, 0]) if x is t else [64, 33, 0])
    t.lens += ints([64, 33, 0])
    lists.lens = [64, 33, 0]
    t.fork(ints([1]), ints([2]))
    lists.fork([1], [2])
    before = [x.clone() for x in (t.pages, t.lens, t.refs)]
    r, want = t.reserve(ints(new)), lists.reserve(new)
    assert r.missing.tolist() == want[3] and want[3][0] == (want[3][0] if lacks is None else lacks)
    if lacks != 0:
        assert (r.src == -1).all() and (r.dst == -1).all() and not r.positions.any() and r.missing[0] > 0
        assert all(torch.equal(x, b) for x, b in zip((t.pages, t.lens, t.refs), before))
