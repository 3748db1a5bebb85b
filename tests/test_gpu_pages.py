"""Positions that move, pages that are copied, and page lists of sequences that fork, grow and go, on the GPU against plain Python.
Needs an MI355X.  Everything here is exact."""
import numpy as np
import pytest
import torch

import paper_2411_03786_amd as ngg
from test_gpu_operators import ints, randn

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16, "fp4": torch.bfloat16}
CACHES = list(DT)


class Pool:
    """A pool of layers, all of whose places are written, and what it should hold: [layers, positions, heads, head_dim]."""

    def __init__(self, cache, layers, n_pages, page, Hkv, hd, seed=0):
        self.kv = ngg.KVPages(n_pages, page, Hkv, hd, cache, layers=layers)
        self.layers, self.n = layers, n_pages * page
        all_ = ints(np.arange(layers * self.n))
        self.kv.write(*(randn(layers * self.n, Hkv, hd, seed=seed + i, dtype="f32" if cache == "f32" else "bf16") for i in (1, 2)), all_)
        self.all, self.dtype = all_, DT[cache]
        self.k, self.v = (t.view(layers, self.n, Hkv, hd).clone() for t in self.kv.read(all_, self.dtype))

    def move(self, src, dst):
        for s, d in zip(src, dst):
            ok = [(a, b) for a, b in zip(s, d) if 0 <= a < self.n and 0 <= b < self.n]
            for x in (self.k, self.v):
                old = x.clone()
                for a, b in ok:
                    x[:, b] = old[:, a]

    def check(self):
        k, v = self.kv.read(self.all, self.dtype)
        assert torch.equal(k.view_as(self.k), self.k) and torch.equal(v.view_as(self.v), self.v)


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("layers,Hkv,hd,page", [(1, 1, 32, 32), (3, 3, 64, 96), (2, 8, 128, 64), (5, 2, 128, 32)])
@pytest.mark.parametrize("lists,n", [(1, 1), (1, 4), (3, 16), (2, 17), (1, 40), (1, 100)])
def test_moves(cache, layers, Hkv, hd, page, lists, n):
    """Sources and destinations in any order, overlapping, with entries left out and out of range."""
    pages = -(-lists * n * 2 // page) + 1
    p = Pool(cache, layers, pages, page, Hkv, hd)
    rng = np.random.default_rng(n)
    for trial in range(2):
        mine = rng.permutation(p.n)[:lists * n * 2].reshape(lists, 2 * n)       # a list's own places
        src = np.stack([rng.permutation(m)[:n] for m in mine])
        dst = np.stack([rng.permutation(m)[:n] for m in mine])
        if trial:
            src[:, ::5], dst[:, 3::7] = -1, p.n
            src[0, -1], dst[0, 0] = 2 ** 31 - 1, -2 ** 31
        p.kv.move(ints(src), ints(dst))
        p.move(src, dst)
        p.check()


@pytest.mark.parametrize("cache", CACHES)
def test_paths_move_behind_the_context(cache):
    """What a verified tree leaves: rising nodes of every sequence's tree go to where the context ends; nothing else changes."""
    B, ctx, page = 4, (0, 31, 45, 100), 32
    p = Pool(cache, 3, B * 5, page, 2, 64)
    table = np.random.default_rng(1).permutation(B * 5).reshape(B, 5)
    paths = [[0, 1, 2], [0, 2, 5, 6, 40], [0], [0, 3, 4, 50]]
    slot = lambda b, q: int(table[b, q // page]) * page + q % page
    src = [[slot(b, c + x) for x in path] + [-1] * (5 - len(path)) for b, (c, path) in enumerate(zip(ctx, paths))]
    dst = [[slot(b, c + i) for i in range(len(path))] + [-1] * (5 - len(path)) for b, (c, path) in enumerate(zip(ctx, paths))]
    p.kv.move(ints(src), ints(dst))
    p.move(src, dst)
    p.check()
    p.kv.move(ints(src[1]), ints(dst[1]))                               # one list without a dimension for lists
    p.move(src[1:2], dst[1:2])
    p.check()


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("n", [16, 20, 1024])
def test_the_last_of_equal_destinations_counts_and_chains_turn(cache, n):
    p = Pool(cache, 2, n // 32 + 2, 32, 1, 64)
    ring = np.arange(n)
    p.kv.move(ints(ring), ints(np.roll(ring, 1)))                       # a cycle through all of them
    p.move([ring], [np.roll(ring, 1)])
    p.check()
    p.kv.move(ints(ring), ints(np.full(n, n + 3)))
    p.move([ring], [np.full(n, n + 3)])
    p.check()
    one = np.full(n, 5)                                                 # one source for many
    p.kv.move(ints(one), ints(ring))
    p.move([one], [ring])
    p.check()


def test_moves_of_slices_and_of_nothing():
    p = Pool("fp4", 2, 4, 32, 2, 32)
    src, dst = ints(np.arange(24).reshape(4, 6)), ints(64 + np.arange(24).reshape(4, 6))
    p.kv.move(src[:, 1:4], dst[:, 2:5])                                 # rows of something wider
    p.move(src[:, 1:4].tolist(), dst[:, 2:5].tolist())
    p.check()
    for a in (src[:0], src[:, :0], ints([])):
        p.kv.move(a, a)
    p.check()
    for exc, a, b in ((TypeError, src.long(), dst), (TypeError, src, dst[:2]), (ValueError, src.T, dst.T), (TypeError, src[None], dst[None]),
                      (ngg.NggError, torch.zeros(1, 1025, dtype=torch.int32, device="cuda"), torch.zeros(1, 1025, dtype=torch.int32, device="cuda")),
                      (ValueError, src.cpu(), dst.cpu())):
        with pytest.raises(exc):
            p.kv.move(a, b)


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("layers,Hkv,hd,page", [(1, 1, 32, 32), (3, 3, 64, 96), (2, 8, 128, 64), (4, 2, 128, 160)])
def test_copies(cache, layers, Hkv, hd, page):
    p = Pool(cache, layers, 12, page, Hkv, hd)
    k, v = (x.view(layers, 12, page, Hkv, hd) for x in (p.k, p.v))
    src, dst = [3, 0, -1, 3, 12, 7, 2 ** 31 - 1], [4, 11, 2, 5, 6, -1, 8]
    for positions in (None, [page, 1, page, 33, page, page, page], [0, -4, 0, page + 50, 9, 9, 9], [8, 9, 1, 24, 1, 1, 1], [31, 16, 1, 7, 1, 1, 1]):
        p.kv.copy(ints(src), ints(dst), None if positions is None else ints(positions))
        for i in (0, 1, 3):
            n = page if positions is None else min(page, -(-max(positions[i], 0) // 8) * 8)
            for x in (k, v):
                x[:, dst[i], :n] = x[:, src[i], :n]
        p.check()
        fresh = randn(page, Hkv, hd, seed=9, dtype="f32" if cache == "f32" else "bf16")
        for layer in range(layers):
            part = p.kv.layer(layer)
            part.write(fresh, fresh, ints(3 * page + np.arange(page)))
            k[layer, 3], v[layer, 3] = part.read(ints(3 * page + np.arange(page)), p.dtype)
    p.check()
    p.kv.copy(ints([]), ints([]))
    for exc, args in ((TypeError, (ints(src).long(), ints(dst))), (TypeError, (ints(src), ints(dst)[:3])), (TypeError, (ints(src), ints(dst), ints([1]))),
                      (ValueError, (ints(src), ints(dst).cpu()))):
        with pytest.raises(exc):
            p.kv.copy(*args)


def test_more_entries_than_a_launch_has_rows():
    p = Pool("fp4", 2, 6, 32, 1, 32)
    n = 65535 + 3
    src, dst = np.full(n, -1), np.full(n, -1)
    for i, (a, b) in {0: (3, 40), 65534: (50, 3), 65535: (7, 60), n - 1: (100, 9)}.items():
        src[i], dst[i] = a, b
    p.kv.move(ints(src[:, None]), ints(dst[:, None]))
    p.move(src[src >= 0][:, None], dst[src >= 0][:, None])
    p.check()
    src[src >= 0], dst[dst >= 0] = [0, 0, 1, 2], [3, 4, 5, -1]
    p.kv.copy(ints(src), ints(dst))
    for x in (p.k, p.v):
        for a, b in ((0, 3), (0, 4), (1, 5)):
            x[:, 32 * b:32 * b + 32] = x[:, 32 * a:32 * a + 32]
    p.check()


def test_layers_of_a_pool_are_pools():
    kv = ngg.KVPages(3, 32, 2, 64, "fp8", layers=4)
    x = randn(5, 2, 64, dtype="bf16")
    one = ngg.KVPages(3, 32, 2, 64, "fp8")
    one.write(x, x, ints([1, 40, 95, 3, 64]))
    kv.layer(2).write(x, x, ints([1, 40, 95, 3, 64]))
    for a, b in zip(kv._memory(), one._memory()):
        a = a.view(4, -1)
        assert torch.equal(a[2], b) and all((a[i] == (127 if len(b) < 1000 else 0)).all() for i in (0, 1, 3))
    assert torch.equal(kv.read(ints([2 * 96 + 95]))[0], one.read(ints([95]))[0])
    assert kv.n_pages == 12 and kv.layer(3).n_pages == 3
    q = randn(1, 1, 4, 64, seed=2, dtype="bf16")
    assert torch.equal(ngg.tree_attention(q, kv.layer(2), ints([[0, 1, 2]]), ints([1])), ngg.tree_attention(q, one, ints([[0, 1, 2]]), ints([1])))
    for i in (-1, 4):
        with pytest.raises(IndexError):
            kv.layer(i)


# ---- page lists -------------------------------------------------------------------------------------------------------

class Lists:
    """Page lists in plain Python."""

    def __init__(self, n_seqs, max_pages, n_pages, page):
        self.rows, self.lens, self.refs = [[] for _ in range(n_seqs)], [0] * n_seqs, [0] * n_pages
        self.max_pages, self.page = max_pages, page

    def cut(self, s, n):
        for p in self.rows[s][n:]:
            self.refs[p] -= 1
        del self.rows[s][n:]

    def fork(self, sources, targets):
        seqs = range(len(self.rows))
        done = set()
        for s, t in zip(sources, targets):
            if s not in seqs or t not in seqs or t in sources or t in done:
                done.add(t)
                continue
            done.add(t)
            self.cut(t, 0)
            self.rows[t] = self.rows[s][:-(-self.lens[s] // self.page)]
            self.lens[t] = self.lens[s]
            for p in self.rows[t]:
                self.refs[p] += 1

    def release(self, keep=None):
        for s in range(len(self.rows)):
            k = self.lens[s] if keep is None else keep[s]
            if k >= 0:
                self.lens[s] = min(self.lens[s], k)
                self.cut(s, -(-self.lens[s] // self.page))

    def reserve(self, new):
        n = len(self.rows)
        src, dst, positions = [-1] * n, [-1] * n, [0] * n
        need, short = [], 0
        part = {s: self.rows[s][self.lens[s] // self.page] for s in range(n)
                if new[s] > 0 and self.lens[s] % self.page and len(self.rows[s]) > self.lens[s] // self.page}
        for s in range(n):
            if new[s] <= 0:
                continue
            end = -(-(self.lens[s] + new[s]) // self.page)
            short += max(0, end - self.max_pages)
            if s in part and self.refs[part[s]] > 1:
                users = [t for t in part if part[t] == part[s]]
                if len(users) < self.refs[part[s]] or s != users[-1]:
                    need.append((s, self.lens[s] // self.page))
            need += [(s, j) for j in range(len(self.rows[s]), min(end, self.max_pages))]
        free = [p for p, r in enumerate(self.refs) if r == 0]
        missing = max(0, len(need) - len(free)) + short
        if not missing:
            for (s, j), p in zip(need, free):
                if j < len(self.rows[s]):
                    src[s], dst[s], positions[s] = self.rows[s][j], p, self.lens[s] % self.page
                    self.refs[self.rows[s][j]] -= 1
                    self.rows[s][j] = p
                else:
                    self.rows[s].append(p)
                self.refs[p] += 1
        return src, dst, positions, [missing]

    def check(self, table):
        rows = [r + [-1] * (self.max_pages - len(r)) for r in self.rows]
        assert table.pages.tolist() == rows and table.lens.tolist() == self.lens and table.refs.tolist() == self.refs
        counts = np.zeros(len(self.refs), int)
        for r in self.rows:
            np.add.at(counts, r, 1)
        assert counts.tolist() == self.refs


@pytest.mark.parametrize("n_seqs,max_pages,n_pages,page,seed", [(1, 1, 1, 32, 0), (3, 4, 9, 32, 1), (8, 20, 64, 64, 2), (40, 30, 500, 32, 3), (200, 9, 1100, 96, 4),
                                                               (1024, 3, 2500, 64, 5), (5, 900, 3000, 32, 6), (17, 300, 70000, 64, 7)])
def test_page_lists_of_a_life(n_seqs, max_pages, n_pages, page, seed):
    """Sequences that are forked, grow, are cut and given back, in any order."""
    rng = np.random.default_rng(seed)
    table, lists = ngg.PageTable(n_seqs, max_pages, n_pages, page), Lists(n_seqs, max_pages, n_pages, page)
    went, lacked = 0, 0
    for step in range(40 if n_seqs < 1000 else 12):
        what = rng.integers(0, 6)
        if what < 3:
            longest = max_pages * page
            new = np.where(rng.random(n_seqs) < 0.6, rng.integers(1, max(2, min(longest // 3, 4 * page)) + 1, n_seqs), rng.integers(-2, 1, n_seqs))
            if step % 7:                                                # sometimes past max_pages
                new = np.minimum(new, longest - np.array(lists.lens))
            r = table.reserve(ints(new))
            want = lists.reserve(new.tolist())
            assert [t.tolist() for t in r] == [list(w) for w in want]
            if want[3] == [0]:
                went += 1
                add = (np.maximum(new, 0) * rng.random(n_seqs)).astype(int) if step % 2 else np.maximum(new, 0)
                lists.lens = [a + int(b) for a, b in zip(lists.lens, add)]
                table.lens += ints(add)
            else:
                lacked += 1
        elif what < 5:
            n = int(rng.integers(1, n_seqs + 1))
            sources, targets = rng.integers(-1, n_seqs + 1, n), rng.integers(-1, n_seqs + 1, n)
            if step % 3:
                half = rng.permutation(n_seqs)
                sources, targets = half[:max(1, n_seqs // 4)].repeat(2), half[max(1, n_seqs // 4):][:2 * max(1, n_seqs // 4)]
                sources = sources[:len(targets)]
            table.fork(ints(sources), ints(targets))
            lists.fork(sources.tolist(), targets.tolist())
        else:
            keep = np.where(rng.random(n_seqs) < 0.5, rng.integers(0, max_pages * page, n_seqs), rng.integers(-2, 3, n_seqs) * 2 ** 30)
            keep = np.minimum(keep, 2 ** 31 - 1)
            if step % 4 == 0:
                table.release()
                lists.release()
            else:
                table.release(ints(keep))
                lists.release(keep.tolist())
        lists.check(table)
    assert went
    table.release(ints(np.zeros(n_seqs)))
    assert not table.refs.any() and (table.pages == -1).all() and not table.lens.any()


def test_more_pages_than_a_workgroup_keeps():
    """Thousands of pages in one call, from between others that are taken."""
    n_seqs, max_pages, n_pages, page = 17, 300, 9000, 32
    table, lists = ngg.PageTable(n_seqs, max_pages, n_pages, page), Lists(n_seqs, max_pages, n_pages, page)
    for new in ([page * (i + 1) for i in range(n_seqs)], [page * 220 - 3 * i for i in range(n_seqs)], [1] * n_seqs):
        r, want = table.reserve(ints(new)), lists.reserve(new)
        assert [t.tolist() for t in r] == [list(w) for w in want] and want[3] == [0]
        keep = [page * (i + 1) if i % 2 else 0 for i in range(n_seqs)]
        table.lens += ints(new)
        lists.lens = [a + b for a, b in zip(lists.lens, new)]
        if new[0] == page:
            table.release(ints(keep))
            lists.release(keep)
        lists.check(table)


def test_who_keeps_a_shared_page():
    """One prompt of 40 positions in pages of 32: its page of 8 positions."""
    def shared():
        t = ngg.PageTable(4, 4, 20, 32)
        t.reserve(ints([40, 0, 0, 0]))
        t.lens[0] = 40
        t.fork(ints([0, 0, 0]), ints([1, 2, 3]))
        assert t.refs.tolist()[:3] == [4, 4, 0] and t.pages[:, :2].tolist() == [[0, 1]] * 4
        return t
    t = shared()
    r = t.reserve(ints([1, 1, 1, 1]))                                   # all go on: the last keeps it
    assert [x.tolist() for x in r] == [[1, 1, 1, -1], [2, 3, 4, -1], [8, 8, 8, 0], [0]]
    assert t.refs.tolist()[:6] == [4, 1, 1, 1, 1, 0]
    t = shared()
    r = t.reserve(ints([0, 5, 0, 5]))                                   # it belongs to the others
    assert [x.tolist() for x in r] == [[-1, 1, -1, 1], [-1, 2, -1, 3], [0, 8, 0, 8], [0]]
    assert t.refs.tolist()[:5] == [4, 2, 1, 1, 0]
    r = t.reserve(ints([0, 5, 0, 5]))                                   # nothing is shared any more
    assert (r.src == -1).all() and (r.dst == -1).all() and not r.missing.any()


def test_too_few_pages_change_nothing():
    t = ngg.PageTable(3, 5, 6, 32)
    t.reserve(ints([64, 33, 0]))
    t.lens += ints([64, 33, 0])
    t.fork(ints([1]), ints([2]))
    before = [x.clone() for x in (t.pages, t.lens, t.refs)]
    for new, lacks in (([1, 1, 1], 0), ([65, 1, 32], 2), ([10 ** 9, 0, 0], 31250000 - 3), ([2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], None), ([0, 0, 130], 2)):
        r = t.reserve(ints(new))
        if lacks == 0:                                                  # two free pages and a copy
            assert r.missing.tolist() == [0]
            t.release()
            for x, b in zip((t.pages, t.lens, t.refs), before):
                x.copy_(b)
            continue
        assert (r.missing[0] > 0) if lacks is None else True
        assert (r.src == -1).all() and (r.dst == -1).all() and not r.positions.any()
        assert all(torch.equal(x, b) for x, b in zip((t.pages, t.lens, t.refs), before))
    r = t.reserve(ints([65, 1, 32]))
    # three pages for the first, a copy for the second (the third keeps the page) and one more for the third, of which two are there
    assert r.missing.tolist() == [3]


def test_tables_refuse_on_the_host():
    t = ngg.PageTable(3, 5, 6, 32)
    for exc, call in ((TypeError, lambda: t.reserve(ints([1, 2]))), (TypeError, lambda: t.reserve(ints([1, 2, 3]).long())), (TypeError, lambda: t.fork(ints([1]), ints([1, 2]))),
                      (TypeError, lambda: t.release(ints([1]))), (ValueError, lambda: t.release(ints([1, 1, 1]).cpu())),
                      (ngg.NggError, lambda: ngg.PageTable(3, 5, 6, 48).release()), (ngg.NggError, lambda: ngg.PageTable(1025, 5, 6, 32).release())):
        with pytest.raises(exc):
            call()
    t.fork(ints([]), ints([]))


def attend(q, kv, table):
    return ngg.tree_attention(q, kv, table.pages, table.lens)


@pytest.mark.parametrize("cache", CACHES)
def test_forked_sequences_read_what_copies_of_them_would(cache):
    """A prompt shared by three sequences that go on by themselves, in two layers, next to sequences that were given the prompt each."""
    page, Hkv, hd, L, n = 32, 2, 64, 2, 75
    dt = "f32" if cache == "f32" else "bf16"
    prompt = [[randn(n, Hkv, hd, seed=10 * i + j, dtype=dt) for j in range(2)] for i in range(L)]
    more = [[randn(3 * 30, Hkv, hd, seed=10 * i + j + 5, dtype=dt) for j in range(2)] for i in range(L)]
    kv, own = (ngg.KVPages(24, page, Hkv, hd, cache, layers=L) for _ in range(2))
    table = ngg.PageTable(3, 5, 24, page)
    slots = lambda s, pos: (table.pages[s, torch.tensor(pos) // page] * page + ints(pos) % page).int()
    table.reserve(ints([n, 0, 0]))
    for i in range(L):
        kv.layer(i).write(*prompt[i], slots(0, range(n)))
        for s in range(3):
            own.layer(i).write(*prompt[i], ints(s * 5 * page + np.arange(n)))
    table.lens += ints([n, 0, 0])
    table.fork(ints([0, 0]), ints([1, 2]))
    for at in range(0, 30, 10):
        r = table.reserve(ints([10, 10, 10]))
        kv.copy(r.src, r.dst, r.positions)
        assert (r.src >= 0).sum() == (2 if at == 0 else 0)
        for i in range(L):
            for s in range(3):
                part = [x[s * 30 + at:s * 30 + at + 10] for x in more[i]]
                kv.layer(i).write(*part, slots(s, range(n + at, n + at + 10)))
                own.layer(i).write(*part, ints(s * 5 * page + n + at + np.arange(10)))
        table.lens += 10
    lists = ints(np.arange(15).reshape(3, 5))
    q = randn(3, 1, 4, hd, seed=3, dtype=dt)
    for i in range(L):
        a = ngg.tree_attention(q, kv.layer(i), table.pages, table.lens - 1)
        b = ngg.tree_attention(q, own.layer(i), lists, table.lens - 1)
        assert torch.equal(a, b)
    assert int((table.refs > 0).sum()) < 12


def test_a_step_of_pages_in_a_graph_and_on_another_stream():
    """Fork, reserve, copy, write, attend, move and release, captured once and replayed with lengths and choices that change in place."""
    B, T, H, Hkv, hd, page, L = 4, 6, 4, 2, 64, 32, 3
    rng = np.random.default_rng(3)

    def start():
        kv = ngg.KVPages(40, page, Hkv, hd, "fp4", layers=L)
        kv.write(randn(L * 40 * page, Hkv, hd, seed=1, dtype="bf16"), randn(L * 40 * page, Hkv, hd, seed=2, dtype="bf16"), ints(np.arange(L * 40 * page)))
        table = ngg.PageTable(B, 8, 40, page)
        table.reserve(ints([70, 20, 0, 0]))
        table.lens += ints([70, 20, 0, 0])
        return kv, table
    sources, targets, new, path = ints([0, 1]), ints([2, 3]), ints([T] * B), ints([[0, 2, 3]] * B)
    keep = ints([2 ** 31 - 1] * B)
    x = randn(B * T, Hkv, hd, seed=4, dtype="bf16")
    q = randn(B, T, H, hd, seed=5, dtype="bf16")
    at = torch.arange(T, dtype=torch.int32, device="cuda")

    def step(kv, table):
        table.fork(sources, targets)
        r = table.reserve(new)
        kv.copy(r.src, r.dst, r.positions)
        place = table.lens[:, None] + at
        slots = torch.gather(table.pages, 1, (place // page).long()) * page + place % page
        outs = []
        for i in range(L):
            kv.layer(i).write(x, x, slots.flatten())
            outs.append(ngg.tree_attention(q, kv.layer(i), table.pages, table.lens))
        kv.move(torch.gather(slots, 1, path.long()), slots[:, :path.shape[1]])
        table.lens += 3
        table.release(keep)
        return [*outs, *r, table.pages.clone(), table.lens.clone(), table.refs.clone(), *kv.read(ints_all)]
    ints_all = ints(np.arange(L * 40 * page))
    kv, table = start()
    kv2, table2 = start()
    state = lambda k, t: (*k._memory(), t.pages, t.lens, t.refs)
    step(kv2, table2)                                                   # warm
    for a, b in zip(state(kv2, table2), state(kv, table)):
        a.copy_(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(kv, table)
    for i in range(4):
        sources.copy_(ints([i % 2, 1])), targets.copy_(ints([2, 3] if i % 2 else [3, 2]))
        new.copy_(ints([T, T + i, T, T])), keep.copy_(ints([2 ** 31 - 1, -1, 30 + i, 0 if i == 2 else 2 ** 31 - 1]))
        path.copy_(ints(np.sort(rng.permutation(T)[:3])[None].repeat(B, 0)))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = step(kv2, table2)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(state(kv, table), state(kv2, table2)))


def test_calls_on_a_named_stream():
    kv, table = ngg.KVPages(8, 32, 2, 32, "fp4", layers=2), ngg.PageTable(2, 4, 8, 32)
    side = torch.cuda.Stream()
    x = randn(16 * 32, 2, 32, dtype="bf16")
    kv.write(x, x, ints(np.arange(16 * 32)))
    side.wait_stream(torch.cuda.current_stream())
    table.reserve(ints([33, 0]), stream=side)
    with torch.cuda.stream(side):
        table.lens += ints([33, 0])
    table.fork(ints([0]), ints([1]), stream=side)
    r = table.reserve(ints([1, 1]), stream=side)
    kv.copy(r.src, r.dst, r.positions, stream=side)
    kv.move(ints([5, 6]), ints([6, 5]), stream=side)
    table.release(ints([0, -1]), stream=side)
    side.synchronize()
    assert r.src.tolist() == [1, -1] and r.dst.tolist() == [2, -1] and table.refs.tolist() == [1, 1, 0, 0, 0, 0, 0, 0]
    k = kv.read(ints(np.arange(16 * 32)))[0].view(2, 8, 32, 2, 32)
    assert torch.equal(k[:, 2, :8], k[:, 1, :8])
