"""Operator cases: a paged cache held in 4 bits, the attention that reads it, and the life of a cache's pages.

Four operators of a program that serves several sequences whose drafts are verified as trees, next to those of ``operators.py``:

* ``cache4``   keys and values written into a paged cache in 4 bits, and read back,
* ``attend4``  attention of every sequence's tree of drafted tokens (or of its single new token) over a cache in 4 bits,
* ``move``     after a step: of every sequence's tree the accepted path moves behind the context, in all layers,
* ``pages``    sequences forked from prompts that they share: page lists and reference counts, pages for the new tokens, and copies
               of the pages that would be written to, in all layers.

Four bits are a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (nearest, ties to the even code), times a power of two for each position,
head and 32 dimensions: the smallest that brings all of them to 6 or below.  Keys in 4 bits are compared unrotated, since the four
bits of a rotated key hang on its last bit.

A case is a dict of plain values.  ``run`` with ``own`` false is the mathematics in elementary torch operations in 32 bits;
with ``own`` true it makes the framework's calls.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

# heads, key/value heads, head_dim: the attention shapes of the benchmark's workloads, all heads their own and four to a key head
HEADS = ((4, 4, 32), (8, 8, 64), (12, 12, 64), (12, 3, 64), (32, 32, 128), (32, 8, 128), (24, 24, 128), (24, 6, 128))
CACHES = ("f32", "bf16", "fp8", "fp4")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 32


def listed():
    return [
        # every sequence's new token, written and read in each layer and step: the smallest launches
        dict(op="cache4", name="cache4_append", batch=32, new=1, kv_heads=8, head_dim=128, dtype="bf16", page=64, start=2047, read=1),
        # the trees of 16 sequences in fp32, heads of 64, pages that end inside a tree
        dict(op="cache4", name="cache4_trees_f32", batch=16, new=61, kv_heads=12, head_dim=64, dtype="f32", page=32, start=777, read=61),
        # a long prompt
        dict(op="cache4", name="cache4_prompt", batch=1, new=16384, kv_heads=8, head_dim=128, dtype="bf16", page=64, start=0, read=16384),
        # the tree of one sequence of the tiny fp32 shape: launch and latency
        dict(op="attend4", name="attend4_tiny_f32", batch=1, tree=13, heads=4, kv_heads=4, head_dim=32, dtype="f32", page=32, context=128, ragged=False),
        # the tree of one sequence at the 7B shape behind a prompt of 2047 tokens
        dict(op="attend4", name="attend4_tree_7b", batch=1, tree=51, heads=32, kv_heads=32, head_dim=128, dtype="bf16", page=64, context=2047, ragged=False),
        # single tokens of many sequences behind long contexts of all lengths: what 4 bits are for
        dict(op="attend4", name="attend4_decode_batch", batch=32, tree=1, heads=32, kv_heads=8, head_dim=128, dtype="bf16", page=64, context=32000,
             ragged=True),
        # small trees in fp32, heads of 64, lengths of all kinds
        dict(op="attend4", name="attend4_trees_f32", batch=9, tree=7, heads=12, kv_heads=3, head_dim=64, dtype="f32", page=160, context=5001, ragged=True),
        # trees over long contexts: what a step costs at its largest
        dict(op="attend4", name="attend4_trees_32k", batch=8, tree=61, heads=32, kv_heads=8, head_dim=128, dtype="bf16", page=64, context=32000,
             ragged=True),
        # one sequence's accepted path in a model of two layers
        dict(op="move", name="move_path", batch=1, tree=13, path=4, layers=2, kv_heads=4, head_dim=32, dtype="f32", cache="f32", page=32, context=140),
        # the accepted paths of 16 sequences in all of 32 layers
        dict(op="move", name="move_paths_32_layers", batch=16, tree=61, path=9, layers=32, kv_heads=8, head_dim=128, dtype="bf16", cache="fp4", page=64,
             context=1000),
        # four continuations of one prompt
        dict(op="pages", name="pages_fork_4", parents=1, children=4, context=500, new=8, layers=12, kv_heads=12, head_dim=64, dtype="bf16", cache="bf16",
             page=64, pool=256),
        # four continuations of each of eight prompts of all lengths, in a pool that is not full
        dict(op="pages", name="pages_fork_32", parents=8, children=4, context=4010, new=100, layers=32, kv_heads=8, head_dim=128, dtype="bf16",
             cache="fp4", page=64, pool=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(("cache4", "cache4", "attend4", "attend4", "attend4", "attend4", "move", "move", "pages", "pages"))
    heads, kv_heads, hd = rng.choice(HEADS)
    dtype, page = rng.choice(("f32", "bf16", "bf16")), rng.choice((32, 64, 64, 160))
    if op == "cache4":
        batch, most = _log(rng, 1, 48), (1 << 24) // (kv_heads * hd)    # tokens
        new, start = _log(rng, 1, max(2, most // batch)), _log(rng, 1, 4096)
        return dict(op=op, batch=batch, new=new, kv_heads=kv_heads, head_dim=hd, dtype=dtype, page=page, start=start,
                    read=min(new + start, max(1, min(_log(rng, 1, 4 * new), most // batch))))
    if op == "attend4":
        while True:
            c = dict(op=op, batch=_log(rng, 1, 48), tree=1 if rng.random() < 0.3 else _log(rng, 2, 128), heads=heads, kv_heads=kv_heads,
                     head_dim=hd, dtype=dtype, page=page, context=_log(rng, 1, 65536), ragged=rng.random() < 0.6)
            w = work(c)
            if w["flops"] < 1.5e11 and w["bytes"] < 6e8 and c["batch"] * c["context"] * kv_heads * hd < 1e9:
                return c
    cache = rng.choice(CACHES)
    dtype = cache if cache in DTYPES else dtype
    layers = _log(rng, 1, 32)
    if op == "move":
        tree = _log(rng, 1, 128)
        batch = max(1, min(_log(rng, 1, 48), (1 << 25) // (layers * tree * kv_heads * hd)))
        return dict(op=op, batch=batch, tree=tree, path=_log(rng, 1, min(tree, 16)), layers=layers, kv_heads=kv_heads, head_dim=hd,
                    dtype=dtype, cache=cache, page=page, context=_log(rng, 1, 4096))
    while True:
        context, new, parents, children = _log(rng, 1, 8192), _log(rng, 1, 300), _log(rng, 1, 16), _log(rng, 1, 16)
        context += context % page == 0                                  # the last page is not full
        need = parents * (-(-context // page) + children * (2 + new // page))
        c = dict(op=op, parents=parents, children=children, context=context, new=new, layers=layers, kv_heads=kv_heads, head_dim=hd, dtype=dtype,
                 cache=cache, page=page, pool=int(need * rng.uniform(1.0, 3.0)))
        if work(c)["bytes"] < 3e8 and layers * c["pool"] * page * kv_heads * hd < 1 << 31:
            return c
        layers = max(1, layers // 2)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed % (1 << 30)) + salt)
    return g


def _fused(n, widths, dtype, gen):
    """Slices of one projection's output [n, sum of heads * head_dim], as [n, heads, head_dim] views.  A few features are larger than
    the others, as those of trained models are."""
    cols = sum(h * d for h, d in widths)
    x = torch.randn(n, cols, generator=gen, device="cuda")
    x *= torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.02, 4.0, 1.0)
    x = x.to(DTYPES[dtype])
    out, at = [], 0
    for h, d in widths:
        out.append(x[:, at:at + h * d].view(n, h, d))
        at += h * d
    return out


def _pages(batch, need, page, rng):
    """A pool with a few pages to spare, and every sequence's pages in it, in no order: [batch, pages of the longest]."""
    per = -(-need // page)
    pool = batch * per + 3
    return pool, torch.from_numpy(rng.permutation(pool)[:batch * per].reshape(batch, per).astype(np.int32)).cuda()


def _slots(table, seq, pos, page):
    """Where position pos of sequence seq lies in the pool."""
    return (table[seq, pos // page].long() * page + pos % page).int()


def _of_layers(slots, layers, positions):
    """The slots of every layer, whose parts of the pool follow each other; places outside the pool stay outside."""
    at = slots[None].long() + torch.arange(layers, device="cuda").view(-1, *[1] * slots.dim()) * positions
    return torch.where(slots[None] < 0, -1, at).int().flatten()


def _kv(s, pool, page, Hkv, hd, cache, layers=1):
    """The cache a program holds: the framework's, or plain arrays of the same values (and a place behind them that nobody reads)."""
    if own:
        import paper_2411_03786_amd as ngg
        s["kv"] = ngg.KVPages(pool, page, Hkv, hd, cache, layers=layers)
        return
    n = layers * pool * page
    kind = DTYPES.get(cache, torch.uint8)
    s["pk"], s["pv"] = (torch.zeros(n + page, Hkv, hd, dtype=kind, device="cuda") for _ in range(2))
    if cache not in DTYPES:                                             # (eight bits hold the values of four, too)
        s["pk"], s["pv"] = s["pk"].view(torch.float8_e4m3fn), s["pv"].view(torch.float8_e4m3fn)
        s["ek"], s["ev"] = (torch.ones(n + page, Hkv, 1 if cache == "fp8" else hd // GROUP, device="cuda") for _ in range(2))


def _arrays(s):
    return [s[n] for n in ("pk", "pv", "ek", "ev") if n in s]


def _bytes(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _lens(case, rng):
    """Cached tokens of every sequence: the given number, or spread below it."""
    c, b = case["context"], case["batch"]
    if not case["ragged"]:
        return np.full(b, c, dtype=np.int32)
    return np.concatenate([[c], rng.integers(max(1, c // 8), c + 1, b - 1)]).astype(np.int32)


def _parents(n, rng):
    """A tree of drafted tokens: a root and n - 1 nodes, each behind one of the latest few, so that paths of several tokens form."""
    return [-1] + [int(rng.integers(max(0, i - 1 - int(rng.integers(0, 12))), i)) for i in range(1, n)]


def _prepare_move(case, rng, seed):
    B, T, L, page, P = (case[x] for x in ("batch", "tree", "layers", "page", "context"))
    Hkv, hd = case["kv_heads"], case["head_dim"]
    s = dict(case=case)
    pool, table = _pages(B, P + T, page, rng)
    _kv(s, pool, page, Hkv, hd, case["cache"], L)
    seq, node = torch.arange(B, device="cuda").repeat_interleave(T), torch.arange(T, device="cuda").repeat(B)
    slots = _of_layers(_slots(table, seq, P + node, page), L, pool * page)
    _, k, v = _fused(L * B * T, [(Hkv, hd)] * 3, case["dtype"], _gen(seed, 5))
    _write(s, k, v, slots)
    # the root and some of the nodes behind it, fewer in most of the sequences
    path = np.full((B, case["path"]), -1, dtype=np.int64)
    for b in range(B):
        n = case["path"] if b == 0 else int(rng.integers(1, case["path"] + 1))
        path[b, :n] = np.concatenate([[0], 1 + np.sort(rng.permutation(T - 1)[:n - 1])])
    path = torch.from_numpy(path).cuda()
    rows, to = torch.arange(B, device="cuda")[:, None], torch.arange(case["path"], device="cuda")[None].expand(B, -1)
    s["src"] = torch.where(path < 0, -1, _slots(table, rows, P + path.clamp(min=0), page))
    s["dst"] = torch.where(path < 0, -1, _slots(table, rows, P + to, page))
    s["read"] = _of_layers(s["dst"].flatten(), L, pool * page)
    s["n"] = L * pool * page
    s["host"] = dict(path=path.flatten().tolist(), k=k, v=v)
    return s


def _prepare_pages(case, rng, seed):
    n, C, L, page, N, new = (case[x] for x in ("parents", "children", "layers", "page", "pool", "new"))
    Hkv, hd = case["kv_heads"], case["head_dim"]
    S, M = n * (1 + C), -(-(case["context"] + new) // page) + 1
    whole = case["context"] // page
    lens = (np.concatenate([[whole], rng.integers(whole // 4, whole + 1, n - 1)]) * page + case["context"] % page).astype(np.int32)
    held = -(-lens // page)
    order = rng.permutation(N)
    pages, refs = np.full((S, M), -1, dtype=np.int32), np.zeros(N, dtype=np.int32)
    at = 0
    for p in range(n):
        pages[p, :held[p]] = order[at:at + held[p]]
        at += held[p]
    refs[order[:at]] = 1
    s = dict(case=case, seqs=S, max_pages=M)
    all_lens = np.concatenate([lens, np.zeros(S - n, dtype=np.int32)])
    if own:
        import paper_2411_03786_amd as ngg
        s["table"] = ngg.PageTable(S, M, N, page)
        for to, x in ((s["table"].pages, pages), (s["table"].lens, all_lens), (s["table"].refs, refs)):
            to.copy_(torch.from_numpy(x))
    else:
        s["pages"], s["lens"], s["refs"] = (torch.from_numpy(x).cuda() for x in (pages, all_lens, refs))
    s["sources"] = torch.arange(n, dtype=torch.int32, device="cuda").repeat_interleave(C)
    s["targets"] = torch.arange(n, S, dtype=torch.int32, device="cuda")
    s["new"] = torch.from_numpy(np.concatenate([np.zeros(n), np.full(S - n, new)]).astype(np.int32)).cuda()
    _kv(s, N, page, Hkv, hd, case["cache"], L)
    # the last pages of the prompts, which their continuations go on writing to
    pos = [np.arange(int(x) // page * page, int(x)) for x in lens]
    mine = np.concatenate([pages[p, q // page].astype(np.int64) * page + q % page for p, q in enumerate(pos)])
    slots = _of_layers(torch.from_numpy(mine).cuda(), L, N * page)
    _, k, v = _fused(len(slots), [(Hkv, hd)] * 3, case["dtype"], _gen(seed, 6))
    _write(s, k, v, slots)
    # where the continuations find them: pages are given out from the lowest number on, sequence by sequence
    free, at, there = np.flatnonzero(refs == 0), 0, []
    for c in range(n, S):
        q = pos[(c - n) // C]
        there.append(free[at] * page + q % page)
        at += -(-(int(lens[(c - n) // C]) + new) // page) - int(lens[(c - n) // C]) // page
    s["read"] = _of_layers(torch.from_numpy(np.concatenate(there)).cuda(), L, N * page)
    s["host"] = dict(pages=pages, lens=all_lens, refs=refs, slots=slots, k=k, v=v)
    return s


def prepare(case, seed):
    rng = np.random.default_rng([seed % (1 << 30), 0x62])
    if case["op"] == "move":
        return _prepare_move(case, rng, seed)
    if case["op"] == "pages":
        return _prepare_pages(case, rng, seed)
    s = dict(case=case)
    page = case["page"]
    if case["op"] == "cache4":
        B, n, Hkv, hd, start = case["batch"], case["new"], case["kv_heads"], case["head_dim"], case["start"]
        pool, table = _pages(B, start + n, page, rng)
        _, s["k"], s["v"] = _fused(B * n, [(Hkv, hd)] * 3, case["dtype"], _gen(seed, 3))
        _kv(s, pool, page, Hkv, hd, "fp4")
        seq = torch.arange(B, device="cuda").repeat_interleave(n)
        s["slots"] = _slots(table, seq, start + torch.arange(n, device="cuda").repeat(B), page)
        r = case["read"]
        seq = torch.arange(B, device="cuda").repeat_interleave(r)
        s["read"] = _slots(table, seq, start + n - r + torch.arange(r, device="cuda").repeat(B), page)
        return s
    B, T, H, Hkv, hd = (case[x] for x in ("batch", "tree", "heads", "kv_heads", "head_dim"))
    lens = _lens(case, rng)
    trees = np.full(B, T) if not case["ragged"] else np.concatenate([[T], rng.integers(max(1, T // 2), T + 1, B - 1)])
    pool, table = _pages(B, int(lens.max()) + T, page, rng)
    gen = _gen(seed, 4)
    s["q"] = _fused(B * T, [(H, hd), (Hkv, hd), (Hkv, hd)], case["dtype"], gen)[0].view(B, T, H, hd) * 1.0
    s.update(table=table, lens=torch.from_numpy(lens).cuda(), trees=torch.from_numpy(trees.astype(np.int32)).cuda(), host_lens=lens, host_trees=trees)
    words = -(-T // 64)
    mask = np.zeros((B, T, words), dtype=np.uint64)
    for b in range(B):
        par = _parents(int(trees[b]), rng)
        for t, p in enumerate(par):
            if p >= 0:
                mask[b, t] = mask[b, p]
            mask[b, t, t // 64] |= np.uint64(1) << np.uint64(t % 64)
    s["mask"] = torch.from_numpy(mask.view(np.int64)).cuda() if T > 1 else None
    _kv(s, pool, page, Hkv, hd, "fp4")
    for b in range(B):                                                  # what the steps before have put there
        n = int(lens[b] + trees[b])
        _, k, v = _fused(n, [(Hkv, hd)] * 3, case["dtype"], gen)
        _write(s, k, v, _slots(table, torch.full((n,), b, device="cuda"), torch.arange(n, device="cuda"), page))
    return s


# ---- the operators in their plain form --------------------------------------------------------------------------------

def _power(top, most):
    """The smallest power of two that brings `top` to `most` (1.75 * 2^8 or 1.5 * 2^2) or below; 1 for zeros."""
    _, e = torch.frexp(top / most)                                      # top / most = m 2^e, m in [1/2, 1)
    e = torch.where(torch.ldexp(torch.full_like(top, most), e - 1) >= top, e - 1, e)
    return torch.where(top > 0, torch.ldexp(torch.ones_like(top), e), torch.ones_like(top))


def _eight_bits(x):
    f = x.float()
    scale = _power(f.abs().amax(-1, keepdim=True), 448.0)
    return (f / scale).to(torch.float8_e4m3fn), scale


def _four_bits(x):
    """Values of four bits, and the power of two of every 32 dimensions [.., head_dim / 32]."""
    f = x.float().unflatten(-1, (-1, GROUP))
    scale = _power(f.abs().amax(-1, keepdim=True), 6.0)
    y = f / scale
    size = y.abs()
    # steps of 0.5 below 2, of 1 below 4, of 2 above; round() takes ties to even
    step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0))
    return (torch.round(y / step) * step).flatten(-2).to(torch.float8_e4m3fn), scale.squeeze(-1)


def _write(s, k, v, slots):
    if own:
        s["kv"].write(k, v, slots)
        return
    at = slots.long()
    if "ek" in s:
        held = _eight_bits if s["ek"].shape[-1] == 1 and s["case"].get("cache") == "fp8" else _four_bits
        for x, vals, exps in ((k, "pk", "ek"), (v, "pv", "ev")):
            q, e = held(x)
            s[vals].view(torch.uint8)[at] = q.view(torch.uint8)
            s[exps][at] = e
    else:
        s["pk"][at] = k
        s["pv"][at] = v


def _read(s, slots, dtype=torch.float32):
    """Keys and values of slots, zeros where there is no such place."""
    at = slots.long()
    at = torch.where(at < 0, s["pk"].shape[0] - 1, at)                  # the place that nobody writes to
    out = []
    for vals, exps in (("pk", "ek"), ("pv", "ev")):
        x = _bytes(s[vals])[at].view(s[vals].dtype)
        if exps in s:
            e = s[exps][at]
            x = (x.float().unflatten(-1, (e.shape[-1], -1)) * e[..., None]).flatten(-2)
        out.append(x.to(dtype))
    return out


def _attend(s):
    q, table, lens, trees = s["q"], s["table"], s["lens"].long(), s["trees"].long()
    B, T, H, hd = q.shape
    Hkv = s["case"]["kv_heads"]
    G, page = H // Hkv, s["case"]["page"]
    n = int(s["host_lens"].max()) + T
    pos = torch.arange(n, device=q.device)
    slots = table[:, (pos // page).clamp(max=table.shape[1] - 1)].long() * page + pos % page
    k, v = _read(s, slots)
    k, v = k.permute(0, 2, 3, 1).reshape(B * Hkv, hd, n), v.permute(0, 2, 1, 3).reshape(B * Hkv, n, hd)
    x = q.float().view(B, T, Hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * T, hd)
    p = torch.bmm(x, k.contiguous()).mul_(1.0 / math.sqrt(hd)).view(B, Hkv, G, T, n)
    node = pos[None] - lens[:, None]                                    # the tree's node at a position; negative: the context
    at = node.clamp(0, T - 1)
    see = torch.ones(B, T, n, dtype=torch.bool, device=q.device)
    if s["mask"] is not None:
        nodes = torch.arange(T, device=q.device)
        bits = ((s["mask"][:, :, nodes // 64] >> (nodes % 64)) & 1).bool()
        see = torch.gather(bits, 2, at[:, None].expand(B, T, n))
    see = (node < 0)[:, None] | (see & ((node >= 0) & (node < trees[:, None]))[:, None] & (at[:, None] <= torch.arange(T, device=q.device)[:, None]))
    see = see & (torch.arange(T, device=q.device) < trees[:, None])[..., None]
    p.masked_fill_(~see[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    tot = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(B * Hkv, G * T, n), v.contiguous()).view(B, Hkv, G, T, hd) / torch.where(tot == 0, 1.0, tot)
    lse = (top + tot.log()).squeeze(-1)
    return dict(out=o.permute(0, 3, 1, 2, 4).reshape(B, T, H, hd).to(q.dtype), lse=lse.permute(0, 3, 1, 2).reshape(B, T, H).contiguous())


def _move(s):
    """All places are read before the first is written; -1: none."""
    L, n = s["case"]["layers"], s["n"]
    at = torch.arange(L, device="cuda")[:, None] * (n // L)
    src, dst = s["src"].flatten().long(), s["dst"].flatten().long()
    frm, to = (torch.where((src < 0) | (dst < 0), n, x + at) for x in (src, dst))
    for t in _arrays(s):
        _bytes(t)[to] = _bytes(t)[frm]


def _count(refs, pages, by):
    """Counts the references of pages [..] up or down; -1: none."""
    there = pages >= 0
    refs.index_add_(0, pages.clamp(min=0).flatten().long(), (there.int() * by).flatten())


def _fork(s):
    pages, lens, refs, page = s["pages"], s["lens"], s["refs"], s["case"]["page"]
    src, to = s["sources"].long(), s["targets"].long()
    _count(refs, pages[to], -1)
    held = (lens[src] + page - 1) // page
    rows = torch.where(torch.arange(s["max_pages"], device="cuda") < held[:, None], pages[src], -1)
    pages[to] = rows
    lens[to] = lens[src]
    _count(refs, rows, 1)


def _reserve(s):
    """Pages for the new tokens behind the cached ones, a sequence's own: the lowest free ones, by sequence and place."""
    pages, lens, refs, page = s["pages"], s["lens"].long(), s["refs"], s["case"]["page"]
    S, M, N = s["seqs"], s["max_pages"], refs.shape[0]
    new = s["new"].long()
    j = torch.arange(M, device="cuda")
    first, end = lens // page, (lens + new + page - 1) // page
    wanted = (j >= first[:, None]) & (j < end[:, None]) & (new > 0)[:, None]
    shared = (pages >= 0) & (refs[pages.clamp(min=0).long()] > 1)
    # of the sequences that go on in a page that nobody else holds, the last keeps it
    part = (lens % page > 0) & (new > 0)
    here = torch.gather(pages, 1, first.clamp(max=M - 1)[:, None]).squeeze(1).long()
    here = torch.where(part & (here >= 0), here, N)
    users = torch.zeros(N + 1, dtype=torch.int32, device="cuda").index_add_(0, here, torch.ones_like(here, dtype=torch.int32))
    seqs = torch.arange(S, device="cuda")
    last = torch.zeros(N + 1, dtype=torch.long, device="cuda").scatter_reduce_(0, here, seqs, "amax")
    keeps = (here < N) & (users[here] == refs[here.clamp(max=N - 1)]) & (last[here] == seqs)
    need = wanted & ((pages < 0) | (shared & ~(keeps[:, None] & (j == first[:, None]))))
    free = torch.argsort((refs != 0).int(), stable=True)                # free pages first, by number
    rank = need.flatten().cumsum(0) - 1
    missing = (rank[-1] + 1 - (refs == 0).sum()).clamp(min=0)
    need = need & (missing == 0)
    got = free[rank.clamp(0, N - 1)].view(S, M).int()
    moved = (torch.gather(need, 1, first.clamp(max=M - 1)[:, None]).squeeze(1)) & part & (here < N)
    pick = lambda t: torch.where(moved, torch.gather(t, 1, first.clamp(max=M - 1)[:, None]).squeeze(1), -1)
    src, dst = pick(pages), pick(got)
    _count(refs, torch.where(need, pages, -1), -1)
    _count(refs, torch.where(need, got, -1), 1)
    pages.copy_(torch.where(need, got, pages))
    return dict(src=src, dst=dst, positions=torch.where(moved, (lens % page).int(), 0).int(), missing=missing.int().view(1))


def _copy(s, src, dst):
    L, N, page = s["case"]["layers"], s["refs"].shape[0], s["case"]["page"]
    at = torch.arange(L, device="cuda")[:, None] * N
    frm, to = (torch.where(src < 0, L * N, x.long() + at) for x in (src, dst))
    for t in _arrays(s):
        x = _bytes(t).view(L * N + 1, page, *t.shape[1:])
        x[to] = x[frm]


def run(s):
    case = s["case"]
    op, dtype = case["op"], DTYPES[case["dtype"]]
    if op == "cache4":
        _write(s, s["k"], s["v"], s["slots"])
        k, v = s["kv"].read(s["read"], dtype) if own else _read(s, s["read"], dtype)
        return dict(k=k, v=v)
    if op == "attend4":
        if own:
            import paper_2411_03786_amd as ngg
            out, lse = ngg.tree_attention(s["q"], s["kv"], s["table"], s["lens"], mask=s["mask"], tree_lens=s["trees"], want_lse=True)
            return dict(out=out, lse=lse)
        return _attend(s)
    if op == "move":
        if own:
            s["kv"].move(s["src"], s["dst"])
            k, v = s["kv"].read(s["read"], dtype)
        else:
            _move(s)
            k, v = _read(s, s["read"], dtype)
        return dict(k=k, v=v)
    if own:
        table = s["table"]
        table.fork(s["sources"], s["targets"])
        r = table.reserve(s["new"])
        s["kv"].copy(r.src, r.dst, r.positions)
        k, v = s["kv"].read(s["read"], dtype)
        return dict(pages=table.pages, lens=table.lens, refs=table.refs, src=r.src, dst=r.dst, positions=r.positions, missing=r.missing, k=k, v=v)
    _fork(s)
    r = _reserve(s)
    _copy(s, r["src"], r["dst"])
    k, v = _read(s, s["read"], dtype)
    return dict(pages=s["pages"], lens=s["lens"], refs=s["refs"], k=k, v=v, **r)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def _held(cache, hd):
    """Bytes of a cached key (or value) of one head."""
    return {"f32": 4.0 * hd, "bf16": 2.0 * hd, "fp8": hd + 1.0, "fp4": hd / 2 + hd / GROUP}[cache]


def work(case):
    e = {"f32": 4, "bf16": 2}[case["dtype"]]
    hd, Hkv = case["head_dim"], case["kv_heads"]
    if case["op"] == "cache4":
        w, r = case["batch"] * case["new"], case["batch"] * case["read"]
        return dict(bytes=2.0 * (w + r) * Hkv * (hd * e + _held("fp4", hd)) + 4.0 * (w + r), flops=2.0 * (w + r) * Hkv * hd)
    if case["op"] == "move":
        rows = case["layers"] * (case["path"] + (case["batch"] - 1) * (case["path"] + 1) / 2) * Hkv * 2
        return dict(bytes=rows * (3 * _held(case["cache"], hd) + hd * e), flops=0.0)
    if case["op"] == "pages":
        S, n = case["parents"] * (1 + case["children"]), case["parents"] * case["children"]
        rows = case["layers"] * (case["context"] % case["page"]) * Hkv * 2
        entries = n * (case["context"] * (1.0 if case["parents"] == 1 else 0.66) + case["new"]) / case["page"]
        return dict(bytes=rows * _held(case["cache"], hd) * (case["parents"] + 2 * n) + rows * n * hd * e + 4.0 * (3 * entries + case["pool"] + 6 * S),
                    flops=0.0)
    B, T, H = case["batch"], case["tree"], case["heads"]
    ctx = B * case["context"] if not case["ragged"] else case["context"] * (1 + (B - 1) * 0.5625)
    trees = B * T if not case["ragged"] else T * (1 + (B - 1) * 0.75)
    pairs = ctx / B * trees + trees * (T + 1) / 2
    return dict(bytes=2.0 * (ctx + trees) * Hkv * _held("fp4", hd) + 2.0 * trees * H * hd * e + 4.0 * trees * H, flops=4.0 * pairs * H * hd)


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _four64(x):
    """x in four bits, as values: of every 32 the power of two, then the nearest of the eight magnitudes by their borders (a border
    itself goes to the even one of its two codes)."""
    x = x.double().unflatten(-1, (-1, GROUP))
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 6.0)))
    scale = torch.where(6.0 * scale < top, 2.0 * scale, scale)          # (the logarithm is rounded)
    scale = torch.where(3.0 * scale >= top, 0.5 * scale, scale)
    scale = torch.where(top > 0, scale, 1.0)
    y, val = x.abs() / scale, torch.zeros_like(x)
    for code in range(1, 8):
        border = (GRID[code - 1] + GRID[code]) / 2
        val = torch.where((y >= border) if code % 2 == 0 else (y > border), GRID[code], val)
    return (torch.sign(x) * val * scale).flatten(-2)


def _eight64(x):
    """x in eight bits: four bits of which the first is 1 (or less of them below 2^-6), times the head's power of two."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)))
    scale = torch.where(448.0 * scale < top, 2.0 * scale, scale)
    scale = torch.where(224.0 * scale >= top, 0.5 * scale, scale)
    scale = torch.where(top > 0, scale, 1.0)
    y = x / scale
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(y / unit) * unit * scale


_HELD64 = {"f32": lambda x: x.double(), "bf16": lambda x: x.double(), "fp8": _eight64, "fp4": _four64}


def _plain_inputs(case, seed):
    """prepare's inputs, with the cache as plain arrays whatever the side."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _exact_pages(case, s):
    """Sequence by sequence, page by page."""
    h, page, n, C, new = s["host"], case["page"], case["parents"], case["children"], case["new"]
    pages, lens, refs = h["pages"].copy(), h["lens"].copy(), h["refs"].copy()
    for c in range(n, len(lens)):
        p = (c - n) // C
        lens[c] = lens[p]
        for j in range(-(-int(lens[p]) // page)):
            pages[c, j] = pages[p, j]
            refs[pages[p, j]] += 1
    src, dst, count = (np.full(len(lens), x, dtype=np.int32) for x in (-1, -1, 0))
    free = iter(np.flatnonzero(refs == 0).tolist())
    for c in range(n, len(lens)):
        for j in range(int(lens[c]) // page, -(-(int(lens[c]) + new) // page)):
            to = next(free)
            if pages[c, j] >= 0:                                        # the prompt's last page, which the prompt keeps
                src[c], dst[c], count[c] = pages[c, j], to, lens[c] % page
                refs[pages[c, j]] -= 1
            pages[c, j], refs[to] = to, 1
    held = _HELD64[case["cache"]]
    out = dict(pages=pages, lens=lens, refs=refs, src=src, dst=dst, positions=count, missing=np.zeros(1, np.int32))
    # every continuation has the prompt's last positions
    r = case["context"] % page
    rows = [(i * n + p) * r + q for i in range(case["layers"]) for p in range(n) for _ in range(C) for q in range(r)]
    rows = torch.tensor(rows, device="cuda")
    return dict(out, k=held(h["k"])[rows], v=held(h["v"])[rows])


def exact(case, seed):
    s = _plain_inputs(case, seed)
    if case["op"] == "cache4":
        B, n, r = case["batch"], case["new"], case["read"]
        out = []
        for x in (_four64(s["k"]), _four64(s["v"])):                    # positions before the new ones hold nothing yet
            x = torch.cat([torch.zeros(B, max(0, r - n), *x.shape[1:], dtype=torch.float64, device="cuda"), x.view(B, n, *x.shape[1:])[:, max(0, n - r):]], 1)
            out.append(x.flatten(0, 1))
        return dict(k=out[0], v=out[1])
    if case["op"] == "pages":
        return _exact_pages(case, s)
    if case["op"] == "move":                                            # behind the context lie the tokens of the path
        h, held = s["host"], _HELD64[case["cache"]]
        L, B, T, n = case["layers"], case["batch"], case["tree"], case["path"]
        rows = [(i * B + b) * T + node if node >= 0 else L * B * T for i in range(L) for b in range(B) for node in h["path"][b * n:(b + 1) * n]]
        return {a: torch.cat([held(h[a]), torch.zeros_like(h[a][:1], dtype=torch.float64)])[rows] for a in "kv"}
    q, mask, page = s["q"], s["mask"], case["page"]
    B, T, H, hd = q.shape
    G = H // case["kv_heads"]
    out = torch.zeros(B, T, H, hd, dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, H), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        P, n = int(s["host_lens"][b]), int(s["host_trees"][b])
        slots = _slots(s["table"], torch.full((P + n,), b, device="cuda"), torch.arange(P + n, device="cuda"), page).long()
        keys, vals = ((s[a].view(torch.uint8)[slots].view(torch.float8_e4m3fn).double() * s[e][slots].double().repeat_interleave(GROUP, -1))
                      for a, e in (("pk", "ek"), ("pv", "ev")))
        see = torch.ones(n, P + n, dtype=torch.bool, device="cuda")
        if mask is not None:
            for j in range(n):
                see[:, P + j] = (mask[b, :n, j // 64] >> (j % 64)) & 1 == 1
        for h in range(H):
            score = q[b, :n, h].double() @ keys[:, h // G].T.contiguous() / hd ** 0.5
            score = torch.where(see, score, torch.full_like(score, -math.inf))
            lse[b, :n, h] = torch.logsumexp(score, -1)
            out[b, :n, h] = torch.softmax(score, -1) @ vals[:, h // G]
    return dict(out=out, lse=lse)
