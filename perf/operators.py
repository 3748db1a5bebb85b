"""Operator cases: the calls around a batched tree verification, over the sizes this framework is used at.

Four operators that a serving program chains in every layer and step of a speculative decoder whose drafts form a tree:

* ``rotary``    rotary positions on queries and keys (half or interleaved pairs, all or part of the head, scaled tables),
* ``cache``     keys and values written into a paged cache, as they are or in 8 bits, and read back,
* ``attend``    attention of every sequence's tree of drafted tokens (or of its single new token) over its cached positions,
* ``logprobs``  log probabilities of given tokens under rows of logits, with the entropy and the likeliest alternatives.

A case is a dict of plain values.  ``run`` with ``own`` false is the mathematics in elementary torch operations in 32 bits;
with ``own`` true it makes the framework's calls.  Queries, keys and values are the slices of one fused projection's output,
as a program has them, so their rows are strided.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

# heads, key/value heads, head_dim: the attention shapes of the benchmark's workloads, all heads their own and four to a key head
HEADS = ((4, 4, 32), (8, 8, 64), (12, 12, 64), (12, 3, 64), (32, 32, 128), (32, 8, 128), (24, 24, 128), (24, 6, 128))
VOCABS = (512, 8192, 32000, 128256)
THETA = 10000.0
PAGE = 64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one verify block of the 7B shape (51 tokens, 32 heads): a small launch in every layer
        dict(op="rotary", name="rotary_block", tokens=51, heads=32, kv_heads=32, head_dim=128, rotary_dim=128, dtype="bf16",
             interleaved=False, scaling="none", start=2047),
        # a long prompt's piece with four query heads to a key head, half of the head rotated, interleaved, a table scaled by bands
        dict(op="rotary", name="rotary_prompt_part", tokens=16384, heads=32, kv_heads=8, head_dim=128, rotary_dim=64, dtype="bf16",
             interleaved=True, scaling="bands", start=4096),
        # one new token of each of 32 sequences, rotated and written as it is: the latency of a decode step
        dict(op="cache", name="cache_append_rotated", batch=32, new=1, kv_heads=8, head_dim=128, dtype="bf16", cache="bf16", rotated=True,
             start=2047, read=1),
        # the trees of 16 sequences (61 tokens each) into an 8-bit cache, read back
        dict(op="cache", name="cache_trees_fp8", batch=16, new=61, kv_heads=8, head_dim=128, dtype="bf16", cache="fp8", rotated=False,
             start=1000, read=61),
        # a 16K prompt into the 8-bit cache, and all of it read back
        dict(op="cache", name="cache_prompt_fp8", batch=1, new=16384, kv_heads=8, head_dim=128, dtype="bf16", cache="fp8", rotated=False,
             start=0, read=16384),
        # the smallest model's tree of 13 tokens over 128 cached ones, fp32: launches and latency
        dict(op="attend", name="attend_tiny_f32", batch=1, tree=13, heads=4, kv_heads=4, head_dim=32, dtype="f32", cache="f32",
             context=128, ragged=False),
        # the headline block: one sequence, 51 tokens, 32 heads of their own, 2K context
        dict(op="attend", name="attend_tree_7b", batch=1, tree=51, heads=32, kv_heads=32, head_dim=128, dtype="bf16", cache="bf16",
             context=2047, ragged=False),
        # plain decoding of 32 sequences of up to 8K tokens, four query heads to a key head
        dict(op="attend", name="attend_decode_batch", batch=32, tree=1, heads=32, kv_heads=8, head_dim=128, dtype="bf16", cache="bf16",
             context=8191, ragged=True),
        # trees of up to 61 tokens of eight sequences of up to 32K tokens in the 8-bit cache
        dict(op="attend", name="attend_trees_32k_fp8", batch=8, tree=61, heads=32, kv_heads=8, head_dim=128, dtype="bf16", cache="fp8",
             context=32000, ragged=True),
        # the rows of one verify block over 32000 tokens, the drafted token of every row and five alternatives
        dict(op="logprobs", name="logprobs_block", rows=51, vocab=32000, dtype="f32", targets=1, top=5, scale=1.0),
        # the rows of a tree over the large vocabulary: the tokens of up to four children and twenty alternatives, at a temperature
        dict(op="logprobs", name="logprobs_tree_128k", rows=97, vocab=128256, dtype="f32", targets=4, top=20, scale=1.25),
        # a prompt scored piece by piece: 4096 rows of 16-bit logits over the large vocabulary
        dict(op="logprobs", name="logprobs_prompt_128k", rows=4096, vocab=128256, dtype="bf16", targets=1, top=8, scale=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(("rotary", "cache", "cache", "attend", "attend", "attend", "attend", "logprobs", "logprobs"))
    heads, kv_heads, hd = rng.choice(HEADS)
    dtype = rng.choice(("f32", "bf16", "bf16"))
    if op == "rotary":
        return dict(op=op, tokens=min(_log(rng, 1, 16384), (1 << 26) // ((heads + kv_heads) * hd)), heads=heads, kv_heads=kv_heads, head_dim=hd,
                    rotary_dim=rng.choice((hd, hd, hd // 2, hd // 4 + 2)), dtype=dtype, interleaved=rng.random() < 0.5,
                    scaling=rng.choice(("none", "linear", "bands")), start=_log(rng, 1, 100000))
    cache = rng.choice((dtype, "fp8"))
    if op == "cache":
        batch = _log(rng, 1, 48)
        new = _log(rng, 1, max(2, 16384 // batch))
        start = _log(rng, 1, 4096)
        # the eight bits of a rotated key hang on its last bit, so rotation goes with the wider caches
        return dict(op=op, batch=batch, new=new, kv_heads=kv_heads, head_dim=hd, dtype=dtype, cache=cache, rotated=cache != "fp8" and rng.random() < 0.5,
                    start=start, read=min(new + start, max(1, min(_log(rng, 1, 4 * new), 16384 // batch))))
    if op == "attend":
        while True:
            c = dict(op=op, batch=_log(rng, 1, 48), tree=1 if rng.random() < 0.25 else _log(rng, 2, 128), heads=heads, kv_heads=kv_heads,
                     head_dim=hd, dtype=dtype, cache=cache, context=_log(rng, 1, 65536), ragged=rng.random() < 0.6)
            w = work(c)
            if w["flops"] < 1.5e11 and w["bytes"] < 6e8 and c["batch"] * c["context"] * kv_heads * hd < 3e8:
                return c
    vocab = rng.choice((rng.choice(VOCABS), _log(rng, 300, 130000)))
    rows = max(1, min(_log(rng, 1, 4096), (1 << 28) // vocab))
    return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, targets=rng.randint(0, 4), top=rng.choice((0, 1, 5, rng.randint(2, 32))),
                scale=rng.choice((1.0, 1.0, 0.7, 1.5)))


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed % (1 << 30)) + salt)
    return g


def _scaling(kind):
    """What stretches a table over more positions than it was made for."""
    return {"none": None, "linear": dict(kind="linear", factor=4.0),
            "bands": dict(kind="bands", factor=8.0, low=1.0, high=4.0, original=8192)}[kind]


def _frequencies(rd, scaling):
    """Angle per position of every pair, in 64 bits."""
    inv = THETA ** (-np.arange(rd // 2, dtype=np.float64) * 2.0 / rd)
    if scaling is None:
        return inv
    if scaling["kind"] == "linear":
        return inv / scaling["factor"]
    turns = scaling["original"] * inv / (2.0 * math.pi)                 # turns of the pair over the original length
    keep = np.clip((turns - scaling["low"]) / (scaling["high"] - scaling["low"]), 0.0, 1.0)
    return inv * keep + inv / scaling["factor"] * (1.0 - keep)


def _tables(rd, n, scaling):
    ang = np.arange(n, dtype=np.float64)[:, None] * _frequencies(rd, scaling)[None]
    return torch.from_numpy(np.cos(ang).astype(np.float32)).cuda(), torch.from_numpy(np.sin(ang).astype(np.float32)).cuda()


def _rope(s, rd, n, interleaved, kind):
    """The table a program makes once per model."""
    if own:
        import paper_2411_03786_amd as ngg
        s["rope"] = ngg.Rope(rd, n, theta=THETA, interleaved=interleaved, scaling=_scaling(kind))
    else:
        s["cos"], s["sin"] = _tables(rd, n, _scaling(kind))


def _fused(n, widths, dtype, gen):
    """Slices of one projection's output [n, sum of heads * head_dim], as [n, heads, head_dim] views.  A few features are larger than
    the others, as those of trained models are."""
    hd = widths[0][1]
    cols = sum(h * d for h, d in widths)
    x = torch.randn(n, cols, generator=gen, device="cuda")
    x *= torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.02, 4.0, 1.0)
    x = x.to(DTYPES[dtype])
    out, at = [], 0
    for h, d in widths:
        out.append(x[:, at:at + h * d].view(n, h, d))
        at += h * d
    assert hd == widths[-1][1]
    return out


def _pages(batch, need, rng):
    """A pool with a few pages to spare, and every sequence's pages in it, in no order: [batch, pages of the longest]."""
    per = -(-need // PAGE)
    pool = batch * per + 3
    return pool, torch.from_numpy(rng.permutation(pool)[:batch * per].reshape(batch, per).astype(np.int32)).cuda()


def _slots(table, seq, pos):
    """Where position pos of sequence seq lies in the pool."""
    return (table[seq, pos // PAGE].long() * PAGE + pos % PAGE).int()


def _kv(s, pool, Hkv, hd, dtype, cache):
    """The cache a program holds: the framework's, or plain arrays of the same values."""
    if own:
        import paper_2411_03786_amd as ngg
        s["kv"] = ngg.KVPages(pool, PAGE, Hkv, hd, cache)
        return
    kind = torch.float8_e4m3fn if cache == "fp8" else DTYPES[cache]
    s["pk"], s["pv"] = (torch.zeros(pool * PAGE, Hkv, hd, device="cuda").to(kind) for _ in range(2))
    if cache == "fp8":
        s["ek"], s["ev"] = (torch.ones(pool * PAGE, Hkv, 1, device="cuda") for _ in range(2))


def _lens(case, rng):
    """Cached tokens of every sequence: the given number, or spread below it."""
    c, b = case["context"], case["batch"]
    if not case["ragged"]:
        return np.full(b, c, dtype=np.int32)
    return np.concatenate([[c], rng.integers(max(1, c // 8), c + 1, b - 1)]).astype(np.int32)


def _parents(n, rng):
    """A tree of drafted tokens: a root and n - 1 nodes, each behind one of the latest few, so that paths of several tokens form."""
    return [-1] + [int(rng.integers(max(0, i - 1 - int(rng.integers(0, 12))), i)) for i in range(1, n)]


def prepare(case, seed):
    rng = np.random.default_rng([seed % (1 << 30), 0x61])
    s = dict(case=case)
    if case["op"] == "rotary":
        n, rd = case["tokens"], case["rotary_dim"]
        s["q"], s["k"], _ = _fused(n, [(case["heads"], case["head_dim"])] + [(case["kv_heads"], case["head_dim"])] * 2, case["dtype"], _gen(seed, 1))
        s["pos"] = case["start"] + torch.arange(n, dtype=torch.int32, device="cuda")
        if n <= 128:                                                    # a block of drafted tokens: few positions, each many times
            s["pos"] = case["start"] + torch.from_numpy(rng.integers(0, 8, n).astype(np.int32)).cuda()
        _rope(s, rd, case["start"] + max(n, 8), case["interleaved"], case["scaling"])
        return s
    if case["op"] == "logprobs":
        n, V, gen = case["rows"], case["vocab"], _gen(seed, 2)
        x = torch.randn(n, V, generator=gen, device="cuda").mul_(2.0)
        # a trained model's rows: a handful of tokens stand out by as much as ten, the end of the vocabulary is padding that is ruled out
        hot = torch.randint(0, V, (n, 24), generator=gen, device="cuda")
        x.scatter_add_(1, hot, torch.rand(n, 24, generator=gen, device="cuda").mul_(10.0))
        pad = V // 500
        if pad:
            x[:, V - pad:] = -math.inf
        s["logits"] = x.to(DTYPES[case["dtype"]])
        s["targets"] = None
        if case["targets"]:
            t = torch.randint(0, V - pad, (n, case["targets"]), generator=gen, device="cuda", dtype=torch.int32)
            t[:, 0] = hot[:, 0].clamp(max=V - pad - 1)
            s["targets"] = t
        return s
    if case["op"] == "cache":
        B, n, Hkv, hd, start = case["batch"], case["new"], case["kv_heads"], case["head_dim"], case["start"]
        pool, table = _pages(B, start + n, rng)
        _, s["k"], s["v"] = _fused(B * n, [(Hkv, hd)] * 3, case["dtype"], _gen(seed, 3))
        _kv(s, pool, Hkv, hd, case["dtype"], case["cache"])
        seq = torch.arange(B, device="cuda").repeat_interleave(n)
        pos = start + torch.arange(n, device="cuda").repeat(B)
        s["slots"], s["pos"] = _slots(table, seq, pos), pos.int()
        r = case["read"]
        seq = torch.arange(B, device="cuda").repeat_interleave(r)
        s["read"] = _slots(table, seq, start + n - r + torch.arange(r, device="cuda").repeat(B))
        if case["rotated"]:
            _rope(s, hd, start + n, False, "none")
        return s
    B, T, H, Hkv, hd = (case[x] for x in ("batch", "tree", "heads", "kv_heads", "head_dim"))
    lens = _lens(case, rng)
    trees = np.full(B, T) if not case["ragged"] else np.concatenate([[T], rng.integers(max(1, T // 2), T + 1, B - 1)])
    pool, table = _pages(B, int(lens.max()) + T, rng)
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
    _kv(s, pool, Hkv, hd, case["dtype"], case["cache"])
    for b in range(B):                                                  # what the steps before have put there
        n = int(lens[b] + trees[b])
        _, k, v = _fused(n, [(Hkv, hd)] * 3, case["dtype"], gen)
        _write(s, k, v, _slots(table, torch.full((n,), b, device="cuda"), torch.arange(n, device="cuda")))
    return s


# ---- the operators in their plain form --------------------------------------------------------------------------------

def _rotate(x, cos, sin, interleaved):
    """x [n, heads, head_dim], cos and sin [n, rotary_dim / 2]: pairs of the first rotary_dim elements turn, the others stay."""
    half = cos.shape[1]
    f = x.float()
    c, sn = cos[:, None], sin[:, None]
    a, b = (f[..., 0:2 * half:2], f[..., 1:2 * half:2]) if interleaved else (f[..., :half], f[..., half:2 * half])
    u, w = a * c - b * sn, b * c + a * sn
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, f[..., 2 * half:]], -1).to(x.dtype)


def _eight_bits(x):
    """Values of eight bits and the power of two they share in a head: the smallest that brings all of them to 448 or below."""
    f = x.float()
    top = f.abs().amax(-1, keepdim=True)
    _, e = torch.frexp(top / 448.0)                                     # top / 448 = m 2^e, m in [1/2, 1)
    e = torch.where(torch.ldexp(torch.full_like(top, 448.0), e - 1) >= top, e - 1, e)
    scale = torch.where(top > 0, torch.ldexp(torch.ones_like(top), e), torch.ones_like(top))
    return (f / scale).to(torch.float8_e4m3fn), scale


def _write(s, k, v, slots):
    if own:
        s["kv"].write(k, v, slots)
        return
    at = slots.long()
    if "ek" in s:
        for x, vals, exps in ((k, "pk", "ek"), (v, "pv", "ev")):
            q, e = _eight_bits(x)
            s[vals].view(torch.uint8)[at] = q.view(torch.uint8)
            s[exps][at] = e
    else:
        s["pk"][at] = k
        s["pv"][at] = v


def _read(s, slots, dtype=torch.float32):
    at = slots.long()
    if "ek" in s:
        return ((s["pk"].view(torch.uint8)[at].view(torch.float8_e4m3fn).float() * s["ek"][at]).to(dtype),
                (s["pv"].view(torch.uint8)[at].view(torch.float8_e4m3fn).float() * s["ev"][at]).to(dtype))
    return s["pk"][at].to(dtype), s["pv"][at].to(dtype)


def _attend(s):
    q, table, lens, trees = s["q"], s["table"], s["host_lens"], s["host_trees"]
    B, T, H, hd = q.shape
    Hkv = s["case"]["kv_heads"]
    G = H // Hkv
    out = torch.zeros_like(q)
    lse = torch.full((B, T, H), -math.inf, device=q.device)
    for b in range(B):
        P, n = int(lens[b]), int(trees[b])
        k, v = _read(s, _slots(table, torch.full((P + n,), b, device=q.device), torch.arange(P + n, device=q.device)))
        k, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
        x = q[b, :n].float().view(n, Hkv, G, hd).permute(1, 2, 0, 3).reshape(Hkv, G * n, hd)
        p = torch.bmm(x, k).mul_(1.0 / math.sqrt(hd)).view(Hkv, G, n, P + n)
        if s["mask"] is not None:
            at = torch.arange(n, device=q.device)
            see = (s["mask"][b, :n][:, at // 64] >> (at % 64)) & 1
            p[..., P:].masked_fill_(see == 0, -math.inf)
        top = p.amax(-1, keepdim=True)
        p = p.sub_(top).exp_()
        tot = p.sum(-1, keepdim=True)
        o = torch.bmm(p.view(Hkv, G * n, P + n), v).view(Hkv, G, n, hd) / tot
        out[b, :n] = o.permute(2, 0, 1, 3).reshape(n, H, hd).to(q.dtype)
        lse[b, :n] = (top + tot.log()).squeeze(-1).permute(2, 0, 1).reshape(n, H)
    return dict(out=out, lse=lse)


def _score(x, targets, top, scale):
    x = x.float() * scale
    best = x.amax(-1, keepdim=True)
    e = (x - best).exp()
    tot = e.sum(-1, keepdim=True)
    mean = torch.where(e > 0, e * (x - best), torch.zeros_like(e)).sum(-1, keepdim=True) / tot
    lse = best + tot.log()
    out = dict(entropy=(tot.log() - mean).squeeze(-1), lse=lse.squeeze(-1))
    if targets is not None:
        out["logprobs"] = x.gather(1, targets.long()) - lse
    if top:
        val, ids = torch.sort(x, dim=-1, descending=True, stable=True)
        out["top_ids"], out["top_logprobs"] = ids[:, :top].int(), val[:, :top] - lse
    return out


def run(s):
    case = s["case"]
    op = case["op"]
    if op == "rotary":
        if own:
            import paper_2411_03786_amd as ngg
            q, k = ngg.rotary(s["rope"], s["pos"], s["q"], s["k"])
        else:
            c, sn = s["cos"][s["pos"].long()], s["sin"][s["pos"].long()]
            q, k = _rotate(s["q"], c, sn, case["interleaved"]), _rotate(s["k"], c, sn, case["interleaved"])
        return dict(q=q, k=k)
    if op == "cache":
        if own:
            s["kv"].write(s["k"], s["v"], s["slots"], **(dict(rope=s["rope"], positions=s["pos"]) if case["rotated"] else {}))
            k, v = s["kv"].read(s["read"], s["k"].dtype)
        else:
            k = s["k"]
            if case["rotated"]:
                k = _rotate(k, s["cos"][s["pos"].long()], s["sin"][s["pos"].long()], False)
            _write(s, k, s["v"], s["slots"])
            k, v = _read(s, s["read"], s["k"].dtype)
        return dict(k=k, v=v)
    if op == "attend":
        if own:
            import paper_2411_03786_amd as ngg
            out, lse = ngg.tree_attention(s["q"], s["kv"], s["table"], s["lens"], mask=s["mask"], tree_lens=s["trees"], want_lse=True)
            return dict(out=out, lse=lse)
        return _attend(s)
    if own:
        import paper_2411_03786_amd as ngg
        r = ngg.token_logprobs(s["logits"], s["targets"], top_n=case["top"], scale=case["scale"])
        out = dict(entropy=r.entropy, lse=r.lse)
        if case["targets"]:
            out["logprobs"] = r.logprobs
        if case["top"]:
            out["top_ids"], out["top_logprobs"] = r.top_ids, r.top_logprobs
        return out
    return _score(s["logits"], s["targets"], case["top"], case["scale"])


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    e = {"f32": 4, "bf16": 2}[case["dtype"]]
    if case["op"] == "rotary":
        n, rd = case["tokens"], case["rotary_dim"]
        elems = n * (case["heads"] + case["kv_heads"])
        rows = 8 if n <= 128 else n
        return dict(bytes=float(2 * elems * case["head_dim"] * e + rows * rd * 4 + 4 * n), flops=3.0 * elems * rd)
    if case["op"] == "logprobs":
        n, V = case["rows"], case["vocab"]
        return dict(bytes=float(n * V * e + n * (8 + 8 * case["targets"] + 8 * case["top"])), flops=5.0 * n * V)
    c = {"f32": 4, "bf16": 2, "fp8": 1}[case["cache"]]
    extra = 1 if case["cache"] == "fp8" else 0                          # the shared power of two of a head
    hd, Hkv = case["head_dim"], case["kv_heads"]
    if case["op"] == "cache":
        w, r = case["batch"] * case["new"], case["batch"] * case["read"]
        rope = case["new"] * hd * 4 if case["rotated"] else 0
        return dict(bytes=float(2 * (w + r) * Hkv * (hd * (e + c) + extra) + 4 * (w + r) + rope), flops=2.0 * (w + r) * Hkv * hd)
    B, T, H = case["batch"], case["tree"], case["heads"]
    ctx = B * case["context"] if not case["ragged"] else case["context"] * (1 + (B - 1) * 0.5625)
    trees = B * T if not case["ragged"] else T * (1 + (B - 1) * 0.75)
    keys = ctx + trees
    pairs = ctx / B * trees + trees * (T + 1) / 2
    return dict(bytes=2.0 * keys * Hkv * (hd * c + extra) + 2.0 * trees * H * hd * e + 4.0 * trees * H, flops=4.0 * pairs * H * hd)


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------

def _turn64(x, pos, freq, interleaved):
    """Pairs as complex numbers times e^{i angle}."""
    rd = 2 * len(freq)
    ang = pos.double()[:, None] * torch.from_numpy(freq).cuda()[None]
    z = x[..., :rd].double()
    z = z.unflatten(-1, (rd // 2, 2)) if interleaved else z.unflatten(-1, (2, rd // 2)).transpose(-1, -2)
    z = torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(ang), ang)[:, None]
    z = torch.view_as_real(z)
    z = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., rd:].double()], -1)


def _eight64(x):
    """x in eight bits, as values: a sign, four bits of which the first is 1 (or less of them below 2^-6), times the head's power of two."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))), torch.ones_like(top))
    scale = torch.where(scale * 448.0 < top, scale * 2.0, scale)
    scale = torch.where((top > 0) & (scale * 224.0 >= top), scale * 0.5, scale)
    y = x / scale
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(y / unit) * unit * scale                         # ties to even


def _exact_inputs(case, seed):
    """prepare's inputs, with the cache as plain arrays whatever the side."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def exact(case, seed):
    s = _exact_inputs(case, seed)
    if case["op"] == "rotary":
        freq = _frequencies(case["rotary_dim"], _scaling(case["scaling"]))
        return {n: _turn64(s[n], s["pos"], freq, case["interleaved"]) for n in ("q", "k")}
    if case["op"] == "cache":
        B, n, r = case["batch"], case["new"], case["read"]
        k, v = s["k"].double(), s["v"].double()
        if case["rotated"]:
            k = _turn64(s["k"], s["pos"], _frequencies(case["head_dim"], None), False)
        if case["cache"] == "fp8":
            k, v = _eight64(k), _eight64(v)
        out = []
        for x in (k, v):                                                # positions before the new ones hold nothing yet
            x = torch.cat([torch.zeros(B, max(0, r - n), *x.shape[1:], dtype=torch.float64, device="cuda"), x.view(B, n, *x.shape[1:])[:, max(0, n - r):]], 1)
            out.append(x.flatten(0, 1))
        return dict(k=out[0], v=out[1])
    if case["op"] == "logprobs":
        parts = []
        step = max(1, (1 << 26) // case["vocab"])
        for i in range(0, case["rows"], step):
            x = s["logits"][i:i + step].double() * case["scale"]
            logp = torch.log_softmax(x, -1)
            o = dict(entropy=-torch.where(logp > -1e300, logp.exp() * logp, torch.zeros_like(logp)).sum(-1), lse=torch.logsumexp(x, -1))
            if case["targets"]:
                o["logprobs"] = torch.take_along_dim(logp, s["targets"][i:i + step].long(), 1)
            if case["top"]:
                ids, at = [], torch.arange(x.shape[1], device="cuda")
                for _ in range(case["top"]):                            # the lowest place of the largest that is left
                    best = torch.where(x == x.amax(-1, keepdim=True), at, x.shape[1]).amin(-1, keepdim=True)
                    ids.append(best)
                    x.scatter_(1, best, -math.inf)
                o["top_ids"] = torch.cat(ids, 1).int()
                o["top_logprobs"] = torch.take_along_dim(logp, o["top_ids"].long(), 1)
            parts.append(o)
        return {n: torch.cat([p[n] for p in parts]) for n in parts[0]}
    q, mask = s["q"], s["mask"]
    B, T, H, hd = q.shape
    Hkv = case["kv_heads"]
    out = torch.zeros(B, T, H, hd, dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, H), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        P, n = int(s["host_lens"][b]), int(s["host_trees"][b])
        k, v = _read(s, _slots(s["table"], torch.full((P + n,), b, device="cuda"), torch.arange(P + n, device="cuda")), torch.float64)
        see = torch.ones(n, P + n, dtype=torch.bool, device="cuda")
        if mask is not None:
            for j in range(n):
                see[:, P + j] = (mask[b, :n, j // 64] >> (j % 64)) & 1 == 1
        for h in range(H):
            score = q[b, :n, h].double() @ k[:, h // (H // Hkv)].T.contiguous() / hd ** 0.5
            score = torch.where(see, score, torch.full_like(score, -math.inf))
            lse[b, :n, h] = torch.logsumexp(score, -1)
            out[b, :n, h] = torch.softmax(score, -1) @ v[:, h // (H // Hkv)]
    return dict(out=out, lse=lse)
