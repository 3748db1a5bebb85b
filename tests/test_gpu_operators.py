"""The operators of a batched tree verification on the GPU against plain implementations in 64 bits: rotary positions, the paged
cache, tree attention and log probabilities.  Needs an MI355X.

Tolerances, derived from the formats: a result rounded to bf16 (8 bits) is off by 2^-8 of itself, to fp32 by 2^-24; fp32 arithmetic adds a few
2^-24 per operation.  What each test allows is written where it is used.
"""
import math

import numpy as np
import pytest
import torch

import paper_2411_03786_amd as ngg

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
NAN, INF = float("nan"), float("inf")


def randn(*shape, seed=0, dtype="f32"):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(DT[dtype]).cuda()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- rotary ---------------------------------------------------------------------------------------------------------

def rotate64(x, pos, rope, inverse=False):
    """x [n, heads, hd] in 64 bits by the table's own entries, and what fp32 arithmetic may be off by."""
    half = rope.rotary_dim // 2
    c, s = rope.cos[pos.long()].double()[:, None], rope.sin[pos.long()].double()[:, None]
    s = -s if inverse else s
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if rope.interleaved else (i, i + half)
    out, slack = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    u, v = x[..., a].double(), x[..., b].double()
    out[..., a], out[..., b] = u * c - v * s, v * c + u * s
    slack[..., a] = slack[..., b] = (u.abs() + v.abs()) * 2.0 ** -22
    return out, slack


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,H,Hkv,hd,rd,inter", [(1, 4, 4, 32, 32, False), (7, 12, 3, 64, 64, True), (51, 32, 32, 128, 128, False), (33, 8, 2, 128, 64, True),
                                                 (65, 3, 1, 80, 80, False), (5, 2, 2, 30, 30, True), (9, 5, 1, 34, 18, False), (300, 32, 8, 128, 34, True),
                                                 (2, 1, 1, 256, 256, False), (1030, 24, 6, 128, 128, False), (3, 2, 2, 2, 2, False)])
def test_rotary_of_strided_rows(dtype, n, H, Hkv, hd, rd, inter):
    x = randn(n, (H + 2 * Hkv) * hd + 6, seed=n, dtype=dtype)            # the slices of a fused projection, an odd row stride behind them
    q, k = x[:, :H * hd].view(n, H, hd), x[:, H * hd:(H + Hkv) * hd].view(n, Hkv, hd)
    rope = ngg.Rope(rd, 500, interleaved=inter)
    pos = torch.randint(0, 500, (n,), dtype=torch.int32, generator=torch.Generator().manual_seed(n)).cuda()
    before = x.clone()
    for inverse in (False, True):
        got = ngg.rotary(rope, pos, q, k, inverse=inverse)
        for g, t in zip(got, (q, k)):
            want, slack = rotate64(t, pos, rope, inverse)
            assert ((g.double() - want).abs() <= slack + want.abs() * ROUND[dtype] * 1.01).all()
            assert torch.equal(g[..., rd:], t[..., rd:])
        assert torch.equal(ngg.rotary(rope, pos, q, inverse=inverse), got[0])     # alone as together
    assert torch.equal(x, before)
    # in place, and into heads that lie apart
    want = ngg.rotary(rope, pos, q, k)
    apart = torch.full((H, n, hd + 3), 7.0, dtype=DT[dtype], device="cuda")
    ngg.rotary(rope, pos, q, k, out=apart.permute(1, 0, 2)[..., :hd], k_out=k)
    assert torch.equal(apart.permute(1, 0, 2)[..., :hd], want[0]) and torch.equal(k, want[1])
    assert (apart[..., hd:] == 7.0).all() and torch.equal(x[:, (H + Hkv) * hd:], before[:, (H + Hkv) * hd:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,H,Hkv,hd,rd,inter,pad", [(700, 32, 8, 128, 128, False, 8), (1025, 32, 8, 64, 64, True, 0), (900, 24, 8, 128, 64, False, 16),
                                                     (901, 40, 8, 96, 32, True, 8), (3000, 7, 1, 80, 48, False, 8), (2050, 9, 0, 256, 128, True, 0),
                                                     (4100, 3, 2, 112, 112, False, 24), (140, 100, 3, 192, 16, False, 8)])
def test_rotary_of_many_aligned_rows(dtype, n, H, Hkv, hd, rd, inter, pad):
    x = randn(n, (H + Hkv) * hd + pad, seed=n, dtype=dtype)
    q, k = x[:, :H * hd].view(n, H, hd), x[:, H * hd:(H + Hkv) * hd].view(n, Hkv, hd)
    rope = ngg.Rope(rd, 900, interleaved=inter)
    pos = torch.randint(0, 900, (n,), dtype=torch.int32, generator=torch.Generator().manual_seed(n)).cuda()
    pos[n // 2] = 900                                                   # behind the table: NaN
    live = torch.arange(n, device="cuda") != n // 2
    for inverse in (False, True):
        got = ngg.rotary(rope, pos, q, k, inverse=inverse) if Hkv else (ngg.rotary(rope, pos, q, inverse=inverse),)
        for g, t in zip(got, (q, k)):
            want, slack = rotate64(t[live], pos[live], rope, inverse)
            assert ((g[live].double() - want).abs() <= slack + want.abs() * ROUND[dtype] * 1.01).all()
            assert torch.equal(g[..., rd:], t[..., rd:]) and torch.isnan(g[n // 2, :, :rd]).all()
        few = ngg.rotary(rope, pos[5:8], q[5:8], inverse=inverse)
        assert torch.equal(few, got[0][5:8])                            # a few rows as many
    want = got[0]
    ngg.rotary(rope, pos, q, inverse=True, out=q)
    assert torch.equal(q[live], want[live])


def test_rotary_inverse_is_the_gradient():
    """d/dx <w, R x> = R^T w, by differences in 64 bits of the fp32 kernel's own results (which are linear in x)."""
    n, H, hd = 4, 2, 16
    rope = ngg.Rope(12, 40, scaling=dict(kind="linear", factor=2.0))
    pos, x, w = ints([0, 3, 39, 7]), randn(n, H, hd, seed=1), randn(n, H, hd, seed=2)
    grad = ngg.rotary(rope, pos, w, inverse=True)
    for i in range(hd):
        step = torch.zeros_like(x)
        step[..., i] = 1.0
        diff = (ngg.rotary(rope, pos, x + step).double() - ngg.rotary(rope, pos, x - step).double()) / 2
        # the sums of 16 products of values below 5, each off by a few 2^-24
        assert ((diff * w.double()).sum(-1) - grad[..., i].double()).abs().max() < 16 * 25 * 8 * 2.0 ** -24


def test_rotary_out_of_range_and_empty():
    rope = ngg.Rope(8, 10)
    x = randn(4, 3, 12, seed=3)
    out = ngg.rotary(rope, ints([0, -1, 10, 9]), x)
    assert torch.isnan(out[1:3, :, :8]).all() and torch.equal(out[1:3, :, 8:], x[1:3, :, 8:]) and torch.isfinite(out[[0, 3]]).all()
    assert torch.equal(out[0], x[0])
    assert ngg.rotary(rope, ints([]), x[:0]).shape == (0, 3, 12)


def test_rotary_refuses_on_the_host():
    rope, x = ngg.Rope(8, 10), randn(4, 3, 12)
    pos = ints([0, 1, 2, 3])
    with pytest.raises(ngg.NggError):
        ngg.rotary(ngg.Rope(16, 10), pos, x)
    with pytest.raises(TypeError):
        ngg.rotary(rope, pos.long(), x)
    with pytest.raises(TypeError):
        ngg.rotary(rope, pos, x.double())
    with pytest.raises(TypeError):
        ngg.rotary(rope, pos[:3], x)
    with pytest.raises(ValueError):
        ngg.rotary(rope, pos, x.transpose(1, 2))
    with pytest.raises(ValueError):
        ngg.rotary(rope, pos, x, x[:, :, :8])
    with pytest.raises(ValueError):
        ngg.rotary(rope, pos, x, out=torch.empty(4, 3, 13, device="cuda"))


# ---- the paged cache --------------------------------------------------------------------------------------------------

def eight_bits(x):
    """x [..., hd] -> its values in 8 bits: all magnitudes of the format, the head's power of two, the nearest of them (ties to even)."""
    mags = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)]
    grid = np.array(mags[:-1])                                          # the last code is NaN; 448 is the largest
    x = x.double().cpu().numpy()
    fin = np.where(np.isfinite(x), x, 0.0)
    top = np.abs(fin).max(-1, keepdims=True)
    e = np.full_like(top, -126.0)
    for k in range(-126, 120):
        e = np.where(448.0 * 2.0 ** k < top, k + 1.0, e)
    e = np.where(top > 0, e, 0.0)
    y = np.abs(fin) / 2.0 ** e
    hi = np.clip(np.searchsorted(grid, y), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    up = (grid[hi] - y < y - grid[lo]) | ((grid[hi] - y == y - grid[lo]) & (hi % 2 == 0))
    val = np.where(up, grid[hi], grid[lo]) * np.sign(fin) * 2.0 ** e
    return torch.from_numpy(np.where(np.isfinite(x), val, np.nan)).cuda()


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("f32", "fp8"), ("bf16", "fp8")])
@pytest.mark.parametrize("hd,Hkv,page", [(32, 4, 32), (64, 3, 96), (128, 8, 64), (64, 90, 32), (32, 200, 64), (128, 200, 32)])
@pytest.mark.parametrize("n,order", [(1, "run"), (5, "run"), (32, "run"), (61, "run"), (200, "run"), (97, "shuffled"), (130, "halves")])
def test_cache_holds_what_was_written(dtype, cache, hd, Hkv, page, n, order):
    pool = 300 // page + 3
    kv = ngg.KVPages(pool, page, Hkv, hd, cache)
    rng = np.random.default_rng(n * hd)
    slots = 13 + np.arange(n)
    if order == "shuffled":
        slots = rng.permutation(pool * page)[:n]
    if order == "halves":                                              # two sequences' runs, one of them backwards
        slots = np.concatenate([100 + np.arange(n // 2), 99 - np.arange(n - n // 2)]).clip(0)
        slots = np.unique(slots)[::-1].copy()
        n = len(slots)
    x = randn(n, 3 * Hkv * hd, seed=n, dtype=dtype) * torch.where(torch.rand(n, 1, generator=torch.Generator().manual_seed(1)) < 0.3, 1000.0, 0.1).cuda().to(DT[dtype])
    k, v = x[:, Hkv * hd:2 * Hkv * hd].view(n, Hkv, hd), x[:, 2 * Hkv * hd:].view(n, Hkv, hd)
    old_k, old_v = (randn(pool * page, Hkv, hd, seed=s, dtype=dtype) for s in (8, 9))
    kv.write(old_k, old_v, ints(np.arange(pool * page)))
    kv.write(k, v, ints(slots))
    asis = (lambda t: eight_bits(t)) if cache == "fp8" else (lambda t: t.double())
    want_k, want_v = asis(old_k), asis(old_v)
    at = torch.from_numpy(slots).cuda()
    want_k[at], want_v[at] = asis(k), asis(v)
    for order2 in (np.arange(pool * page), rng.permutation(pool * page)[:77], slots):
        got_k, got_v = kv.read(ints(order2), DT[dtype])
        o = torch.from_numpy(order2).cuda()
        assert torch.equal(got_k.double(), want_k[o].to(DT[dtype]).double()) and torch.equal(got_v.double(), want_v[o].to(DT[dtype]).double())
    # writing what was read changes no byte
    bytes_before = [t.clone() for t in (kv.k_bytes, kv.v_bytes)]
    kv.write(*kv.read(ints(slots), DT[dtype]), ints(slots))
    again = kv.read(ints(slots), DT[dtype])
    assert torch.equal(again[0].double(), want_k[at].to(DT[dtype]).double()) and torch.equal(again[1].double(), want_v[at].to(DT[dtype]).double())
    if cache != "fp8":
        assert torch.equal(bytes_before[0], kv.k_bytes) and torch.equal(bytes_before[1], kv.v_bytes)


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("f32", "fp8"), ("bf16", "fp8")])
@pytest.mark.parametrize("hd,Hkv", [(32, 5), (64, 3), (128, 2)])
@pytest.mark.parametrize("tree,start", [(61, 0), (13, 5), (8, 8), (9, 7), (3, 30), (40, 1)])
def test_cache_of_many_sequences_runs(dtype, cache, hd, Hkv, tree, start):
    """Runs of slots that begin and end inside the groups that move together, with places left out, as one call and row by row."""
    B, page = 20 + 1200 // tree, 64
    rng = np.random.default_rng(tree)
    slots = np.concatenate([(2 * page * b + start + 3 * (b % 5) + np.arange(tree)) for b in rng.permutation(B)])
    slots[rng.permutation(len(slots))[:5]] = -1
    n, pool = len(slots), 2 * B + 2
    x = randn(n, 2 * Hkv * hd, seed=tree, dtype=dtype)
    k, v = x[:, :Hkv * hd].view(n, Hkv, hd), x[:, Hkv * hd:].view(n, Hkv, hd)
    whole, parts = (ngg.KVPages(pool, page, Hkv, hd, cache) for _ in range(2))
    whole.write(k, v, ints(slots))
    for at in range(0, n, 200):
        parts.write(k[at:at + 200], v[at:at + 200], ints(slots[at:at + 200]))
    assert torch.equal(whole.k_bytes, parts.k_bytes) and torch.equal(whole.v_bytes, parts.v_bytes)
    if cache == "fp8":
        assert torch.equal(whole.k_exps, parts.k_exps) and torch.equal(whole.v_exps, parts.v_exps)
    got = whole.read(ints(slots), DT[dtype])
    there = torch.from_numpy(slots >= 0).cuda()
    for g, t in zip(got, (k, v)):
        want = eight_bits(t).to(DT[dtype]) if cache == "fp8" else t
        assert torch.equal(g[there], want[there]) and (g[~there] == 0).all()
    some = whole.read(ints(slots[:100]), DT[dtype])
    assert torch.equal(some[0], got[0][:100]) and torch.equal(some[1], got[1][:100])


def test_eight_bit_corners():
    """Heads of zeros, the largest value exactly and just above, the smallest exponents, numbers that are not finite."""
    hd = 32
    rows = torch.zeros(12, 1, hd)
    rows[1, 0, 0] = 448.0
    rows[2, 0, :2] = torch.tensor([448.00003, 1.0])
    rows[3, 0] = torch.linspace(-3.4e38, 3.4e38, hd)
    rows[4, 0] = 1e-40
    rows[5, 0, :3] = torch.tensor([INF, -2.0, 3.3])
    rows[6, 0, :3] = torch.tensor([NAN, 1e-3, -7.0])
    rows[7, 0] = INF
    rows[8, 0, :4] = torch.tensor([1.0, 1.0 / 16 + 1.0, 0.002, -0.0])
    rows[9, 0] = torch.linspace(1e-38, 3e-36, hd)
    rows[10, 0, :5] = torch.tensor([448.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 5 * 2.0 ** -10])
    rows[11, 0] = torch.linspace(-1, 1, hd)
    for heads in (1, 400):
        x = rows.expand(-1, heads, -1).contiguous().cuda()
        kv = ngg.KVPages(2, 32, heads, hd, "fp8")
        slots = ints(range(20, 32))
        kv.write(x, x.flip(0).contiguous(), slots)
        k, v = (t[:, -1:] for t in kv.read(slots, torch.float32))
        check_corners(rows.cuda(), k, v)


def check_corners(x, k, v):
    want = eight_bits(x).float()
    assert torch.equal(torch.nan_to_num(k, nan=-77.0), torch.nan_to_num(want, nan=-77.0))
    assert torch.equal(torch.nan_to_num(v, nan=-77.0), torch.nan_to_num(want.flip(0), nan=-77.0))


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("H", [2, 2100])
def test_cache_slots_out_of_range(cache, H):
    kv = ngg.KVPages(2, 32, H, 64, cache)
    x = randn(6, H, 64, seed=1, dtype="bf16")
    kv.write(x[:2], x[2:4], ints([5, 6]))
    before = [t.clone() for t in (kv.k_bytes, kv.v_bytes)]
    kv.write(x[:4], x[2:6], ints([-1, 64, 2 ** 31 - 1, -2 ** 31]))
    assert torch.equal(before[0], kv.k_bytes) and torch.equal(before[1], kv.v_bytes)
    k, v = kv.read(ints([-1, 5, 64, 2 ** 31 - 1, 6]))
    assert (k[[0, 2, 3]] == 0).all() and (v[[0, 2, 3]] == 0).all() and (k[[1, 4]] != 0).any()
    # runs that leave the pool or begin before it
    kv.write(x, x, ints(range(61, 67)))
    kv.write(x, x, ints(range(-3, 3)))
    k2, _ = kv.read(ints([61, 62, 63, 0, 1, 2]))
    want = torch.cat([x[:3], x[3:]])
    assert torch.equal(k2, want if cache == "bf16" else eight_bits(want).bfloat16())
    kv.write(x[:0], x[:0], ints([]))
    assert kv.read(ints([]))[0].shape == (0, H, 64)


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("f32", "fp8"), ("bf16", "fp8")])
@pytest.mark.parametrize("hd,rd,inter", [(32, 32, False), (64, 32, True), (128, 128, True), (128, 128, False), (128, 34, False), (64, 6, True)])
@pytest.mark.parametrize("Hkv,n", [(3, 75), (60, 75)])
def test_cache_rotates_as_rotary_does(dtype, cache, hd, rd, inter, Hkv, n):
    rope, pos = ngg.Rope(rd, 300, interleaved=inter), ints(np.random.default_rng(2).integers(0, 300, n))
    x = randn(n, 2 * Hkv * hd + 2, seed=hd, dtype=dtype)
    k, v = x[:, :Hkv * hd].view(n, Hkv, hd), x[:, Hkv * hd:2 * Hkv * hd].view(n, Hkv, hd)
    a, b = (ngg.KVPages(4, 32, Hkv, hd, cache) for _ in range(2))
    slots = ints(7 + np.arange(n))
    a.write(k, v, slots, rope=rope, positions=pos)
    b.write(ngg.rotary(rope, pos, k), v, slots)
    assert torch.equal(a.k_bytes, b.k_bytes) and torch.equal(a.v_bytes, b.v_bytes)
    if cache == "fp8":
        assert torch.equal(a.k_exps, b.k_exps) and torch.equal(a.v_exps, b.v_exps)


def test_cache_beyond_32_bits_of_elements():
    """The last pages of a pool whose keys alone pass 2^32 bytes and 2^31 elements."""
    Hkv, hd, page = 8, 128, 256
    pool = (1 << 31) // (Hkv * hd * page) + 3
    kv = ngg.KVPages(pool, page, Hkv, hd, "bf16")
    n = 100
    slots = ints(pool * page - n - 20 + np.arange(n))
    k, v = randn(n, Hkv, hd, seed=1, dtype="bf16"), randn(n, Hkv, hd, seed=2, dtype="bf16")
    kv.write(k, v, slots)
    got = kv.read(slots)
    assert torch.equal(got[0], k) and torch.equal(got[1], v)
    q = randn(1, 1, Hkv, hd, seed=3, dtype="bf16")
    table = ints([[pool - 1]])
    kv.write(k, v, ints((pool - 1) * page + np.arange(n)))
    out, lse = ngg.tree_attention(q, kv, table, ints([n - 1]), want_lse=True)
    check_attention(out, lse, *attention64(q, [k], [v], [n - 1], [1], None, hd ** -0.5), "bf16")
    assert not kv.k_bytes[:1 << 20].any()


# ---- tree attention ---------------------------------------------------------------------------------------------------

def attention64(q, ks, vs, ctx, trees, mask, scale):
    """Out, lse, and for the tolerances sum p |v| and the largest sum of |q k| of a row, in 64 bits.  mask [B, T, T] bool or None."""
    B, T, H, hd = q.shape
    out, mag = (torch.zeros(B, T, H, hd, dtype=torch.float64, device="cuda") for _ in range(2))
    lse, qk = torch.full((B, T, H), -INF, dtype=torch.float64, device="cuda"), torch.zeros(B, T, H, dtype=torch.float64, device="cuda")
    for b in range(B):
        P, n = max(ctx[b], 0), trees[b]
        if n == 0:
            continue
        G = H // ks[b].shape[1]
        k, v = ks[b][:P + n].double(), vs[b][:P + n].double()
        see = torch.ones(n, P + n, dtype=torch.bool, device="cuda")
        see[:, P:] = torch.tril(torch.ones(n, n, dtype=torch.bool, device="cuda"))
        if mask is not None:
            see[:, P:] &= mask[b][:n, :n]
        for h in range(H):
            kh, vh = k[:, h // G], v[:, h // G]
            x = q[b, :n, h].double()
            for t in range(n):
                on = see[t]
                if not on.any():
                    continue
                s = (kh[on] @ x[t]) * scale
                m = s.max()
                p = torch.exp(s - m)
                out[b, t, h] = (p[:, None] * vh[on]).sum(0) / p.sum()
                mag[b, t, h] = (p[:, None] * vh[on].abs()).sum(0) / p.sum()
                lse[b, t, h] = m + torch.log(p.sum())
                qk[b, t, h] = (kh[on].abs() @ x[t].abs()).max() * scale
    return out, lse, mag, qk


def check_attention(out, lse, want, want_lse, mag, qk, dtype):
    """fp32: scores off by (head_dim + 8) 2^-24 of the sum of |q k|, twice that in a quotient of sums; bf16: the probabilities' and the
    result's rounding besides.  Sums of up to 10^5 terms in up to 10^3 pieces: 2^-15."""
    hd = out.shape[-1]
    e = (2 * (hd + 8) * 2.0 ** -24 * qk + 2.0 ** -15)[..., None]
    tol = mag * (e + (2.0 ** -8 if dtype == "bf16" else 0)) + want.abs() * ROUND[dtype] + 1e-30
    bad = (out.double() - want).abs() > tol
    assert not bad.any(), ((out.double() - want).abs() / tol).max()
    assert torch.isfinite(out).all()
    dead = want_lse == -INF
    assert (lse[dead] == -INF).all() and (out[dead] == 0).all()
    err = (lse.double() - want_lse).abs()[~dead]
    assert (err <= (((hd + 8) * 2.0 ** -24 * qk + 2.0 ** -15) + 2.0 ** -22 * want_lse.abs())[~dead]).all()


class Case:
    """Sequences of random keys and values in a pool of shuffled pages whose unwritten places hold NaN."""

    def __init__(self, ctx, trees, T, H, Hkv, hd, dtype="bf16", cache=None, page=32, seed=0, spare=1, sharp=1.0, wide=False):
        cache = cache or dtype
        rng = np.random.default_rng(seed)
        B = len(ctx)
        per = max(max(max(c, 0) + t for c, t in zip(ctx, trees)), 1)
        per = -(-per // page) + spare
        pool = B * per + 2
        self.kv = ngg.KVPages(pool, page, Hkv, hd, cache)
        self.kv.k_bytes.fill_(255)                                     # NaN in all three types
        self.kv.v_bytes.fill_(255)
        if cache == "fp8":
            self.kv.k_exps.fill_(255)
            self.kv.v_exps.fill_(255)
        self.table = ints(rng.permutation(pool)[:B * per].reshape(B, per))
        if wide:                                                        # a page list long enough for the kernels of long contexts
            more = -(-max(1 << 19, (42 << 20) // (T * (H // Hkv))) // (page * B * Hkv))
            self.table = torch.cat([self.table, torch.full((B, more), -1, dtype=torch.int32, device="cuda")], 1)
        self.ks, self.vs = [], []
        for b in range(B):
            n = max(ctx[b], 0) + trees[b]
            k, v = randn(n, Hkv, hd, seed=seed * 100 + b, dtype=dtype) * sharp, randn(n, Hkv, hd, seed=seed * 100 + b + 50, dtype=dtype)
            pos = torch.arange(n, device="cuda")
            slots = (self.table[b, pos // page] * page + pos % page).int()
            self.kv.write(k, v, slots)
            k, v = self.kv.read(slots, DT[dtype])
            self.ks.append(k)
            self.vs.append(v)
        self.ctx, self.trees, self.T, self.dtype = list(ctx), list(trees), T, dtype
        self.q = randn(B, T, H, hd, seed=seed + 7, dtype=dtype)
        self.scale = hd ** -0.5

    def masks(self, seed=0, empty=()):
        """A random tree per sequence as bool [B, T, T] and as words."""
        rng = np.random.default_rng(seed)
        B, T = len(self.ctx), self.T
        see, words = np.zeros((B, T, T), bool), np.zeros((B, T, -(-T // 64)), np.uint64)
        for b in range(B):
            for t in range(T):
                p = int(rng.integers(-1, t)) if t else -1
                if p >= 0:
                    see[b, t] = see[b, p]
                see[b, t, t] = True
            for t in empty:
                see[b, t] = False
            for t in range(T):
                for j in np.flatnonzero(see[b, t]):
                    words[b, t, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        return torch.from_numpy(see).cuda(), torch.from_numpy(words.view(np.int64)).cuda()

    def check(self, words=None, see=None, **more):
        lens = ints(self.trees) if self.trees != [self.T] * len(self.trees) else None
        out, lse = ngg.tree_attention(self.q, self.kv, self.table, ints(self.ctx), mask=words, tree_lens=lens, want_lse=True, **more)
        check_attention(out, lse, *attention64(self.q, self.ks, self.vs, self.ctx, self.trees, see, self.scale), self.dtype)
        return out, lse


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f32", "fp8"), ("bf16", "fp8")]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("H,Hkv,hd", [(4, 4, 32), (6, 2, 64), (8, 2, 128), (3, 3, 128)])
@pytest.mark.parametrize("T,ctx", [(1, 0), (1, 1), (1, 31), (1, 300), (2, 127), (5, 0), (13, 128), (17, 65), (33, 200), (65, 97), (70, 1000)])
@pytest.mark.parametrize("wide", [False, True])
def test_tree_attention_one_sequence(dtype, cache, H, Hkv, hd, T, ctx, wide):
    c = Case([ctx], [T], T, H, Hkv, hd, dtype, cache, seed=T + ctx, wide=wide)
    see, words = c.masks(seed=T)
    c.check(words, see)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("page", [32, 64, 160])
@pytest.mark.parametrize("wide", [False, True])
def test_tree_attention_ragged_batch(dtype, cache, page, wide):
    ctx = [0, 1, 31, 32, 33, 500, 1999, 64, 5]
    trees = [3, 19, 0, 19, 1, 7, 18, 19, 2]
    c = Case(ctx, trees, 19, 8, 2, 64, dtype, cache, page=page, seed=3, wide=wide)
    see, words = c.masks(seed=4)
    c.check(words, see)
    c.check(None, None)                                                 # a chain each
    c.check(words[0].contiguous(), see[:1].expand(len(ctx), -1, -1))    # one tree for all


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_tree_attention_many_short_sequences(dtype, cache):
    rng = np.random.default_rng(5)
    ctx = [int(x) for x in rng.integers(0, 90, 70)]
    c = Case(ctx, [1] * 70, 1, 4, 1, 32, dtype, cache, seed=6)
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("H,Hkv,hd,T,ctx", [(4, 1, 128, 64, 3000), (2, 2, 64, 150, 513), (8, 1, 32, 33, 700), (1, 1, 128, 300, 100)])
@pytest.mark.parametrize("wide", [False, True])
def test_tree_attention_wide_trees(dtype, cache, H, Hkv, hd, T, ctx, wide):
    """More rows than a tile, masks of several words."""
    c = Case([ctx, ctx // 3], [T, T - 5], T, H, Hkv, hd, dtype, cache, page=64, seed=T, wide=wide)
    see, words = c.masks(seed=T + 1)
    c.check(words, see)
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_tree_attention_long_context(dtype, cache):
    c = Case([40000, 9, 17001], [6, 6, 6], 6, 4, 1, 64, dtype, cache, page=256, seed=8)
    see, words = c.masks(seed=8)
    c.check(words, see)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("H,Hkv,hd,T", [(4, 2, 128, 1), (8, 1, 64, 2), (3, 3, 32, 13), (16, 1, 128, 1)])
def test_tree_attention_page_lists_beyond_the_caches(dtype, cache, H, Hkv, hd, T):
    """Few rows and page lists of more keys than any cache holds."""
    ctx = [0, 1000, 63]
    c = Case(ctx, [T] * 3, T, H, Hkv, hd, dtype, cache, seed=hd + T)
    room = (1 << 29) // (2 * hd * Hkv * 3)                              # positions, one byte an element
    c.table = torch.cat([c.table, torch.full((3, room // 32), -1, dtype=torch.int32, device="cuda")], 1)
    see, words = c.masks(seed=8)
    c.check(words, see)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("wide", [False, True])
def test_tree_attention_sharp_scores(dtype, cache, wide):
    """Scores in the hundreds: the running maximum moves, and single keys carry rows."""
    c = Case([700, 33], [20, 20], 20, 4, 2, 128, dtype, cache, seed=9, sharp=30.0, wide=wide)
    see, words = c.masks(seed=9)
    c.check(words, see)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("wide", [False, True])
def test_tree_attention_rows_that_see_nothing(dtype, cache, wide):
    c = Case([0, 40], [9, 9], 9, 8, 2, 64, dtype, cache, seed=10, wide=wide)
    see, words = c.masks(seed=10, empty=(0, 4, 8))
    c.check(words, see)
    c = Case([-5, 0], [0, 4], 4, 4, 2, 64, dtype, cache, seed=10)       # a sequence that is not there
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("wide", [False, True])
def test_tree_attention_masked_numbers_that_are_not_finite(dtype, cache, bad, wide):
    """One tree token's key, then another's value, is not finite: the rows that do not see it are as they were."""
    T, ctx = 21, 50
    c = Case([ctx], [T], T, 4, 2, 64, dtype, cache, seed=11, wide=wide)
    see, words = c.masks(seed=11)
    clean, clean_lse = c.check(words, see)
    for j, which in ((7, "k"), (12, "v")):
        k, v = c.ks[0][ctx + j:ctx + j + 1].clone(), c.vs[0][ctx + j:ctx + j + 1].clone()
        (k if which == "k" else v)[..., 3] = bad
        slot = c.table[0, (ctx + j) // 32] * 32 + (ctx + j) % 32
        c.kv.write(k, v, slot[None].int())
        out, lse = ngg.tree_attention(c.q, c.kv, c.table, ints([ctx]), mask=words, want_lse=True)
        hit = see[0, :, j]
        assert hit.any() and not hit.all()
        assert torch.equal(out[0, ~hit], clean[0, ~hit]) and torch.equal(lse[0, ~hit], clean_lse[0, ~hit])
        if which == "v" and cache == "fp8":                             # the head's other values have a power of two of their own then
            assert torch.isnan(out[0, hit][..., 3]).all()
        elif which == "v":
            assert not torch.isfinite(out[0, hit][..., 3]).any()
            if bad != bad:
                assert torch.isnan(out[0, hit][..., 3]).all()
            others = [d for d in range(64) if d != 3]
            assert torch.equal(out[0, hit][..., others], clean[0, hit][..., others])
        c.kv.write(c.ks[0][ctx + j:ctx + j + 1].contiguous(), c.vs[0][ctx + j:ctx + j + 1].contiguous(), slot[None].int())
    assert torch.equal(ngg.tree_attention(c.q, c.kv, c.table, ints([ctx]), mask=words), clean)


@pytest.mark.parametrize("wide,T", [(False, 5), (True, 40)])
def test_tree_attention_a_bad_number_in_the_context_reaches_every_row(wide, T):
    c = Case([100], [T], T, 2, 2, 64, "bf16", seed=12, wide=wide)
    k, v = c.ks[0][10:11].clone(), c.vs[0][10:11].clone()
    v[..., 0] = NAN
    c.kv.write(k, v, (c.table[0, 0] * 32 + 10)[None].int())
    out = ngg.tree_attention(c.q, c.kv, c.table, ints([100]))
    assert torch.isnan(out[..., 0]).all() and torch.isfinite(out[..., 1:]).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("H", [4, 24])
def test_tree_attention_pages_and_lengths_out_of_range(dtype, cache, H):
    """A page outside the pool hides its positions; lengths past the page list are cut."""
    T, ctx = 3, 150
    c = Case([ctx], [T], T, H, 2, 64, dtype, cache, seed=13, spare=0)
    for wrong in (-1, c.kv.n_pages, 2 ** 31 - 1, -2 ** 31):
        table = c.table.clone()
        table[0, 2] = wrong                                             # positions 64 .. 95
        out, lse = ngg.tree_attention(c.q, c.kv, table, ints([ctx]), want_lse=True)
        keep = torch.cat([torch.arange(64), torch.arange(96, ctx + T)]).cuda()
        check_attention(out, lse, *attention64(c.q, [c.ks[0][keep]], [c.vs[0][keep]], [ctx - 32], [T], None, c.scale), dtype)
    out, lse = ngg.tree_attention(c.q, c.kv, torch.full_like(c.table, -1), ints([ctx]), want_lse=True)
    assert (out == 0).all() and (lse == -INF).all()
    # the same with the kernels of long contexts
    w = Case([ctx], [40], 40, H, 2, 64, dtype, cache, seed=21, wide=True)
    w.table[0, 2] = -1
    out, lse = ngg.tree_attention(w.q, w.kv, w.table, ints([ctx]), want_lse=True)
    keep = torch.cat([torch.arange(64), torch.arange(96, ctx + 40)]).cuda()
    check_attention(out, lse, *attention64(w.q, [w.ks[0][keep]], [w.vs[0][keep]], [ctx - 32], [40], None, w.scale), dtype)
    n = c.table.shape[1] * 32                                           # 160 places, 153 of them written
    x = randn(7, 2, 64, seed=14, dtype=dtype)
    c.kv.write(x, x, (c.table[0, -1] * 32 + torch.arange(25, 32, device="cuda")).int())
    full = c.kv.read((c.table[0, torch.arange(n, device="cuda") // 32] * 32 + torch.arange(n, device="cuda") % 32).int(), DT[dtype])
    for long in (n, 10 ** 6, 2 ** 31 - 1):
        out, lse = ngg.tree_attention(c.q, c.kv, c.table, ints([long]), want_lse=True)
        see = torch.zeros(1, T, T, dtype=torch.bool, device="cuda")     # no place is left for the tree's own keys
        pad = [torch.cat([t, t[:T]]) for t in full]
        check_attention(out, lse, *attention64(c.q, pad[:1], pad[1:], [n], [T], see, c.scale), dtype)
    out = ngg.tree_attention(c.q, c.kv, c.table, ints([ctx]), tree_lens=ints([2 ** 31 - 1]))
    assert torch.equal(out, ngg.tree_attention(c.q, c.kv, c.table, ints([ctx])))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,wide", [(5, False), (20, True)])
def test_tree_attention_strides(dtype, T, wide):
    """Queries and outputs as slices of something larger, at odd offsets, and a page list with a stride."""
    B, H, Hkv, hd = 3, 4, 2, 64
    c = Case([40, 7, 130], [T] * 3, T, H, Hkv, hd, dtype, seed=15, wide=wide)
    want = c.check()[0]
    for gap in (0, 1, 2, 8):
        big = torch.zeros(T, B, H, hd + gap, dtype=DT[dtype], device="cuda")
        qv = big.permute(1, 0, 2, 3)[..., gap:]
        qv.copy_(c.q)
        dst = torch.full((B, H, T, hd + gap), 5.0, dtype=DT[dtype], device="cuda")
        ov = dst.permute(0, 2, 1, 3)[..., gap:]
        table = torch.full((B, c.table.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
        table[:, :-3] = c.table
        ngg.tree_attention(qv, c.kv, table[:, :-3], ints(c.ctx), out=ov)
        assert torch.equal(ov, want) and (gap == 0 or (dst[..., :gap] == 5.0).all())
    one = c.q[:1].expand(B, -1, -1, -1)                                 # one query for all sequences
    got = ngg.tree_attention(one, c.kv, c.table, ints(c.ctx))
    assert torch.equal(got, ngg.tree_attention(one.contiguous(), c.kv, c.table, ints(c.ctx)))
    # another scale
    c.scale = 0.3
    c.check(scale=0.3)


def test_operators_on_another_stream_and_in_a_graph():
    """A layer's chain, captured and replayed with inputs, lengths and slots that change in place; and on a stream of its own."""
    B, T, H, Hkv, hd = 2, 9, 4, 2, 64
    c = Case([100, 37], [T] * B, T, H, Hkv, hd, "bf16", "fp8", seed=16, spare=2)
    see, words = c.masks(seed=16)
    rope = ngg.Rope(hd, 512)
    x = randn(B * T, (H + 2 * Hkv) * hd, seed=17, dtype="bf16")
    lens, depth = ints(c.ctx), see.sum(-1).int() - 1
    logits = randn(B * T, 1000, seed=18)
    at = torch.arange(T, device="cuda", dtype=torch.int32)

    def step():
        pos = (lens[:, None] + depth).flatten().int()
        place = lens[:, None] + at
        slots = (torch.gather(c.table, 1, (place // 32).long()) * 32 + place % 32).flatten().int()
        q, k, v = (x[:, a:b].unflatten(1, (-1, hd)) for a, b in ((0, H * hd), (H * hd, (H + Hkv) * hd), ((H + Hkv) * hd, x.shape[1])))
        q = ngg.rotary(rope, pos, q)
        c.kv.write(k, v, slots, rope=rope, positions=pos)
        out, lse = ngg.tree_attention(q.view(B, T, H, hd), c.kv, c.table, lens, mask=words, want_lse=True)
        back = c.kv.read(slots)
        r = ngg.token_logprobs(logits, slots % 1000, top_n=4)
        return [out, lse, *back, *r]

    eager = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    q = c.q.clone()
    side.wait_stream(torch.cuda.current_stream())
    named = ngg.tree_attention(q, c.kv, c.table, lens, mask=words, stream=side)
    del q                                                              # its memory must stay until the call is done
    side.synchronize()
    assert torch.equal(named, ngg.tree_attention(c.q, c.kv, c.table, lens, mask=words))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for shift in (0, 3, -20, 0):
        lens.copy_(ints([100 + shift, 37 + shift]))
        x.copy_(randn(*x.shape, seed=30 + shift, dtype="bf16"))
        logits.copy_(randn(*logits.shape, seed=40 + shift))
        kept = [t.clone() for t in (c.kv.k_bytes, c.kv.v_bytes, c.kv.k_exps, c.kv.v_exps)]
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        for t, was in zip((c.kv.k_bytes, c.kv.v_bytes, c.kv.k_exps, c.kv.v_exps), kept):
            t.copy_(was)
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("wide", [False, True])
def test_tree_attention_repeats_itself(wide):
    c = Case([3000, 100, 900], [40, 11, 33], 40, 8, 2, 128, "bf16", "fp8", page=64, seed=19, wide=wide)
    see, words = c.masks(seed=19)
    a = c.check(words, see)
    for _ in range(5):
        b = ngg.tree_attention(c.q, c.kv, c.table, ints(c.ctx), mask=words, tree_lens=ints(c.trees), want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_tree_attention_refuses_on_the_host():
    c = Case([10], [2], 2, 4, 2, 64, "bf16", seed=20)
    call = lambda **kw: ngg.tree_attention(**{**dict(q=c.q, kv=c.kv, pages=c.table, context_lens=ints([10])), **kw})
    for exc, kw in ((ngg.NggError, dict(q=c.q[:, :, :3])), (ngg.NggError, dict(q=c.q.float())), (TypeError, dict(q=c.q.half())),
                    (ValueError, dict(q=c.q[..., :32])), (TypeError, dict(pages=c.table.long())), (TypeError, dict(context_lens=ints([1, 2]))),
                    (TypeError, dict(mask=torch.zeros(2, 2, dtype=torch.int64, device="cuda"))), (TypeError, dict(tree_lens=ints([1, 1]))),
                    (ValueError, dict(out=torch.empty(1, 2, 4, 32, dtype=torch.bfloat16, device="cuda"))), (ngg.NggError, dict(scale=-1.0)),
                    (ValueError, dict(q=c.q.transpose(2, 3).contiguous().transpose(2, 3))), (ValueError, dict(q=c.q.cpu())),
                    (TypeError, dict(workspace=torch.empty(64, device="cuda")))):
        with pytest.raises(exc):
            call(**kw)
    with pytest.raises(ValueError):
        ngg.tree_attention(c.q, c.kv, c.table.cpu(), ints([10]))


# ---- log probabilities --------------------------------------------------------------------------------------------------

def score64(x, targets, top, scale):
    x = x.double().cpu().numpy() * np.float32(scale).astype(np.float64)
    n, V = x.shape
    lse, ent = np.zeros(n), np.zeros(n)
    lp = np.zeros(targets.shape) if targets is not None else None
    ids, tlp = np.zeros((n, top), np.int32), np.zeros((n, top))
    for r in range(n):
        row = x[r]
        bad = np.isnan(row).any() or (row == INF).any()
        m = row.max()
        fin = row[row > -INF]
        if bad:
            lse[r] = ent[r] = NAN
        elif not len(fin):
            lse[r], ent[r] = -INF, 0.0
        else:
            p = np.exp(fin - m)
            lse[r] = m + np.log(p.sum())
            ent[r] = np.log(p.sum()) - (p * (fin - m)).sum() / p.sum()
        one = lambda v: NAN if bad else row[v] - lse[r] if row[v] > -INF else -INF
        order = np.lexsort((np.arange(V), -np.where(np.isnan(row), 0, row), ~np.isnan(row)))[:top]
        ids[r], tlp[r] = order, [one(v) for v in order]
        if lp is not None:
            lp[r] = [0.0 if v < 0 else NAN if v >= V else one(v) for v in targets[r]]
    return lp, ent, lse, ids, tlp


def check_scores(x, targets=None, top=0, scale=1.0):
    got = ngg.token_logprobs(x, None if targets is None else ints(targets), top_n=top, scale=scale)
    lp, ent, lse, ids, tlp = score64(x, None if targets is None else np.asarray(targets).reshape(x.shape[0], -1), top, scale)
    # x * scale is rounded (2^-24 of itself, of the values that have a share); sums of V terms in V / 64 steps per lane and some more
    y = x.double().cpu().numpy() * scale
    top_of = np.where(np.isfinite(y), y, -INF).max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        big = np.where(np.isfinite(y) & (y > top_of - 110), np.abs(y), 0.0).max(1)
    tol = 2.0 ** -22 * (big + 4) + (x.shape[1] / 64 + 64) * 2.0 ** -24
    listed = np.where(np.isfinite(y), np.abs(y), 0.0).max(1, keepdims=True) * 2.0 ** -22 + tol[:, None]

    def close(g, w, t, what):
        g = g.double().cpu().numpy().reshape(w.shape)
        with np.errstate(invalid="ignore"):
            same = (np.isnan(g) & np.isnan(w)) | (g == w) | (np.abs(g - w) <= t)
        assert same.all(), (what, g[~same][:5], w[~same][:5], t)
    close(got.lse, lse, tol, "lse")
    close(got.entropy, ent, tol * (2 + 2 * np.minimum(big, 100.0)), "entropy")
    if targets is not None:
        close(got.logprobs, lp, listed, "logprobs")
        assert got.logprobs.shape == torch.Size(np.shape(targets))
    else:
        assert got.logprobs is None
    if top:
        assert (got.top_ids.cpu().numpy() == ids).all()
        close(got.top_logprobs, tlp, listed, "top_logprobs")
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,top,m", [(1, 1, 1, 1), (1, 2, 2, 3), (3, 7, 5, 1), (2, 64, 64, 0), (5, 255, 20, 4), (1, 512, 1, 1), (4, 1000, 0, 2), (2, 1023, 64, 1),
                                       (7, 8192, 5, 1), (1, 32000, 20, 2), (33, 4097, 8, 1), (2, 50001, 32, 64), (1, 128256, 64, 1), (300, 700, 3, 1), (3, 130001, 10, 0)])
def test_token_logprobs(dtype, n, V, top, m):
    x = (randn(n, V, seed=V + n) * 3).to(DT[dtype])
    rng = np.random.default_rng(V)
    check_scores(x, rng.integers(0, V, (n, m)) if m else None, top, 1.0)
    check_scores(x, rng.integers(0, V, (n, m)) if m else None, top, 0.37)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 5000, 40003])
def test_token_logprobs_orders_that_are_hard(dtype, V):
    """Rising, falling, all equal, few values with many ties, one giant, and everything at the type's lowest value."""
    up = torch.arange(V, dtype=torch.float32) / V * 20 - 10
    few = torch.randint(0, 3, (V,), generator=torch.Generator().manual_seed(1)).float()
    giant = torch.randn(V, generator=torch.Generator().manual_seed(2))
    giant[V // 2] = 1000.0
    low = torch.full((V,), torch.finfo(DT[dtype]).min)
    spot = low.clone()
    spot[V - 1] = 0.5
    zeros = torch.zeros(V)
    zeros[::2] = -0.0                                                   # equal to 0.0: ties by id
    blocks = torch.zeros(V)
    blocks[-40:] = 1.0
    x = torch.stack([up, up.flip(0), torch.full((V,), 2.5), few, giant, spot, zeros, blocks]).to(DT[dtype]).cuda()
    check_scores(x, np.tile([[0, V - 1, V // 2]], (8, 1)), min(64, V), 1.0)
    got = ngg.token_logprobs(low[None].to(DT[dtype]).cuda(), top_n=3)
    assert got.top_ids.tolist() == [[0, 1, 2]] and abs(float(got.entropy) - math.log(V)) < 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [9, 300, 33000])
def test_token_logprobs_not_finite(dtype, V):
    x = randn(8, V, seed=V).to(DT[dtype])
    x[0] = -INF
    x[1, :-1] = -INF
    x[2, 3] = NAN
    x[3, V - 2] = INF
    x[4, ::2] = -INF
    x[5, 0], x[5, V - 1], x[5, 4] = NAN, NAN, INF
    x[6, 5:] = -INF
    check_scores(x, [[0, V - 1, -1, V, -5]] * 8, min(V, 12), 1.5)


def test_token_logprobs_rows_with_strides_and_offsets():
    n, V = 6, 777
    for dtype in ("f32", "bf16"):
        big = (randn(n, 2 * V + 11, seed=5) * 2).to(DT[dtype])
        for at in (0, 1, 3, 8):
            x = big[:, at:at + V]
            got, want = ngg.token_logprobs(x, ints([3] * n), top_n=9), ngg.token_logprobs(x.contiguous(), ints([3] * n), top_n=9)
            for g, w in zip(got, want):
                assert torch.allclose(g, w, rtol=2.0 ** -20, atol=2.0 ** -20)
            assert torch.equal(got.top_ids, want.top_ids)
            check_scores(x, [3] * n, 9)
        one = big[:1, :V].expand(4, -1)
        got = ngg.token_logprobs(one, top_n=2)
        assert (got.lse == got.lse[0]).all()
    r = ngg.token_logprobs(big[:0, :V], ints(np.zeros((0, 2))), top_n=2)
    assert r.logprobs.shape == (0, 2) and r.top_ids.shape == (0, 2)


def test_token_logprobs_rows_beyond_32_bits():
    V = 131072
    n = (1 << 31) // V + 2
    x = torch.zeros(n, V, dtype=torch.bfloat16, device="cuda")
    x[-1, V - 1] = 9.0
    x[-2, 5] = 8.0
    r = ngg.token_logprobs(x, torch.full((n,), V - 1, dtype=torch.int32, device="cuda"), top_n=1)
    assert r.top_ids[-1, 0] == V - 1 and r.top_ids[-2, 0] == 5 and r.top_ids[0, 0] == 0
    assert abs(float(r.lse[-1]) - math.log(math.exp(9.0) + V - 1)) < 1e-4
    repeat = ngg.token_logprobs(x, torch.full((n,), V - 1, dtype=torch.int32, device="cuda"), top_n=1)
    assert all(torch.equal(a, b) for a, b in zip(r, repeat))


def test_token_logprobs_refuses_on_the_host():
    x = randn(3, 50)
    for exc, args, kw in ((TypeError, (x.double(),), {}), (TypeError, (x, torch.zeros(3, device="cuda")), {}), (TypeError, (x, ints([1, 2])), {}),
                          (ngg.NggError, (x,), dict(top_n=51)), (ngg.NggError, (x,), dict(scale=0.0)), (ValueError, (x.T,), {}),
                          (RuntimeError, (x.cpu(),), {})):
        with pytest.raises(exc):
            ngg.token_logprobs(*args, **kw)
