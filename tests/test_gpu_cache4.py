"""A paged cache held in 4 bits on the GPU, and the attention that reads it, against plain implementations in 64 bits.  Needs an MI355X.

What is cached is exact: the nearest of eight magnitudes times a power of two.  Attention is held to what the formats allow (check4).
"""
import numpy as np
import pytest
import torch

import paper_2411_03786_amd as ngg
from test_gpu_operators import Case, attention64, ints, randn

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN, INF = float("nan"), float("inf")
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def four_bits(x):
    """x [..., hd] -> its values in 4 bits: of every 32 the power of two by trying them all, the nearest magnitude (ties to the even code)."""
    shape = x.shape
    x = x.double().cpu().numpy().reshape(-1, 32)
    fin = np.isfinite(x).all(-1, keepdims=True)
    y = np.where(fin, x, 0.0)
    top = np.abs(y).max(-1, keepdims=True)
    e = np.full_like(top, -126.0)
    for k in range(-126, 127):
        e = np.where(6.0 * 2.0 ** k < top, k + 1.0, e)
    e = np.where(top > 0, e, 0.0)
    m = np.abs(y) / 2.0 ** e
    hi = np.clip(np.searchsorted(GRID, m), 0, 7)
    lo = np.maximum(hi - 1, 0)
    up = (GRID[hi] - m < m - GRID[lo]) | ((GRID[hi] - m == m - GRID[lo]) & (hi % 2 == 0))
    val = np.where(up, GRID[hi], GRID[lo]) * np.sign(y) * 2.0 ** e
    big = np.abs(val) >= 2.0 ** 128
    val[big] = np.sign(val[big]) * INF
    return torch.from_numpy(np.where(fin, val, NAN).reshape(shape)).cuda()


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=-77.0, posinf=1e300, neginf=-1e300), torch.nan_to_num(b.double(), nan=-77.0, posinf=1e300, neginf=-1e300))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,Hkv,page", [(32, 4, 32), (64, 3, 96), (128, 8, 64), (64, 90, 32), (32, 200, 64), (128, 200, 32), (128, 1, 160)])
@pytest.mark.parametrize("n,order", [(1, "run"), (5, "run"), (32, "run"), (61, "run"), (200, "run"), (97, "shuffled"), (130, "halves")])
def test_cache_holds_what_was_written(dtype, hd, Hkv, page, n, order):
    pool = 300 // page + 3
    kv = ngg.KVPages(pool, page, Hkv, hd, "fp4")
    rng = np.random.default_rng(n * hd)
    slots = 13 + np.arange(n)
    if order == "shuffled":
        slots = rng.permutation(pool * page)[:n]
    if order == "halves":                                              # two sequences' runs, one of them backwards
        slots = np.concatenate([100 + np.arange(n // 2), 99 - np.arange(n - n // 2)]).clip(0)
        slots = np.unique(slots)[::-1].copy()
        n = len(slots)
    size = torch.where(torch.rand(n, 1, generator=torch.Generator().manual_seed(1)) < 0.3, 1000.0, 0.1).cuda().to(DT[dtype])
    x = randn(n, 3 * Hkv * hd, seed=n, dtype=dtype) * size
    k, v = x[:, Hkv * hd:2 * Hkv * hd].view(n, Hkv, hd), x[:, 2 * Hkv * hd:].view(n, Hkv, hd)
    old_k, old_v = (randn(pool * page, Hkv, hd, seed=s, dtype=dtype) for s in (8, 9))
    kv.write(old_k, old_v, ints(np.arange(pool * page)))
    kv.write(k, v, ints(slots))
    want_k, want_v = four_bits(old_k), four_bits(old_v)
    at = torch.from_numpy(slots).cuda()
    want_k[at], want_v[at] = four_bits(k), four_bits(v)
    for order2 in (np.arange(pool * page), rng.permutation(pool * page)[:77], slots):
        o = torch.from_numpy(order2).cuda()
        for out in ("f32", "bf16"):                                     # (the values fit either)
            got_k, got_v = kv.read(ints(order2), DT[out])
            assert torch.equal(got_k.double(), want_k[o]) and torch.equal(got_v.double(), want_v[o])
    # writing what was read changes no value
    kv.write(*kv.read(ints(slots), DT[dtype]), ints(slots))
    again = kv.read(ints(np.arange(pool * page)), DT[dtype])
    assert torch.equal(again[0].double(), want_k) and torch.equal(again[1].double(), want_v)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,Hkv", [(32, 5), (64, 3), (128, 2)])
@pytest.mark.parametrize("tree,start", [(61, 0), (13, 5), (8, 8), (9, 7), (3, 30), (40, 1)])
def test_cache_of_many_sequences_runs(dtype, hd, Hkv, tree, start):
    """Runs of slots that begin and end inside tiles, with places left out, as one call and in pieces."""
    B, page = 20 + 1200 // tree, 64
    rng = np.random.default_rng(tree)
    slots = np.concatenate([(2 * page * b + start + 3 * (b % 5) + np.arange(tree)) for b in rng.permutation(B)])
    slots[rng.permutation(len(slots))[:5]] = -1
    n, pool = len(slots), 2 * B + 2
    x = randn(n, 2 * Hkv * hd, seed=tree, dtype=dtype)
    k, v = x[:, :Hkv * hd].view(n, Hkv, hd), x[:, Hkv * hd:].view(n, Hkv, hd)
    whole, parts = (ngg.KVPages(pool, page, Hkv, hd, "fp4") for _ in range(2))
    whole.write(k, v, ints(slots))
    for at in range(0, n, 50):
        parts.write(k[at:at + 50], v[at:at + 50], ints(slots[at:at + 50]))
    for name in ("k_bytes", "v_bytes", "k_exps", "v_exps"):
        assert torch.equal(getattr(whole, name), getattr(parts, name)), name
    got = whole.read(ints(slots), DT[dtype])
    there = torch.from_numpy(slots >= 0).cuda()
    for g, t in zip(got, (k, v)):
        assert torch.equal(g[there].double(), four_bits(t)[there]) and (g[~there] == 0).all()
    some = whole.read(ints(slots[:100]), DT[dtype])
    assert torch.equal(some[0], got[0][:100]) and torch.equal(some[1], got[1][:100])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,Hkv,n,gap", [(32, 301, 470, 0), (32, 301, 470, 3), (64, 150, 300, 0), (128, 33, 900, 0)])
def test_cache_of_many_heads(dtype, hd, Hkv, n, gap):
    """More heads than a workgroup takes at once, with an odd number left over; runs, single places and places left out."""
    rng = np.random.default_rng(n)
    slots = np.concatenate([5 + np.arange(n // 2), n + 40 + rng.permutation(n)[:n - n // 2]])
    slots[[3, n - 1]] = -1
    kv = ngg.KVPages(2 * n // 32 + 3, 32, Hkv, hd, "fp4")
    x = randn(n, 2 * Hkv * hd + gap, seed=n, dtype=dtype)
    k, v = x[:, gap:gap + Hkv * hd].view(n, Hkv, hd), x[:, gap + Hkv * hd:].view(n, Hkv, hd)
    kv.write(k, v, ints(slots))
    there = torch.from_numpy(slots >= 0).cuda()
    for out in ("f32", "bf16"):
        for g, t in zip(kv.read(ints(slots), DT[out]), (k, v)):
            assert torch.equal(g[there].double(), four_bits(t)[there]) and (g[~there] == 0).all()


def test_four_bit_corners():
    """Zeros, the largest value exactly and just above, every tie, the smallest and largest exponents, numbers that are not finite; each
    32 dimensions by themselves."""
    rows = torch.zeros(13, 1, 64)
    rows[1, 0, 0] = 6.0
    rows[2, 0, :2] = torch.tensor([6.0000005, 1.0])
    rows[3, 0, :32] = torch.linspace(-3.4e38, 3.4e38, 32)
    rows[4, 0] = 1e-40
    rows[5, 0, :3] = torch.tensor([INF, -2.0, 3.3])
    rows[6, 0, 33:36] = torch.tensor([NAN, 1e-3, -7.0])
    rows[6, 0, :3] = torch.tensor([1.0, 2.0, -7.0])
    rows[7, 0] = -INF
    rows[8, 0, :14] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -5.0])
    rows[8, 0, 32:39] = torch.tensor([6.0, 0.2500001, 0.7499999, 1.2500001, 1.7499999, 2.5000002, 4.9999995])
    rows[9, 0] = torch.linspace(1e-38, 3e-36, 64)
    rows[10, 0, :5] = torch.tensor([1.75 * 2.0 ** 127, 2.0 ** 127, -1.7499999 * 2.0 ** 127, 1.0, -0.0])
    rows[11, 0] = torch.linspace(-1, 1, 64)
    rows[12, 0] = torch.linspace(-1e-44, 1e-44, 64)
    want = four_bits(rows)
    assert torch.isinf(want[10, 0, 0]) and want[10, 0, 1] == 2.0 ** 127
    for heads in (1, 400):
        x = rows.expand(-1, heads, -1).contiguous().cuda()
        kv = ngg.KVPages(2, 32, heads, 64, "fp4")
        slots = ints(range(20, 33))
        kv.write(x, x.flip(0).contiguous(), slots)
        k, v = (t[:, -1:] for t in kv.read(slots, torch.float32))
        assert same(k, want) and same(v, want.flip(0))


def test_every_value_of_a_16_bit_type():
    """All finite bf16 numbers, 32 with the same exponent to a group and all mixed."""
    u = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    u = u[torch.isfinite(u.float())]
    u = torch.cat([u, u[torch.randperm(len(u), generator=torch.Generator().manual_seed(1))]])
    x = u[:len(u) // 128 * 128].view(-1, 1, 128).cuda()
    n = len(x)
    kv = ngg.KVPages(n // 64 + 1, 64, 1, 128, "fp4")
    kv.write(x, x.flip(0).contiguous(), ints(np.arange(n)))
    k, v = kv.read(ints(np.arange(n)), torch.float32)
    want = four_bits(x)
    assert same(k, want) and same(v, want.flip(0))


@pytest.mark.parametrize("H", [2, 700])
def test_cache_slots_out_of_range(H):
    kv = ngg.KVPages(2, 32, H, 64, "fp4")
    x = randn(6, H, 64, seed=1, dtype="bf16")
    kv.write(x[:2], x[2:4], ints([5, 6]))
    before = [t.clone() for t in kv._memory()]
    kv.write(x[:4], x[2:6], ints([-1, 64, 2 ** 31 - 1, -2 ** 31]))
    assert all(torch.equal(a, b) for a, b in zip(before, kv._memory()))
    k, v = kv.read(ints([-1, 5, 64, 2 ** 31 - 1, 6]))
    assert (k[[0, 2, 3]] == 0).all() and (v[[0, 2, 3]] == 0).all() and (k[[1, 4]] != 0).any()
    kv.write(x, x, ints(range(61, 67)))
    kv.write(x, x, ints(range(-3, 3)))
    k2, _ = kv.read(ints([61, 62, 63, 0, 1, 2]))
    assert torch.equal(k2.double(), four_bits(x))
    kv.write(x[:0], x[:0], ints([]))
    assert kv.read(ints([]))[0].shape == (0, H, 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gap", [0, 1, 2, 8])
@pytest.mark.parametrize("n", [3, 400])
def test_cache_takes_rows_with_strides(dtype, gap, n):
    Hkv, hd = 3, 64
    big = randn(n, Hkv, 2 * hd + gap, seed=gap, dtype=dtype)
    k, v = big[..., gap:gap + hd], big[..., gap + hd:].transpose(0, 1).contiguous().transpose(0, 1)
    kv = ngg.KVPages(n // 32 + 1, 32, Hkv, hd, "fp4")
    kv.write(k, v, ints(np.arange(n)))
    got = kv.read(ints(np.arange(n)), DT[dtype])
    assert torch.equal(got[0].double(), four_bits(k)) and torch.equal(got[1].double(), four_bits(v))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,rd,inter", [(32, 32, False), (64, 32, True), (128, 128, True), (128, 128, False), (128, 34, False), (64, 6, True)])
@pytest.mark.parametrize("Hkv,n", [(3, 75), (120, 75), (203, 700)])
def test_cache_rotates_as_rotary_does(dtype, hd, rd, inter, Hkv, n):
    rope, pos = ngg.Rope(rd, 300, interleaved=inter), ints(np.random.default_rng(2).integers(0, 300, n))
    pos[3] = 300                                                        # behind the table: NaN
    x = randn(n, 2 * Hkv * hd + 2, seed=hd, dtype=dtype)
    k, v = x[:, :Hkv * hd].view(n, Hkv, hd), x[:, Hkv * hd:2 * Hkv * hd].view(n, Hkv, hd)
    a, b = (ngg.KVPages(23, 32, Hkv, hd, "fp4") for _ in range(2))
    slots = ints(7 + np.arange(n))
    a.write(k, v, slots, rope=rope, positions=pos)
    b.write(ngg.rotary(rope, pos, k), v, slots)
    assert all(torch.equal(s, t) for s, t in zip(a._memory(), b._memory()))
    assert torch.isnan(a.read(slots)[0][3, :, :min(32, rd)]).all()


def test_cache_beyond_32_bits_of_bytes():
    """The last pages of a pool whose keys alone pass 2^32 bytes."""
    Hkv, hd, page = 8, 128, 256
    pool = (1 << 32) // (Hkv * hd * page // 2) + 3
    kv = ngg.KVPages(pool, page, Hkv, hd, "fp4")
    n = 100
    k, v = randn(n, Hkv, hd, seed=1, dtype="bf16"), randn(n, Hkv, hd, seed=2, dtype="bf16")
    slots = ints((pool - 1) * page + np.arange(n))
    kv.write(k, v, slots)
    got = kv.read(slots)
    assert torch.equal(got[0].double(), four_bits(k)) and torch.equal(got[1].double(), four_bits(v))
    q = randn(1, 1, Hkv, hd, seed=3, dtype="bf16")
    out, lse = ngg.tree_attention(q, kv, ints([[pool - 1]]), ints([n - 1]), want_lse=True)
    check4(out, lse, q, [got[0]], [got[1]], [n - 1], [1], None, hd ** -0.5, "bf16")
    kv.move(slots[:3], slots[:3] - 2 * page)
    moved = kv.read(slots[:3] - 2 * page)
    assert torch.equal(moved[0], got[0][:3]) and torch.equal(moved[1], got[1][:3])
    kv.copy(ints([pool - 1]), ints([pool - 2]), ints([n]))
    moved = kv.read(slots - page)
    assert torch.equal(moved[0], got[0]) and torch.equal(moved[1], got[1])
    assert not kv.k_bytes[:1 << 20].any()


# ---- attention --------------------------------------------------------------------------------------------------------

def check4(out, lse, q, ks, vs, ctx, trees, see, scale, dtype):
    """Scores: fp32 sums of head_dim products, off by (head_dim + 10) 2^-24 of the sum of |q k| (2 2^-24 of it where fp32 queries are
    taken apart).  Outputs: twice that in a quotient of sums, 2^-15 for sums of up to 10^5
    terms in up to 10^3 pieces, the result's rounding, and, for bf16, 2^-8 of the sum of p |v| (a probability rounded to bf16)."""
    want, want_lse, mag, qk = attention64(q, ks, vs, ctx, trees, see, scale)
    hd = q.shape[-1]
    err = (hd + 10) * 2.0 ** -24 * qk
    tol = mag * (2 * err + 2.0 ** -15 + (2.0 ** -8 if dtype == "bf16" else 0))[..., None] + want.abs() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) + 1e-30
    assert torch.isfinite(out).all()
    bad = (out.double() - want).abs() > tol
    assert not bad.any(), ((out.double() - want).abs() / tol).max()
    dead = want_lse == -INF
    assert (lse[dead] == -INF).all() and (out[dead] == 0).all()
    assert ((lse.double() - want_lse).abs()[~dead] <= (err + 2.0 ** -15 + 2.0 ** -22 * want_lse.abs())[~dead]).all()


class Case4(Case):
    """As there, in 4 bits, with all bits set in the places that nobody wrote."""

    def __init__(self, ctx, trees, T, H, Hkv, hd, dtype="bf16", page=32, **more):
        super().__init__(ctx, trees, T, H, Hkv, hd, dtype, "fp4", page, **more)
        for t in self.kv._memory():
            t.fill_(255)
        for b, (k, v) in enumerate(zip(self.ks, self.vs)):
            pos = torch.arange(len(k), device="cuda")
            self.kv.write(k, v, (self.table[b, pos // page] * page + pos % page).int())

    def check(self, words=None, see=None, **more):
        lens = ints(self.trees) if self.trees != [self.T] * len(self.trees) else None
        out, lse = ngg.tree_attention(self.q, self.kv, self.table, ints(self.ctx), mask=words, tree_lens=lens, want_lse=True, **more)
        check4(out, lse, self.q, self.ks, self.vs, self.ctx, self.trees, see, self.scale, self.dtype)
        return out, lse


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,hd", [(4, 4, 32), (6, 2, 64), (8, 2, 128), (3, 3, 128)])
@pytest.mark.parametrize("T,ctx", [(1, 0), (1, 1), (1, 31), (1, 300), (2, 127), (5, 0), (13, 128), (17, 65), (33, 200), (65, 97), (70, 1000)])
@pytest.mark.parametrize("wide", [False, True])
def test_one_sequence(dtype, H, Hkv, hd, T, ctx, wide):
    c = Case4([ctx], [T], T, H, Hkv, hd, dtype, seed=T + ctx, wide=wide)
    see, words = c.masks(seed=T)
    c.check(words, see)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("page", [32, 64, 160])
@pytest.mark.parametrize("wide", [False, True])
def test_ragged_batch(dtype, hd, page, wide):
    ctx = [0, 1, 31, 32, 33, 500, 1999, 64, 5]
    trees = [3, 19, 0, 19, 1, 7, 18, 19, 2]
    c = Case4(ctx, trees, 19, 8, 2, hd, dtype, page=page, seed=3, wide=wide)
    see, words = c.masks(seed=4)
    c.check(words, see)
    c.check(None, None)                                                 # a chain each
    c.check(words[0].contiguous(), see[:1].expand(len(ctx), -1, -1))    # one tree for all


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_short_sequences(dtype):
    rng = np.random.default_rng(5)
    ctx = [int(x) for x in rng.integers(0, 90, 70)]
    Case4(ctx, [1] * 70, 1, 4, 1, 32, dtype, seed=6).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,hd,T,ctx", [(4, 1, 128, 64, 3000), (2, 2, 64, 150, 513), (8, 1, 32, 33, 700), (1, 1, 128, 300, 100)])
@pytest.mark.parametrize("wide", [False, True])
def test_wide_trees(dtype, H, Hkv, hd, T, ctx, wide):
    """More rows than a tile, masks of several words."""
    c = Case4([ctx, ctx // 3], [T, T - 5], T, H, Hkv, hd, dtype, page=64, seed=T, wide=wide)
    see, words = c.masks(seed=T + 1)
    c.check(words, see)
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_context(dtype):
    c = Case4([40000, 9, 17001], [6, 6, 6], 6, 4, 1, 64, dtype, page=256, seed=8)
    see, words = c.masks(seed=8)
    c.check(words, see)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,hd,T", [(4, 2, 128, 1), (8, 1, 64, 2), (3, 3, 32, 13), (16, 1, 128, 1)])
def test_page_lists_beyond_the_caches(dtype, H, Hkv, hd, T):
    ctx = [0, 1000, 63]
    c = Case4(ctx, [T] * 3, T, H, Hkv, hd, dtype, seed=hd + T)
    room = (1 << 30) // (hd * Hkv * 3)                                  # positions, half a byte an element of keys and of values
    c.table = torch.cat([c.table, torch.full((3, room // 32), -1, dtype=torch.int32, device="cuda")], 1)
    see, words = c.masks(seed=8)
    c.check(words, see)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
def test_sharp_scores(dtype, wide):
    """Scores in the hundreds: the running maximum moves, and single keys carry rows."""
    c = Case4([700, 33], [20, 20], 20, 4, 2, 128, dtype, seed=9, sharp=30.0, wide=wide)
    see, words = c.masks(seed=9)
    c.check(words, see)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("wide", [False, True])
def test_queries_of_many_sizes(dtype, hd, wide):
    """Rows whose elements lie far apart, rows of zeros, tiny rows and huge ones (with keys that make up for it)."""
    T = 24
    c = Case4([300], [T], T, 4, 2, hd, dtype, seed=22, wide=wide)
    far = torch.exp2(torch.randint(-18, 3, c.q.shape, generator=torch.Generator().manual_seed(3)).float()).cuda()
    c.q = (c.q.float() * far).to(DT[dtype])
    c.q[:, 3] = 0
    c.q[:, 4] *= 2.0 ** -60
    c.q[:, 5] *= 2.0 ** -120
    c.q[:, 6, :, 1:] = 0
    c.check()
    c.q[:] = randn(*c.q.shape, seed=5, dtype=dtype) * 2.0 ** 40
    c.scale = 2.0 ** -42
    c.check(scale=c.scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
def test_rows_that_see_nothing(dtype, wide):
    c = Case4([0, 40], [9, 9], 9, 8, 2, 64, dtype, seed=10, wide=wide)
    see, words = c.masks(seed=10, empty=(0, 4, 8))
    c.check(words, see)
    Case4([-5, 0], [0, 4], 4, 4, 2, 64, dtype, seed=10).check()         # a sequence that is not there


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [NAN, INF, -INF, 3.2e38])
@pytest.mark.parametrize("wide", [False, True])
def test_masked_numbers_that_are_not_finite(dtype, bad, wide):
    """One tree token's key, then another's value, is not finite (the last: as it is read): the rows that do not see it are as they were."""
    T, ctx = 21, 50
    c = Case4([ctx], [T], T, 4, 2, 64, dtype, seed=11, wide=wide)
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
        if which == "v":
            assert not torch.isfinite(out[0, hit][..., 3]).any()
            if not abs(bad) < INF:                                      # the 32 are NaN
                assert torch.isnan(out[0, hit][..., :32]).all()
            assert torch.equal(out[0, hit][..., 32:], clean[0, hit][..., 32:])
        c.kv.write(c.ks[0][ctx + j:ctx + j + 1].contiguous(), c.vs[0][ctx + j:ctx + j + 1].contiguous(), slot[None].int())
    assert torch.equal(ngg.tree_attention(c.q, c.kv, c.table, ints([ctx]), mask=words), clean)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wide,T", [(False, 5), (True, 40)])
def test_a_bad_number_in_the_context_reaches_every_row(dtype, wide, T):
    c = Case4([100], [T], T, 2, 2, 64, dtype, seed=12, wide=wide)
    k, v = c.ks[0][10:11].clone(), c.vs[0][10:11].clone()
    v[..., 0] = NAN
    c.kv.write(k, v, (c.table[0, 0] * 32 + 10)[None].int())
    out = ngg.tree_attention(c.q, c.kv, c.table, ints([100]))
    assert torch.isnan(out[..., :32]).all() and torch.isfinite(out[..., 32:]).all()
    k[..., 40] = NAN
    c.kv.write(k, c.vs[0][10:11].contiguous(), (c.table[0, 0] * 32 + 10)[None].int())
    assert torch.isnan(ngg.tree_attention(c.q, c.kv, c.table, ints([100]))).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H", [4, 24])
@pytest.mark.parametrize("T,wide", [(3, False), (40, True)])
def test_pages_and_lengths_out_of_range(dtype, H, T, wide):
    """A page outside the pool hides its positions; lengths past the page list are cut."""
    ctx = 150
    c = Case4([ctx], [T], T, H, 2, 64, dtype, seed=13, spare=0, wide=wide)
    keep = torch.cat([torch.arange(64), torch.arange(96, ctx + T)]).cuda()
    for wrong in (-1, c.kv.n_pages, 2 ** 31 - 1, -2 ** 31):
        t = c.table.clone()
        t[0, 2] = wrong                                                 # positions 64 .. 95
        out, lse = ngg.tree_attention(c.q, c.kv, t, ints([ctx]), want_lse=True)
        check4(out, lse, c.q, [c.ks[0][keep]], [c.vs[0][keep]], [ctx - 32], [T], None, c.scale, dtype)
    out, lse = ngg.tree_attention(c.q, c.kv, torch.full_like(c.table, -1), ints([ctx]), want_lse=True)
    assert (out == 0).all() and (lse == -INF).all()
    short = c.table[:, :4]                                              # 128 positions of the context, none of the tree
    see = torch.zeros(1, T, T, dtype=torch.bool, device="cuda")
    pad = [torch.cat([t[0][:128], t[0][:T]]) for t in (c.ks, c.vs)]
    for long in (ctx, 10 ** 6, 2 ** 31 - 1):
        out, lse = ngg.tree_attention(c.q, c.kv, short, ints([long]), want_lse=True)
        check4(out, lse, c.q, pad[:1], pad[1:], [128], [T], see, c.scale, dtype)
    out = ngg.tree_attention(c.q, c.kv, c.table, ints([ctx]), tree_lens=ints([2 ** 31 - 1]))
    assert torch.equal(out, ngg.tree_attention(c.q, c.kv, c.table, ints([ctx])))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("T,wide", [(5, False), (20, True)])
def test_strides(dtype, hd, T, wide):
    """Queries and outputs as slices of something larger, at odd offsets, and a page list with a stride."""
    B, H, Hkv = 3, 4, 2
    c = Case4([40, 7, 130], [T] * 3, T, H, Hkv, hd, dtype, seed=15, wide=wide)
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
    c.scale = 0.3
    c.check(scale=0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_four_bits_attend_as_the_same_values_in_16(dtype):
    """The 4-bit cache and one that holds its values as they are give the same but for the order of sums."""
    c = Case4([900, 333], [30, 17], 30, 8, 2, 128, dtype, seed=23)
    see, words = c.masks(seed=1)
    out, _ = c.check(words, see)
    kv = ngg.KVPages(c.kv.n_pages, 32, 2, 128, dtype)
    for b in range(2):
        pos = torch.arange(len(c.ks[b]), device="cuda")
        kv.write(c.ks[b], c.vs[b], (c.table[b, pos // 32] * 32 + pos % 32).int())
    other = ngg.tree_attention(c.q, kv, c.table, ints(c.ctx), mask=words, tree_lens=ints(c.trees))
    # both are within check4's bound of the true value; the outputs are means of some values of up to 5
    assert (out.float() - other.float()).abs().max() < (5 * 2.0 ** -6 if dtype == "bf16" else 5 * 2.0 ** -12)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
def test_repeats_itself(dtype, wide):
    c = Case4([3000, 100, 900], [40, 11, 33], 40, 8, 2, 128, dtype, page=64, seed=19, wide=wide)
    see, words = c.masks(seed=19)
    a = c.check(words, see)
    for _ in range(5):
        b = ngg.tree_attention(c.q, c.kv, c.table, ints(c.ctx), mask=words, tree_lens=ints(c.trees), want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_refuses_on_the_host():
    c = Case4([10], [2], 2, 4, 2, 64, "bf16", seed=20)
    call = lambda **kw: ngg.tree_attention(**{**dict(q=c.q, kv=c.kv, pages=c.table, context_lens=ints([10])), **kw})
    for exc, kw in ((ngg.NggError, dict(q=c.q[:, :, :3])), (TypeError, dict(q=c.q.half())), (ValueError, dict(q=c.q[..., :32])),
                    (RuntimeError, dict(q=c.q.clone().requires_grad_()))):
        with pytest.raises(exc):
            call(**kw)
    assert call(q=c.q.float()).dtype == torch.float32                   # either type of queries
