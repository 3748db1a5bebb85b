"""Attention over a cache of 4 bits by what a launch is planned as: tiles of 16, 32 and 128 rows; lists that go whole, in pieces and in shares.  The
plan shows in the workspace that a call asks for, which every test here checks, so that another rule cannot leave a kernel untested.  And the
bits that the kernels keep: bounds that a kernel with a bfloat16 term less would miss, which is shown beside them.  Needs an MI355X."""
import ctypes as C
import threading

import numpy as np
import pytest
import torch

import paper_2411_03786_amd as ngg
import test_gpu_cache4
from test_gpu_cache4 import Case4
from test_gpu_operators import ints, randn

pytestmark = pytest.mark.gpu


def workspace(c):
    """Bytes that the call of a Case4 asks for."""
    B, T, H, hd = c.q.shape
    a = ngg.ngg_tree_args(max_pages=c.table.shape[1], batch=B, tree=T, n_heads=H, dtype=ngg.NGG_F32 if c.dtype == "f32" else ngg.NGG_BF16, scale=1.0)
    need = C.c_int64(-1)
    assert ngg.load_library().ngg_tree_attention_workspace(c.kv._c, a, need) == ngg.NGG_OK
    return need.value


def held(dtype, hd, rows):
    """Workgroups that a launch of shares is planned for."""
    wide = dtype == "f32"
    if rows == 128:
        return 512
    if rows == 32:
        return 256 * (3 if hd == 32 and not wide else 1 if hd == 128 and wide else 2)
    return 256 * ((4 if hd == 32 else 3 if hd == 64 else 2) if wide else 3 if hd == 128 else 4)


def tiles(c, rows):
    B, T, H, hd = c.q.shape
    Hkv = c.kv.n_kv_heads
    steps = -(-c.table.shape[1] * c.kv.page_size // (64 if rows == 128 else 128))
    return B * Hkv, -(-T * (H // Hkv) // rows), steps, rows * (hd * 4 + 8)


def shares(c, rows):
    """What a launch of shares asks for: two parts for each."""
    lists, Z, steps, part = tiles(c, rows)
    want = -(-held(c.dtype, c.q.shape[-1], rows) // Z)
    r = max(1, min(want, steps * lists))
    r = r if r < 8 else -(-r // 8) * 8 if r < want else r // 8 * 8
    return r * Z * 2 * part


def pieces(c, rows, n):
    """What lists in n pieces ask for."""
    lists, Z, _, part = tiles(c, rows)
    return lists * n * Z * part


def widen(c, positions):
    """A page list for so many positions: the call is planned for them."""
    more = max(-(-positions // c.kv.page_size) - c.table.shape[1], 0)
    c.table = torch.cat([c.table, torch.full((len(c.table), more), -1, dtype=torch.int32, device="cuda")], 1)


def exact(c, b, h, terms=None):
    """Sequence b's chain under head h in 64 bits: out, sum p |v| / sum p, log sum, and the largest sum of |q k|; terms: with probabilities that are
    the sum of so many bfloat16 numbers, each the rounding of what the ones before left."""
    T, H = c.T, c.q.shape[2]
    n = c.ctx[b] + c.trees[b]
    k, v = (x[b][:n, h // (H // c.kv.n_kv_heads)].double() for x in (c.ks, c.vs))
    x = c.q[b, :, h].double()
    see = torch.arange(n, device="cuda") <= c.ctx[b] + torch.arange(T, device="cuda")[:, None]
    s = torch.where(see, (x @ k.T.contiguous()) * c.scale, -float("inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    tot = p.sum(-1, keepdim=True)
    if terms:
        rest, p = p, torch.zeros_like(p)
        for _ in range(terms):
            part = rest.bfloat16().double()
            p, rest = p + part, rest - part
    qk = torch.where(see, (x.abs() @ k.abs().T.contiguous()) * abs(c.scale), 0.0).amax(-1)
    return (p @ v) / tot, (p @ v.abs()) / tot, (top + tot.log()).squeeze(-1), qk


@pytest.mark.parametrize("rows,n,H,Hkv,hd,T,positions", [(16, 0, 8, 2, 64, 3, 0), (16, 0, 4, 4, 128, 1, 0), (16, 40, 8, 2, 128, 9, 20000), (32, 61, 8, 2, 128, 9, 70000),
                                                         (32, 61, 8, 2, 64, 9, 70000), (32, 79, 8, 1, 32, 9, 70000), (128, None, 8, 2, 128, 20, 220000),
                                                         (128, None, 4, 1, 64, 33, 260000)])
def test_sixteen_bit_calls_keep_16_bits_of_a_probability(rows, n, H, Hkv, hd, T, positions):
    """Values of either sign leave little of a row's sum, so that what its terms lose is seen beside the rounding of the output.  Queries of
    four dimensions: scores off by (4 + 10) 2^-24 of the sum of |q k|, outputs by twice that; two bfloat16 terms of a probability by
    2^-8 2^-8 of it; sums of n terms, of probabilities and of both terms' products, by 3 n 2^-24; the result's rounding 2^-8 of itself.
    With one term some outputs are further off than that."""
    ctx = 60 - T
    c = Case4([ctx, ctx // 2], [T, T], T, H, Hkv, hd, "bf16", page=64, seed=31)
    widen(c, positions)
    c.q[..., 4:] = 0
    c.scale = 1.0
    assert workspace(c) == (shares(c, rows) if n is None else pieces(c, rows, n))
    out, lse = ngg.tree_attention(c.q, c.kv, c.table, ints(c.ctx), scale=1.0, want_lse=True)
    beyond = 0
    for b in range(2):
        keys = c.ctx[b] + T
        for h in range(H):
            want, mag, want_lse, qk = exact(c, b, h)
            tol = mag * (2 * (4 + 10) * 2.0 ** -24 * qk[:, None] + 2.0 ** -16 + 3 * keys * 2.0 ** -24) + want.abs() * 2.0 ** -8
            assert ((out[b, :, h].double() - want).abs() <= tol).all()
            assert ((lse[b, :, h].double() - want_lse).abs() <= (4 + 10) * 2.0 ** -24 * qk + (keys + 8) * 2.0 ** -24 + 2.0 ** -23 * want_lse.abs()).all()
            beyond += int(((exact(c, b, h, 1)[0] - want).abs() > tol).sum())
            assert ((exact(c, b, h, 2)[0] - want).abs() <= tol).all()
    assert beyond > 20


def test_calls_of_two_host_threads():
    """Tiles of 32 rows of 128 dimensions take more than 64 KB of LDS, and the more the larger the batch: two threads that call with a batch of 1 and
    of 1024, each on a stream of its own, through the C entry (which, unlike the binding, lets both in at once)."""
    lib, calls = ngg.load_library(), []
    for batch, positions in ((1, 200000), (1024, 256)):
        c = Case4([20] * min(batch, 8), [1] * min(batch, 8), 1, 32, 1, 128, "bf16", page=64, seed=batch)
        widen(c, positions)
        c.table, c.q = (x.repeat(batch // len(x), *[1] * (x.dim() - 1)).contiguous() for x in (c.table, c.q))
        assert workspace(c) == (pieces(c, 32, 391) if batch == 1 else 0)
        lens = ints([20] * batch)
        want = ngg.tree_attention(c.q, c.kv, c.table, lens)
        out, ws = torch.zeros_like(c.q), torch.empty(max(workspace(c), 16), dtype=torch.uint8, device="cuda")
        a = ngg.ngg_tree_args(q=c.q.data_ptr(), out=out.data_ptr(), q_batch=32 * 128, q_token=32 * 128, q_head=128, out_batch=32 * 128, out_token=32 * 128, out_head=128,
                              pages=c.table.data_ptr(), pages_batch=c.table.stride(0), context_lens=lens.data_ptr(), max_pages=c.table.shape[1], batch=batch, tree=1,
                              n_heads=32, dtype=ngg.NGG_BF16, scale=128 ** -0.5)
        calls.append((c, a, ws, torch.cuda.Stream(), out, want, lens))
    torch.cuda.synchronize()
    bad = []

    def many(c, a, ws, stream, *_):
        for _ in range(300):
            if lib.ngg_tree_attention(c.kv._c, a, ws.data_ptr(), ws.numel(), stream.cuda_stream) != ngg.NGG_OK:
                bad.append(lib.ngg_last_error(None).decode())
    threads = [threading.Thread(target=many, args=x) for x in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad, bad[:3]
    assert all(torch.equal(x[4], x[5]) for x in calls)


def test_the_largest_tree_of_the_most_heads():
    """1024 tokens of 1024 heads over one key head in fp32: 2^20 rows, which in tiles of 16 would be more than the joining launch can count.  (Tiles of 32,
    which no other call of heads of 128 in fp32 has.)  Every output, to the bounds of test_gpu_cache4."""
    T = H = 1024
    hd, ctx = 128, 1500
    c = Case4([ctx], [T], T, 1, 1, hd, "f32", page=64, seed=41)
    c.q = torch.randn(1, T, H, hd, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    assert workspace(c) == shares(c, 32) > 0
    out, lse = ngg.tree_attention(c.q, c.kv, c.table, ints(c.ctx), want_lse=True)
    n, at = ctx + T, torch.arange(ctx + T, device="cuda")
    k, v = (x[0][:n, 0].double() for x in (c.ks, c.vs))
    kt, kt_abs, v_abs = k.T.contiguous(), k.abs().T.contiguous(), v.abs()
    for t in range(0, T, 8):
        x = c.q[0, t:t + 8].double().flatten(0, 1)
        s = (x @ kt) * c.scale
        see = (at <= ctx + torch.arange(t, t + 8, device="cuda").repeat_interleave(H)[:, None])
        s = torch.where(see, s, -float("inf"))
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        tot = p.sum(-1, keepdim=True)
        want, want_lse = (p @ v) / tot, (top + tot.log()).squeeze(-1)
        err = (hd + 10) * 2.0 ** -24 * ((x.abs() @ kt_abs).amax(-1) * c.scale)
        tol = (p @ v_abs) / tot * (2 * err + 2.0 ** -15)[:, None] + want.abs() * 2.0 ** -24
        assert ((out[0, t:t + 8].flatten(0, 1).double() - want).abs() <= tol).all(), t
        assert ((lse[0, t:t + 8].flatten().double() - want_lse).abs() <= err + 2.0 ** -15 + 2.0 ** -22 * want_lse.abs()).all(), t


def ragged(B, T, longest, seed):
    """Lengths of all kinds: sequences that are not there, contexts of none and one, trees that are missing and short."""
    rng = np.random.default_rng(seed)
    ctx = rng.integers(longest // 2, longest - T, B)
    ctx[::7], ctx[1::11] = 0, 1
    trees = rng.integers(1, T + 1, B)
    trees[3::9], trees[0] = 0, T
    return [int(x) for x in ctx], [int(x) for x in trees]


# type, head_dim, tile rows, pieces (None: shares), sequences, query and key heads, tree, planned positions, longest list
PLANS = [
    # shares of all lists, single tokens
    ("bf16", 128, 16, None, 40, 16, 4, 2, 3000, 2900), ("f32", 64, 16, None, 40, 16, 4, 2, 3000, 2900), ("bf16", 32, 16, None, 40, 16, 4, 2, 3000, 2900),
    ("f32", 128, 16, None, 40, 16, 4, 2, 3000, 2900), ("f32", 32, 16, None, 40, 16, 4, 2, 3000, 2900), ("bf16", 64, 16, None, 40, 16, 4, 2, 3000, 2900),
    # by non-temporal loads
    ("bf16", 128, 16, None, 60, 16, 4, 1, 13500, 2000), ("f32", 32, 16, None, 80, 16, 4, 1, 41000, 2000),
    # shares, trees in tiles of 16 and 32 rows, several a tree
    ("f32", 128, 16, None, 20, 16, 4, 9, 3000, 2900), ("bf16", 64, 16, None, 20, 16, 4, 9, 1400, 1300), ("bf16", 128, 32, None, 20, 16, 4, 9, 3000, 2900),
    ("bf16", 64, 32, None, 20, 16, 4, 13, 3000, 2900), ("bf16", 32, 32, None, 20, 16, 4, 13, 3000, 2900), ("f32", 64, 32, None, 20, 16, 4, 9, 3000, 2900),
    ("f32", 32, 32, None, 20, 16, 4, 9, 12000, 2900),
    # lists in pieces that are joined: of 16 rows, by non-temporal loads, of 32 rows
    ("bf16", 128, 16, 33, 3, 4, 1, 13, 4100, 4000), ("f32", 128, 16, 36, 2, 8, 2, 9, 9000, 8900), ("bf16", 128, 16, 4, 40, 16, 4, 1, 20480, 15000),
    ("bf16", 128, 16, 253, 3, 4, 1, 2, 1100000, 40000), ("f32", 128, 16, 169, 3, 4, 1, 2, 1100000, 40000),
    ("bf16", 128, 32, 59, 2, 8, 2, 9, 45000, 9000), ("bf16", 64, 32, 59, 2, 8, 2, 9, 45000, 9000), ("f32", 64, 32, 59, 2, 8, 2, 9, 60000, 9000),
    ("f32", 32, 32, 63, 2, 8, 2, 9, 240000, 30000), ("bf16", 32, 32, 59, 2, 8, 2, 9, 45000, 9000),
    # shares of tiles of 128 rows
    ("bf16", 128, 128, None, 3, 8, 2, 20, 150016, 6000), ("bf16", 64, 128, None, 3, 8, 2, 33, 90000, 6000),
]


@pytest.mark.parametrize("plan", PLANS, ids=lambda p: "-".join(map(str, p)))
def test_plans(plan):
    """Lists that several workgroups work on, and workgroups that work on several lists."""
    dtype, hd, rows, n, B, H, Hkv, T, positions, longest = plan
    ctx, trees = ragged(B, T, longest, B)
    ctx[0 if B < 7 else 2] = longest - T
    c = Case4(ctx, trees, T, H, Hkv, hd, dtype, page=64, seed=B + T)
    widen(c, positions)
    assert workspace(c) == (shares(c, rows) if n is None else pieces(c, rows, n))
    see, words = c.masks(seed=B, empty=(T - 1,) if T > 2 else ())
    out, lse = c.check(words, see)
    again, lse2 = ngg.tree_attention(c.q, c.kv, c.table, ints(ctx), mask=words, tree_lens=ints(trees), want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,hd,T", [("bf16", 64, 1), ("f32", 32, 3), ("bf16", 128, 2)])
def test_shares_among_many_short_sequences(dtype, hd, T):
    """More sequences than a wave looks through at once, most of them of one step and some not there, between a few long ones."""
    B = 300
    ctx, trees = [17 * b % 120 for b in range(B)], [1 + b % T for b in range(B)]
    for b in (0, 60, 63, 64, 65, 127, 128, 200, 290, 299):
        ctx[b] = 2300 + b
    for b in range(130, 199):
        ctx[b], trees[b] = 0, 0
    c = Case4(ctx, trees, T, 4, 1, hd, dtype, page=32, seed=T)
    widen(c, 2700)
    assert workspace(c) == shares(c, 16)
    c.check()


class Tall(Case4):
    """As there, with four times the query heads (over 64 rows) and a page list long enough for tiles of 128 rows."""

    def __init__(self, ctx, trees, T, H, Hkv, hd, dtype="bf16", page=32, **more):
        super().__init__(ctx, trees, T, 4 * H, Hkv, hd, dtype, page=page, **{**more, "wide": False})
        widen(self, -(-(64 << 20) // (T * 4 * H * len(ctx))))
        assert workspace(self) == shares(self, 128)


@pytest.mark.parametrize("call", [
    *[(name, dict(T=T, ctx=ctx, H=H, Hkv=Hkv, hd=hd)) for name in ("test_one_sequence",) for H, Hkv, hd in ((6, 2, 64), (8, 2, 128)) for T, ctx in ((6, 0), (17, 65), (70, 300))],
    *[("test_ragged_batch", dict(hd=hd, page=page)) for hd in (64, 128) for page in (32, 160)],
    ("test_sharp_scores", {}), ("test_queries_of_many_sizes", dict(hd=64)), ("test_queries_of_many_sizes", dict(hd=128)), ("test_repeats_itself", {}),
    *[("test_masked_numbers_that_are_not_finite", dict(bad=bad)) for bad in (float("nan"), float("inf"), -float("inf"), 3.2e38)],
    ("test_a_bad_number_in_the_context_reaches_every_row", dict(T=40))], ids=lambda c: "-".join([c[0][5:], *map(str, c[1].values())]))
def test_tiles_of_128_rows(monkeypatch, call):
    """The tests of test_gpu_cache4 that pad their page lists, by more."""
    monkeypatch.setattr(test_gpu_cache4, "Case4", Tall)
    getattr(test_gpu_cache4, call[0])(**call[1], dtype="bf16", wide=True)


def test_rows_of_tall_tiles_that_see_nothing():
    c = Tall([0, 40], [9, 9], 9, 8, 2, 64, "bf16", seed=10)
    see, words = c.masks(seed=10, empty=(0, 4, 8))
    c.check(words, see)


@pytest.mark.parametrize("hd", [64, 128])
def test_pages_out_of_range_under_tall_tiles(hd):
    """A page outside the pool hides its positions, at each place of a step of two pages."""
    ctx, T = 150, 20
    c = Tall([ctx], [T], T, 4, 1, hd, "bf16", seed=13, spare=0)
    for at in (1, 2, 3):
        keep = torch.cat([torch.arange(32 * at), torch.arange(32 * at + 32, ctx + T)]).cuda()
        for wrong in (-1, c.kv.n_pages, 2 ** 31 - 1, -2 ** 31):
            t = c.table.clone()
            t[0, at] = wrong
            out, lse = ngg.tree_attention(c.q, c.kv, t, ints([ctx]), want_lse=True)
            test_gpu_cache4.check4(out, lse, c.q, [c.ks[0][keep]], [c.vs[0][keep]], [ctx - 32], [T], None, c.scale, "bf16")


@pytest.mark.parametrize("hd", [64, 128])
def test_strides_of_tall_tiles(hd):
    c = Tall([40, 7, 130], [20] * 3, 20, 4, 2, hd, "bf16", seed=15)
    want = c.check()[0]
    for gap in (1, 2, 8):
        big = torch.zeros(20, 3, 16, hd + gap, dtype=torch.bfloat16, device="cuda")
        q = big.permute(1, 0, 2, 3)[..., gap:]
        q.copy_(c.q)
        dst = torch.full((3, 16, 20, hd + gap), 5.0, dtype=torch.bfloat16, device="cuda")
        out = dst.permute(0, 2, 1, 3)[..., gap:]
        ngg.tree_attention(q, c.kv, c.table, ints(c.ctx), out=out)
        assert torch.equal(out, want) and (dst[..., :gap] == 5.0).all()


def put(c, k, v):
    """Keys and values [positions, heads, head_dim], which 4 bits hold as they are, for the one sequence of a Case4."""
    pos = torch.arange(len(k), device="cuda")
    slots = (c.table[0, pos // 64] * 64 + pos % 64).int()
    c.kv.write(k.contiguous(), v.contiguous(), slots)
    c.ks[0], c.vs[0] = c.kv.read(slots, torch.float32)
    assert torch.equal(c.ks[0], k) and torch.equal(c.vs[0], v)


FP32 = [(16, 0, 4, 4, 128, 1, 0), (16, 0, 8, 2, 64, 3, 0), (16, 0, 4, 1, 32, 4, 0), (16, 71, 8, 2, 128, 9, 18000), (16, 71, 8, 2, 64, 9, 18000), (32, 118, 8, 2, 64, 9, 120000),
        (32, 125, 8, 2, 32, 9, 480000)]


@pytest.mark.parametrize("rows,n,H,Hkv,hd,T,positions", FP32)
def test_fp32_calls_keep_24_bits_of_a_query(rows, n, H, Hkv, hd, T, positions):
    """Sixteen dimensions that are alike, of which the first two bfloat16 terms leave 2^-17, all of one sign: without the third the scores, and with them
    the log sums, are off by 2^-17 of themselves.  They may be off by (16 + 14) 2^-24 of the sum of |q k|, sums of n terms by (n + 8) 2^-24 and the
    logarithm by 2^-23 of itself."""
    x = 1 + 16448 * 2.0 ** -23
    c = Case4([5], [T], T, H, Hkv, hd, "f32", page=64, seed=51)
    widen(c, positions)
    assert workspace(c) == pieces(c, rows, n)
    keys = 5 + T
    k = torch.zeros(keys, Hkv, hd, device="cuda")
    k[..., :16] = torch.tensor([3.0, 4.0, 6.0], device="cuda")[torch.arange(keys, device="cuda") % 3][:, None, None]
    put(c, k, torch.ones_like(k))
    c.q.zero_()
    c.q[..., :16] = x
    c.scale = 0.25
    _, lse = ngg.tree_attention(c.q, c.kv, c.table, ints([5]), scale=0.25, want_lse=True)
    first = torch.tensor(x, dtype=torch.float64).bfloat16().double()
    two = (first + (x - first).bfloat16().double()).item()
    for h in range(H):
        want, qk = exact(c, 0, h)[2:]
        tol = (16 + 14) * 2.0 ** -24 * qk + (keys + 8) * 2.0 ** -24 + 2.0 ** -23 * want.abs()
        assert ((lse[0, :, h].double() - want).abs() <= tol).all()
    c.q = c.q.double() / x * two
    assert ((exact(c, 0, 0)[2] - want).abs() > 2 * tol).all()


@pytest.mark.parametrize("rows,n,H,Hkv,hd,T,positions", FP32)
def test_fp32_calls_keep_24_bits_of_a_probability(rows, n, H, Hkv, hd, T, positions):
    """Keys of two kinds: the first have the row's largest score and values of zero, the others a probability beside them of 0.50224686, of which two
    bfloat16 terms leave 2^-17, and values of one.  Without the third term outputs are off by 2^-17 of themselves; they may be by 2 (1 + 10) 2^-24 of the
    sum of |q k| (of one dimension), by 3 n 2^-24 for sums of n terms, and by their rounding."""
    c = Case4([1], [T], T, H, Hkv, hd, "f32", page=64, seed=52)
    widen(c, positions)
    assert workspace(c) == pieces(c, rows, n)
    keys = 1 + T
    second = torch.arange(keys, device="cuda") % 2 == 1
    k, v = (torch.zeros(keys, Hkv, hd, device="cuda") for _ in range(2))
    k[..., 0] = torch.where(second, 0.5, 1.0)[:, None]
    v[:] = second.float()[:, None, None]
    put(c, k, v)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.scale = float(np.float32(-2 * np.log(0.50224686)))
    out = ngg.tree_attention(c.q, c.kv, c.table, ints([1]), scale=c.scale)
    for h in range(H):
        want, mag, _, qk = exact(c, 0, h)
        tol = mag * (2 * (1 + 10) * 2.0 ** -24 * qk[:, None] + 3 * keys * 2.0 ** -24) + want.abs() * 2.0 ** -24
        assert ((out[0, :, h].double() - want).abs() <= tol).all()
        assert ((exact(c, 0, h, 3)[0] - want).abs() <= tol).all()
        assert ((exact(c, 0, h, 2)[0] - want).abs() > 1.5 * tol).all()
