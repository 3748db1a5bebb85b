"""Corners of the operators of a batched tree verification on the GPU.  Needs an MI355X."""
import numpy as np
import pytest
import torch

import paper_2411_03786_amd as ngg
from paper_2411_03786_amd import tree_verify as tv
from test_gpu_operators import DT, Case, attention64, check_scores, eight_bits, ints, randn, score64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,scale,size", [(300, 5e8, 20.0), (33000, 5e8, 20.0), (33000, 1e7, 300.0), (5000, 1.0, 3e9), (5000, 1.0, 1e30), (33000, 0.5, 1e38), (700, 1e30, 1.0)])
def test_token_logprobs_of_large_scores(dtype, V, scale, size):
    """Finite rows have finite sums whatever their size.  x * scale is off by 2^-24 of itself, a difference of two and a sum of up to V terms by a
    few of those."""
    x = randn(9, V, seed=V)
    x = (x / x.abs().amax() * size).to(DT[dtype])
    targets, top = np.array([[0, V - 1, V // 2]] * 9), min(V, 7)
    got = ngg.token_logprobs(x, ints(targets), top_n=top, scale=scale)
    lp, ent, lse, ids, tlp = score64(x, targets, top, scale)
    big = np.abs(lse) + 4
    assert torch.isfinite(got.lse).all() and (np.abs(got.lse.double().cpu().numpy() - lse) <= 2.0 ** -22 * big).all()
    assert torch.isfinite(got.entropy).all() and (np.abs(got.entropy.double().cpu().numpy() - ent) <= (V / 64 + 64) * 2.0 ** -22).all()
    assert (got.top_ids.cpu().numpy() == ids).all() and (got.top_logprobs[:, 0] > -1.0).all()
    for g, w in ((got.logprobs, lp), (got.top_logprobs, tlp)):
        assert (np.abs(g.double().cpu().numpy() - w) <= 2.0 ** -22 * (np.abs(w) + big[:, None])).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-1e7, -1e9, -1e12, -1e30])
def test_token_logprobs_of_rows_with_low_parts(dtype, low):
    """Ruled-out tokens at a low number instead of minus infinity, in runs longer than what a wave takes at a time, and rows of nothing else."""
    x = randn(6, 40003, seed=3)
    x[0, :20000] = low
    x[1, 20000:] = low
    x[2, 5000:39000] = low
    x[3] = low
    x[4] += low
    x[5, ::2] = low
    check_scores(x.to(DT[dtype]), [[0, 39999, 20000]] * 6, 5, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2000, 32000, 40003])
@pytest.mark.parametrize("scale", [0.7, 1.0, 1.25, 3e4, 1e6, 1e8])
def test_token_logprobs_of_peaked_rows(dtype, V, scale):
    """One token far ahead.  What is left near 0 is off by the roundings of a sum near 1 and of its logarithm, 16 at most, however large the
    logits are; a probability is never above 1, an entropy never below 0."""
    n = 60
    x = randn(n, V, seed=V)
    rng = np.random.default_rng(V)
    best = rng.integers(0, V, n)
    x[torch.arange(n), torch.from_numpy(best).cuda()] = torch.from_numpy(rng.uniform(20.0, 70.0, n)).float().cuda()
    x = x.to(DT[dtype])
    targets = np.stack([best, rng.integers(0, V, n)], 1)
    got = ngg.token_logprobs(x, ints(targets), top_n=3, scale=scale)
    lp, ent, lse, ids, tlp = score64(x, targets, 3, scale)
    assert (got.top_ids.cpu().numpy() == ids).all()
    for g, w in ((got.logprobs, lp), (got.top_logprobs, tlp)):
        assert (g <= 0).all()
        assert (np.abs(g.double().cpu().numpy() - w) <= 16 * 2.0 ** -24 + 2.0 ** -22 * np.abs(w)).all()
    assert (got.entropy >= 0).all()
    # the same roundings, of sums whose terms are up to 1 as well
    assert (np.abs(got.entropy.double().cpu().numpy() - ent) <= 32 * 2.0 ** -24).all()
    assert (np.abs(got.lse.double().cpu().numpy() - lse) <= 2.0 ** -22 * np.abs(lse)).all()


def test_token_logprobs_of_more_rows_than_a_launch_has_workgroups():
    n, V = (1 << 24) + 5, 3
    x = torch.randn(n, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    t = torch.randint(0, V, (n,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(2))
    got = ngg.token_logprobs(x, t, top_n=2)
    want = x.log_softmax(-1)
    # a handful of fp32 operations on values of a few units, on either side
    assert (got.logprobs - want.gather(1, t.long()[:, None])[:, 0]).abs().max() < 16 * 2.0 ** -22
    assert torch.equal(got.top_ids[:, 0].long(), x.argmax(-1)) and (got.lse - x.logsumexp(-1)).abs().max() < 16 * 2.0 ** -22


def test_cache_of_more_tokens_than_a_launch_has_workgroups():
    """2^29 tokens and some, one row for all but a few of them, and read back from the places around the parts."""
    n, hd = (1 << 29) + 70, 32
    kv = ngg.KVPages((n + 63) // 64, 64, 1, hd, "fp8")
    rows = (torch.arange(2 * hd, device="cuda", dtype=torch.float32) / 64 - 0.5).to(torch.bfloat16).view(2, 1, 1, hd)
    k, v = (r.expand(n, 1, hd) for r in rows)
    kv.write(k, v, torch.arange(n, dtype=torch.int32, device="cuda"))
    at = ints([0, 1 << 20, (1 << 28) - 1, 1 << 28, (1 << 28) + 33, (1 << 29) - 1, 1 << 29, n - 1])
    for got, row in zip(kv.read(at), rows):
        assert torch.equal(got, eight_bits(row).to(torch.bfloat16).expand(8, 1, hd))
    got = kv.read(torch.arange(n, dtype=torch.int32, device="cuda").fill_(5))       # all of them from one place
    for g, row in zip(got, rows):
        assert torch.equal(g[-3:], eight_bits(row).to(torch.bfloat16).expand(3, 1, hd)) and torch.equal(g[(1 << 28) - 2:(1 << 28) + 2], g[:4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
def test_tree_attention_of_a_slot_that_nobody_wrote(dtype, wide):
    """A tree position inside the sequence that no row sees: whatever its bytes and exponents hold, the rows are as they were."""
    T, ctx, j = 21, 50, 12
    c = Case([ctx], [T], T, 4, 2, 64, dtype, "fp8", seed=11, wide=wide)
    see, words = c.masks(seed=11)
    see[:, :, j] = False
    words &= ~(1 << j)
    clean, clean_lse = c.check(words, see)
    slot = c.table[0, (ctx + j) // 32] * 32 + (ctx + j) % 32
    x = torch.full((1, 2, 64), float("nan"), dtype=DT[dtype], device="cuda")
    c.kv.write(x, x, slot[None].int())
    page, at = int(slot) // 32, int(slot) % 32
    for e in (255, 254, 0):
        for exps in (c.kv.k_exps, c.kv.v_exps):
            exps.view(c.kv.n_pages, 2, 32)[page, :, at] = e
        out, lse = ngg.tree_attention(c.q, c.kv, c.table, ints([ctx]), mask=words, want_lse=True)
        assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


def test_a_table_in_host_memory_is_refused():
    rope, x, pos = ngg.Rope(32, 16, device="cpu"), randn(3, 2, 32, dtype="bf16"), ints([0, 1, 2])
    kv = ngg.KVPages(1, 32, 2, 32, "bf16")
    side = torch.cuda.Stream()
    for stream in (None, side):
        with pytest.raises(ValueError):
            kv.write(x, x, pos, rope=rope, positions=pos, stream=stream)
        with pytest.raises(ValueError):
            ngg.rotary(rope, pos, x, stream=stream)
    with pytest.raises(ValueError):
        kv.write(x, x, pos, rope=ngg.Rope(32, 16))                     # no positions
    assert not kv.k_bytes.any()


def test_rotary_of_an_empty_projection():
    """No tokens, and rows that are slices of something wider."""
    H, Hkv, hd = 4, 2, 64
    q, k, _ = torch.empty(0, H + 2 * Hkv, hd, dtype=torch.bfloat16, device="cuda").split((H, Hkv, Hkv), 1)
    assert q.stride(0) != H * hd
    rope = ngg.Rope(hd, 16)
    a, b = ngg.rotary(rope, ints([]), q, k)
    assert a.shape == (0, H, hd) and b.shape == (0, Hkv, hd)
    assert ngg.rotary(rope, ints([]), q, out=q).shape == (0, H, hd)


def operator_calls():
    """The operators' calls on a tensor of queries (keys, values) and on logits, each by its name."""
    rope, kv = ngg.Rope(64, 32), ngg.KVPages(2, 32, 4, 64, "bf16")
    one, at = ints([[0, 1]]), ints(range(6))
    return dict(rotary=lambda x: ngg.rotary(rope, at, x), rotary_k=lambda x: ngg.rotary(rope, at, x.detach(), x), keys=lambda x: kv.write(x, x.detach(), at),
                values=lambda x: kv.write(x.detach(), x, at), attention=lambda x: ngg.tree_attention(x[None], kv, one, ints([0])),
                logprobs=lambda x: ngg.token_logprobs(x.flatten(1), top_n=2), rotary_out=lambda x: ngg.rotary(rope, at, x.detach(), out=x),
                attention_out=lambda x: ngg.tree_attention(x.detach()[None], kv, one, ints([0]), out=x[None]))


@pytest.mark.parametrize("name", ["rotary", "rotary_k", "keys", "values", "attention", "logprobs", "rotary_out", "attention_out"])
def test_tensors_that_require_gradients_are_refused(name):
    call, x = operator_calls()[name], randn(6, 4, 64, dtype="bf16")
    call(x)
    x.requires_grad_(True)
    with pytest.raises(RuntimeError, match="gradient"):
        call(x)
    with torch.no_grad():
        call(x)
    with torch.inference_mode():
        call(x.clone())


def test_outputs_written_in_place_raise_their_version():
    rope, at, x = ngg.Rope(64, 32), ints(range(6)), randn(6, 4, 64, dtype="bf16")
    before = x._version
    ngg.rotary(rope, at, x, out=x)
    assert x._version > before
    y = torch.empty(1, 6, 4, 64, dtype=torch.bfloat16, device="cuda")
    before = y._version
    ngg.tree_attention(x[None], ngg.KVPages(2, 32, 4, 64, "bf16"), ints([[0, 1]]), ints([0]), out=y)
    assert y._version > before


def test_outputs_whose_elements_share_memory_are_refused():
    rope, at, x = ngg.Rope(64, 32), ints(range(6)), randn(6, 4, 64, dtype="bf16")
    kv = ngg.KVPages(2, 32, 4, 64, "bf16")
    flat = torch.zeros(6 * 4 * 64, dtype=torch.bfloat16, device="cuda")
    for out in (flat[:4 * 64].view(1, 4, 64).expand(6, -1, -1), flat[:6 * 64].view(6, 1, 64).expand(-1, 4, -1), flat.as_strided((6, 4, 64), (128, 64, 1)),
                flat.as_strided((6, 4, 64), (256, 63, 1))):
        with pytest.raises(ValueError):
            ngg.rotary(rope, at, x, out=out)
        with pytest.raises(ValueError):
            ngg.rotary(rope, at, x, x, k_out=out)
        with pytest.raises(ValueError):
            ngg.tree_attention(x[None], kv, ints([[0, 1]]), ints([0]), out=out[None])
    assert not flat.any()
    for out in (torch.empty(4, 6, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1), torch.empty(6, 4, 70, dtype=torch.bfloat16, device="cuda")[..., 3:67]):
        assert torch.equal(ngg.rotary(rope, at, x, out=out), ngg.rotary(rope, at, x))


def test_decoder_tables_reach_as_far_as_its_pages():
    prompts = np.random.default_rng(1).integers(0, 100, (2, 20)).tolist()
    runs = [tv.TreeDecoder(2, 1, 2, 1, 32, 100, n, cache="f32", page=32, d_ffn=64, seed=4).decode(prompts, 40, lambda b, s: []) for n in (40, 64)]
    assert np.isfinite(runs[0][1]).all() and runs[0] == runs[1]


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("H,Hkv,hd,T,ctx", [(8, 2, 64, 1, 300), (8, 2, 128, 5, 900), (4, 1, 128, 30, 400), (16, 4, 32, 13, 2000)])
def test_tree_attention_keeps_16_bits_of_a_probability(cache, H, Hkv, hd, T, ctx):
    """Values of either sign leave little of a row's sum, so that what its terms lose is seen beside the rounding of the output: 2^-16 of
    a term's share, not the 2^-9 of a probability in bf16, besides what fp32 sums may be off by (test_gpu_operators)."""
    c = Case([ctx, ctx // 2], [T, T], T, H, Hkv, hd, "bf16", cache, seed=5)
    see, words = c.masks(seed=5)
    out = ngg.tree_attention(c.q, c.kv, c.table, ints(c.ctx), mask=words)
    want, _, mag, qk = attention64(c.q, c.ks, c.vs, c.ctx, c.trees, see, c.scale)
    e = (2 * (hd + 8) * 2.0 ** -24 * qk + 2.0 ** -15)[..., None]
    assert ((out.double() - want).abs() <= mag * (e + 2.0 ** -16) + want.abs() * 2.0 ** -8).all()


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("f32", "fp8"), ("bf16", "fp8")])
@pytest.mark.parametrize("rows", [1536, 3072, 4096])
def test_cache_by_rows_and_by_groups_alike(dtype, cache, rows):
    """Calls on either side of the sizes from which rows move in groups, in runs of 13 slots that begin anywhere: one call as two halves."""
    Hkv, hd = 4, 128
    for n in (rows // Hkv, rows // Hkv + 1):
        slots = 5 + np.arange(n) // 13 * 17 + np.arange(n) % 13
        pool = int(slots[-1]) // 64 + 1
        x = randn(n, 2 * Hkv, hd, seed=rows, dtype=dtype)
        rope, pos = ngg.Rope(hd, 300), ints(np.arange(n) % 300)
        for turn in (dict(), dict(rope=rope)):
            a, b = (ngg.KVPages(pool, 64, Hkv, hd, cache) for _ in range(2))
            for kv, parts in ((a, [(0, n)]), (b, [(0, n // 2), (n // 2, n)])):
                for i, j in parts:
                    kv.write(x[i:j, :Hkv], x[i:j, Hkv:], ints(slots[i:j]), **(dict(turn, positions=pos[i:j]) if turn else {}))
            assert torch.equal(a.k_bytes, b.k_bytes) and torch.equal(a.v_bytes, b.v_bytes)
            if cache == "fp8":
                assert torch.equal(a.k_exps, b.k_exps) and torch.equal(a.v_exps, b.v_exps)
            whole, half = a.read(ints(slots), DT[dtype]), a.read(ints(slots[:n // 2]), DT[dtype])
            assert all(torch.equal(w[:n // 2], h) for w, h in zip(whole, half))
            assert torch.equal(whole[1], eight_bits(x[:, Hkv:]).to(DT[dtype]) if cache == "fp8" else x[:, Hkv:])


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_trees_of_16_bit_models_accept_what_single_tokens_wrote(cache):
    """The single tokens' run as drafts of eight: every step takes nine tokens until the runs part, and they part only where two tokens are
    as likely but for 16-bit sums.  Those are off by 2^-9 a dozen times on the way to logits of up to 4 (an 8-bit cache by some of its
    2^-4 steps where such a sum turns one): some hundredths, and 1 / 8 at most; a wrong mask, depth or kept path changes them by whole units."""
    prompt, n = 130, 48
    dec = tv.TreeDecoder(4, 2, 8, 2, 64, 1000, 400, cache=cache, page=64, d_ffn=512, seed=5)
    prompts = np.random.default_rng(2).integers(0, 1000, (4, prompt)).tolist()
    plain, lp, _ = dec.decode(prompts, n, lambda b, s: [])
    follow = lambda b, s: [plain[b][len(s) - prompt:len(s) - prompt + 8]] if s[prompt:] == plain[b][:len(s) - prompt] else []
    got, got_lp, steps = dec.decode(prompts, n, follow)
    most = 0
    for b in range(4):
        same = next((i for i in range(n) if got[b][i] != plain[b][i]), n)
        assert np.abs(np.array(got_lp[b][:same + 1]) - np.array(lp[b][:same + 1])).max() < 0.125
        most = max(most, -(-same // 9) + n - same)
    assert steps <= most + 1
