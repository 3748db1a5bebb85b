"""The operators together: greedy decoding of several sequences with drafts verified as trees.  Needs an MI355X."""
import numpy as np
import pytest
import torch

from paper_2411_03786_amd import tree_verify as tv

pytestmark = pytest.mark.gpu


def dense_logits(dec, tokens):
    """The model on one sequence at once, without a cache, in 64 bits: logits [n, vocab]."""
    n, hd = len(tokens), dec.hd
    norm = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    w64 = lambda w: w.double()
    turn = lambda y: torch.cat([y[..., :hd // 2] * c - y[..., hd // 2:] * s, y[..., hd // 2:] * c + y[..., :hd // 2] * s], -1)
    c, s = (t[:n, None].double() for t in (dec.rope.cos, dec.rope.sin))
    x = w64(dec.embed)[torch.tensor(tokens, device="cuda")]
    for w in dec.layers:
        q, k, v = (norm(x) @ w64(w["qkv"])).view(n, -1, hd).split((dec.heads, dec.kv_heads, dec.kv_heads), 1)
        q, k = turn(q), turn(k)
        group = dec.heads // dec.kv_heads
        heads = []
        for h in range(dec.heads):
            p = (q[:, h] @ k[:, h // group].T.contiguous() * hd ** -0.5).masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), -float("inf")).softmax(-1)
            heads.append(p @ v[:, h // group].contiguous())
        x = x + torch.cat(heads, -1) @ w64(w["proj"])
        y = norm(x)
        x = x + (torch.nn.functional.silu(y @ w64(w["gate"])) * (y @ w64(w["up"]))) @ w64(w["down"])
    return norm(x) @ w64(dec.unembed)


def drafts_from(truth, prompts, seed):
    """Rows that begin with the true continuation and leave it after some tokens, in any order."""
    rng = np.random.default_rng(seed)

    def draft(b, seq):
        at = len(seq) - len(prompts[b])
        rows = []
        for _ in range(int(rng.integers(0, 5))):
            row = truth[b][at:at + int(rng.integers(1, 7))] + rng.integers(0, 500, 2).tolist()
            rows.append(row)
        rng.shuffle(rows)
        return rows
    return draft


def test_trees_decode_what_single_tokens_do_and_the_dense_model_says():
    dec = tv.TreeDecoder(3, 2, 4, 2, 32, 500, 300, cache="f32", page=32, d_ffn=256, seed=3)
    prompts = np.random.default_rng(1).integers(0, 500, (3, 70)).tolist()
    n = 40
    plain, plain_lp, steps = dec.decode(prompts, n, lambda b, s: [])
    assert steps == n
    trees, trees_lp, fewer = dec.decode(prompts, n, drafts_from(plain, prompts, 2))
    assert trees == plain and fewer < n
    # fp32 sums of a few hundred terms in two layers, values of a few units
    assert np.abs(np.array(trees_lp) - np.array(plain_lp)).max() < 1e-3
    own, _, _ = dec.decode(prompts, n, lambda b, s: tv.context_rows(s, 4, 5))
    assert own == plain
    for b in range(3):
        logits = dense_logits(dec, prompts[b] + plain[b])[len(prompts[b]) - 1:-1]
        lp = logits.log_softmax(-1)
        got = torch.tensor(plain[b], device="cuda")
        assert ((lp.max(-1).values - lp.gather(1, got[:, None])[:, 0]) < 1e-3).all()      # the greedy token, or one as likely
        assert (lp.gather(1, got[:, None])[:, 0].cpu() - torch.tensor(plain_lp[b], dtype=torch.float64)).abs().max() < 1e-3


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_trees_of_16_bit_models_follow_their_own_drafts(cache):
    """Tokens of one run as the drafts of the next: nearly all are accepted (near-ties may turn), and the run repeats itself."""
    dec = tv.TreeDecoder(4, 2, 8, 2, 64, 1000, 400, cache=cache, page=64, d_ffn=512, seed=5)
    prompts = np.random.default_rng(2).integers(0, 1000, (4, 130)).tolist()
    n = 48
    plain, lp, _ = dec.decode(prompts, n, lambda b, s: [])
    follow = lambda b, s: [plain[b][len(s) - 130:len(s) - 130 + 8]] if s[130:] == plain[b][:len(s) - 130] else []
    a, a_lp, steps = dec.decode(prompts, n, follow)
    again, again_lp, steps2 = dec.decode(prompts, n, follow)
    assert a == again and a_lp == again_lp and steps == steps2 < n
    assert all(np.isfinite(x).all() for x in (lp, a_lp))


def test_the_command(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", "tree_verify --batch 3 --layers 2 --heads 8 --kv-heads 2 --head-dim 64 --vocab 600 --prompt 90 --new 70 --cycle 20".split())
    tv.main()
    lines = capsys.readouterr().out.splitlines()
    steps = [int(x.split(" steps")[0].split()[-1]) for x in lines[:2]]
    assert steps[0] == 70 and steps[1] < 35 and lines[2] == "3 of 3 sequences alike"


def test_a_tree_beyond_the_pages_is_refused():
    dec = tv.TreeDecoder(2, 1, 2, 1, 32, 100, 64, cache="f32", page=32, d_ffn=64)
    dec.prefill(torch.zeros(2, 61, dtype=torch.int32, device="cuda"))
    assert len(dec.step([1, 2], [[[3, 4, 5]], []])) == 2                 # 60 cached, trees of up to four
    with pytest.raises(ValueError):
        dec.step([1, 2], [[[3, 4, 5, 6]], []])


def test_draft_trees_share_their_beginnings():
    tokens, parents, children = tv.draft_tree(9, [[1, 2, 3], [1, 2, 4], [5], [1]])
    assert tokens == [9, 1, 2, 3, 4, 5] and parents == [-1, 0, 1, 2, 2, 0]
    assert children[0] == {1: 1, 5: 5} and children[2] == {3: 3, 4: 4}
    assert tv.context_rows([1, 2, 3, 1, 2, 4, 1, 2], 4, 2) == [[4, 1], [3, 1]]
    assert tv.context_rows([1], 4, 2) == []
