"""The operators together, with a cache in 4 bits, page lists that grow, shared beginnings and paths that move.  Needs an MI355X."""
import numpy as np
import pytest
import torch

from paper_2411_03786_amd import tree_verify as tv
from test_gpu_tree_verify import drafts_from

pytestmark = pytest.mark.gpu


def held(dec):
    """The pages that the sequences list, checked against the counts."""
    refs = np.zeros(dec.table.refs.numel(), int)
    for row in dec.pages.tolist():
        live = [p for p in row if p >= 0]
        assert row == live + [-1] * (len(row) - len(live))
        np.add.at(refs, live, 1)
    assert dec.table.refs.tolist() == refs.tolist()
    return refs


@pytest.mark.parametrize("shared,page", [(64, 32), (70, 32), (31, 32), (100, 64), (1, 32)])
def test_shared_beginnings_decode_as_prompts_of_their_own(shared, page):
    dec = tv.TreeDecoder(4, 2, 4, 2, 32, 500, 300, cache="f32", page=page, d_ffn=256, seed=3)
    prompts = np.random.default_rng(1).integers(0, 500, (4, 101))
    prompts[:, :shared] = prompts[0, :shared]
    prompts = prompts.tolist()
    n = 30
    own, own_lp, _ = dec.decode(prompts, n, lambda b, s: [])
    most = (held(dec) > 0).sum()
    assert held(dec).max() == 1
    for draft in (lambda b, s: [], drafts_from(own, prompts, 2)):
        got, lp, _ = dec.decode(prompts, n, draft, share=True)
        assert got == own
        # fp32 sums of a few hundred terms in two layers, values of a few units
        assert np.abs(np.array(lp) - np.array(own_lp)).max() < 1e-3
        refs = held(dec)
        assert (refs == 4).sum() == shared // page                      # the full pages of the beginning, the last one is everybody's own
        assert (refs > 0).sum() <= most - 3 * (shared // page) + 4
    dec.clear()
    assert not dec.table.refs.any()


def test_prompts_that_are_all_alike():
    dec = tv.TreeDecoder(3, 1, 2, 1, 32, 100, 90, cache="f32", page=32, d_ffn=64)
    prompt = np.random.default_rng(4).integers(0, 100, 50).tolist()
    got, _, _ = dec.decode([prompt] * 3, 20, lambda b, s: tv.context_rows(s, 3, 4), share=True)
    assert got[0] == got[1] == got[2] == dec.decode([prompt] * 3, 20, lambda b, s: [])[0][0]


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_trees_over_four_bits_follow_their_own_drafts(hd):
    """Tokens of one run as the drafts of the next: nearly all are accepted (near-ties may turn), and the run repeats itself."""
    dec = tv.TreeDecoder(4, 2, 8, 2, hd, 1000, 400, cache="fp4", page=64, d_ffn=512, seed=5)
    prompts = np.random.default_rng(2).integers(0, 1000, (4, 130)).tolist()
    n = 48
    plain, lp, _ = dec.decode(prompts, n, lambda b, s: [])
    follow = lambda b, s: [plain[b][len(s) - 130:len(s) - 130 + 8]] if s[130:] == plain[b][:len(s) - 130] else []
    a, a_lp, steps = dec.decode(prompts, n, follow)
    again, again_lp, steps2 = dec.decode(prompts, n, follow)
    assert a == again and a_lp == again_lp and steps == steps2 < n
    assert all(np.isfinite(x).all() for x in (lp, a_lp))


def test_what_moves_is_what_was_read_and_written_before():
    """keep() against reading every layer's path and writing it behind the context."""
    dec = tv.TreeDecoder(3, 3, 4, 2, 64, 200, 200, cache="fp8", page=32, d_ffn=128)
    dec.prefill(torch.randint(0, 200, (3, 40), dtype=torch.int32, device="cuda"))
    tokens = torch.randint(0, 200, (3, 20), dtype=torch.int32, device="cuda")
    dec.forward(tokens, torch.arange(20, device="cuda"), logits=False)
    paths = [[0, 3, 4, 19], [0], [0, 1, 2, 7, 8, 9]]
    want = []
    for kv in dec.kv:
        for b, path in enumerate(paths):
            at = dec.slots(torch.full((3, len(path)), -1, device="cuda").index_put((torch.tensor(b), torch.arange(len(path))), dec.lens[b] + torch.tensor(path, device="cuda", dtype=torch.int32).long()))
            want.append([t.clone() for t in kv.read(at[at >= 0])])
    dec.keep(paths)
    assert dec.lens.tolist() == [39 + 4, 39 + 1, 39 + 6] == dec.cached
    i = 0
    for kv in dec.kv:
        for b, path in enumerate(paths):
            pos = 39 + torch.arange(len(path), device="cuda")
            got = kv.read((dec.pages[b, pos // 32] * 32 + pos % 32).int())
            assert all(torch.equal(g, w) for g, w in zip(got, want[i]))
            i += 1


def test_the_command_with_shared_prompts_in_four_bits(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ("tree_verify --batch 3 --layers 2 --heads 8 --kv-heads 2 --head-dim 64 --vocab 600 --prompt 90 --shared 70 --new 70 "
                                     "--cycle 20 --cache fp4").split())
    tv.main()
    lines = capsys.readouterr().out.splitlines()
    steps = [int(x.split(" steps")[0].split()[-1]) for x in lines[:2]]
    assert steps[0] == 70 and steps[1] < 40
