"""Host-side checks of the operators of a batched tree verification: rotary tables against their formulas in 64 bits, masks of
trees against walks along the parents, sizes, and the refusals that come before any device work."""
import ctypes as C
import math
import os

import numpy as np
import pytest

import paper_2411_03786_amd as ngg


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ngg.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return ngg.load_library()


def table(lib, theta, rd, n, scaling=None):
    cos, sin = np.full((n, rd // 2), 7, np.float32), np.full((n, rd // 2), 7, np.float32)
    st = lib.ngg_rope_table(theta, rd, n, C.byref(scaling) if scaling is not None else None, cos.ctypes.data, sin.ctypes.data)
    assert st == ngg.NGG_OK, lib.ngg_last_error(None)
    return cos, sin


def frequencies(theta, rd, sc):
    """Pair by pair, as ngg.h states it."""
    if sc is not None and sc.kind == 2:
        theta = theta * sc.factor ** (rd / (rd - 2))
    out = []
    for i in range(rd // 2):
        f = theta ** (-2.0 * i / rd)
        if sc is not None and sc.kind == 1:
            f /= sc.factor
        if sc is not None and sc.kind == 3:
            n = sc.original * f / (2 * math.pi)
            if n <= sc.low:
                f /= sc.factor
            elif n < sc.high:
                w = (n - sc.low) / (sc.high - sc.low)
                f = w * f + (1 - w) * f / sc.factor
        if sc is not None and sc.kind == 4:
            at = lambda turns: rd * math.log(sc.original / (2 * math.pi * turns)) / (2 * math.log(theta))
            lo, hi = max(0, math.floor(at(sc.high))), min(rd - 1, math.ceil(at(sc.low)))
            w = 1.0 if i <= lo else 0.0 if i >= hi else (hi - i) / (hi - lo)
            f = w * f + (1 - w) * f / sc.factor
        out.append(f)
    return np.array(out)


SCALINGS = [None, ngg.ngg_rope_scaling(1, 0, 4.0, 0, 0, 0), ngg.ngg_rope_scaling(2, 0, 8.0, 0, 0, 0),
            ngg.ngg_rope_scaling(3, 8192, 8.0, 1.0, 4.0, 0), ngg.ngg_rope_scaling(4, 4096, 16.0, 1.0, 32.0, 0.1 * math.log(16.0) + 1.0)]


@pytest.mark.parametrize("sc", SCALINGS, ids=["plain", "linear", "base", "bands", "ramp"])
@pytest.mark.parametrize("theta,rd,n", [(10000.0, 128, 300), (500000.0, 64, 5000), (10000.0, 6, 9), (10000.0, 32, 1)])
def test_rotary_tables_are_the_formulas_rounded_once(lib, sc, theta, rd, n):
    cos, sin = table(lib, theta, rd, n, sc)
    ang = np.arange(n)[:, None] * frequencies(theta, rd, sc)[None]
    amp = sc.amplitude if sc is not None and sc.amplitude else 1.0
    # an angle in 64 bits is off by less than 2^-50 of itself (up to 5000 radians here), the rest is the rounding to 32 bits
    for got, want in ((cos, amp * np.cos(ang)), (sin, amp * np.sin(ang))):
        assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + amp * 5000 * 2.0 ** -48).all()


def test_rotary_table_refuses(lib):
    buf = np.zeros((4, 4), np.float32)
    p = buf.ctypes.data
    bad = [(10000.0, 7, 4, None), (10000.0, 0, 4, None), (10000.0, 2048, 4, None), (10000.0, 8, 0, None), (1.0, 8, 4, None),
           (float("nan"), 8, 4, None), (float("inf"), 8, 4, None), (1e4, 8, 4, ngg.ngg_rope_scaling(9, 0, 2.0, 0, 0, 0)),
           (1e4, 8, 4, ngg.ngg_rope_scaling(1, 0, 0.5, 0, 0, 0)), (1e4, 8, 4, ngg.ngg_rope_scaling(1, 0, float("nan"), 0, 0, 0)),
           (1e4, 8, 4, ngg.ngg_rope_scaling(3, 0, 2.0, 1.0, 4.0, 0)), (1e4, 8, 4, ngg.ngg_rope_scaling(3, 64, 2.0, 4.0, 1.0, 0)),
           (1e4, 2, 4, ngg.ngg_rope_scaling(2, 0, 2.0, 0, 0, 0)), (1e4, 8, 4, ngg.ngg_rope_scaling(1, 0, 2.0, 0, 0, -1.0))]
    for theta, rd, n, sc in bad:
        assert lib.ngg_rope_table(theta, rd, n, C.byref(sc) if sc is not None else None, p, p) == ngg.NGG_EINVAL, (theta, rd, n)
        assert b"ngg_rope_table" in lib.ngg_last_error(None)
    assert lib.ngg_rope_table(1e4, 8, 4, None, None, p) == ngg.NGG_EINVAL


@pytest.mark.parametrize("n,seed", [(1, 0), (2, 0), (13, 1), (63, 2), (64, 3), (65, 4), (130, 5), (1024, 6)])
def test_tree_masks_hold_the_ancestors(n, seed):
    rng = np.random.default_rng(seed)
    parents = [int(rng.integers(-1, j)) if j else -1 for j in range(n)]
    if seed == 3:
        parents = list(range(-1, n - 1))                            # a chain
    mask, depth = ngg.tree_mask(parents)
    assert mask.shape == (n, (n + 63) // 64)
    bits = mask.view(np.uint64)
    for t in range(n):
        line, j = set(), t
        while j >= 0:
            line.add(j)
            j = parents[j]
        assert {j for j in range(64 * mask.shape[1]) if int(bits[t, j // 64]) >> (j % 64) & 1} == line
        assert depth[t] == len(line) - 1


def test_tree_mask_refuses(lib):
    for parents in ([0], [-1, 1], [-1, 2, 1], [-2], [], [-1] * 1025):
        with pytest.raises(ngg.NggError) as e:
            ngg.tree_mask(parents)
        assert e.value.status == ngg.NGG_EINVAL
    assert lib.ngg_tree_mask(None, 1, None, None) == ngg.NGG_EINVAL


def pages(**over):
    base = dict(k=16, v=16, k_exp=16, v_exp=16, n_pages=4, page_size=64, n_kv_heads=2, head_dim=64, dtype=ngg.NGG_FP8)
    base.update(over)
    return ngg.ngg_kv_pages(*[base[n] for n, _ in ngg.ngg_kv_pages._fields_])


@pytest.mark.parametrize("over,frag", [
    (dict(dtype=3), "dtype"), (dict(head_dim=48), "head_dim"), (dict(page_size=48), "page_size"), (dict(page_size=0), "page_size"),
    (dict(n_pages=0), "pages"), (dict(n_kv_heads=0), "key heads"), (dict(n_pages=1 << 30), "slot"), (dict(k=None), "null"), (dict(v=24), "aligned"),
    (dict(k_exp=None), "k_exp"), (dict(v_exp=8), "aligned"),
])
def test_pages_are_checked_by_every_call(lib, over, frag):
    p, st = pages(**over), (C.c_int64 * 4)(128, 64, 128, 64)
    a = ngg.ngg_tree_args()
    calls = [lambda: lib.ngg_kv_write(p, 16, 16, ngg.NGG_BF16, st, 16, 1, None, None, None),
             lambda: lib.ngg_kv_read(p, 16, 1, ngg.NGG_BF16, 16, 16, st, None), lambda: lib.ngg_tree_attention(p, a, 16, 1 << 30, None)]
    for call in calls:
        assert call() in (ngg.NGG_EINVAL, ngg.NGG_ECAPACITY) and frag in lib.ngg_last_error(None).decode()


def test_kv_bytes(lib):
    v, e = C.c_int64(-1), C.c_int64(-1)
    for dtype, size in ((ngg.NGG_F32, 4), (ngg.NGG_BF16, 2), (ngg.NGG_FP8, 1)):
        assert lib.ngg_kv_bytes(pages(dtype=dtype, k=None, v=None, n_pages=1 << 20), v, e) == ngg.NGG_OK
        assert v.value == (1 << 20) * 64 * 2 * 64 * size and e.value == ((1 << 20) * 64 * 2 if size == 1 else 0)
    assert lib.ngg_kv_bytes(None, v, e) == ngg.NGG_EINVAL


def test_cache_calls_refuse(lib):
    p, bf = pages(), pages(dtype=ngg.NGG_BF16)
    st = (C.c_int64 * 4)(128, 64, 128, 64)
    rope = ngg.ngg_rope(16, 16, 8, 64, 0)
    assert lib.ngg_kv_write(p, 16, 16, ngg.NGG_FP8, st, 16, 1, None, None, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(bf, 16, 16, ngg.NGG_F32, st, 16, 1, None, None, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(p, 16, 16, ngg.NGG_BF16, st, 16, -1, None, None, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(p, 16, 16, ngg.NGG_BF16, None, 16, 1, None, None, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(p, 16, 16, ngg.NGG_BF16, st, None, 1, None, None, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(p, None, 16, ngg.NGG_BF16, st, 16, 1, None, None, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(p, 16, 16, ngg.NGG_BF16, st, 16, 1, rope, None, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(p, 16, 16, ngg.NGG_BF16, st, 16, 1, ngg.ngg_rope(16, 16, 8, 66, 0), 16, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_read(bf, 16, 1, ngg.NGG_F32, 16, 16, st, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(p, None, None, ngg.NGG_BF16, st, None, 0, None, None, None) == ngg.NGG_OK       # nothing to do


def test_rotary_refuses(lib):
    rope, rows = ngg.ngg_rope(16, 16, 8, 64, 0), ngg.ngg_rotary_rows(16, 32, 128, 64, 128, 64, 2)
    ok = [rope, 16, 1, 64, ngg.NGG_BF16, rows, None, 0, None]
    for at, bad in ((0, None), (0, ngg.ngg_rope(None, 16, 8, 64, 0)), (0, ngg.ngg_rope(16, 16, 0, 64, 0)), (0, ngg.ngg_rope(16, 16, 8, 63, 0)),
                    (0, ngg.ngg_rope(16, 16, 8, 66, 0)), (1, None), (2, -1), (3, 1), (3, 2000), (4, ngg.NGG_FP8), (5, None),
                    (5, ngg.ngg_rotary_rows(16, 32, 128, 64, 128, 64, 0)), (5, ngg.ngg_rotary_rows(16, 16, 128, 64, 256, 64, 2)),
                    (6, ngg.ngg_rotary_rows(None, 32, 128, 64, 128, 64, 2))):
        args = list(ok)
        args[at] = bad
        assert lib.ngg_rotary(*args) == ngg.NGG_EINVAL, (at, bad)


def tree_args(**over):
    base = dict(q=16, out=16, lse=None, q_batch=0, q_token=256, q_head=64, out_batch=0, out_token=256, out_head=64, pages=16, pages_batch=4,
                context_lens=16, tree_lens=None, mask=None, mask_batch=0, mask_token=1, max_pages=4, batch=1, tree=5, n_heads=4,
                dtype=ngg.NGG_BF16, scale=0.125)
    base.update(over)
    return ngg.ngg_tree_args(*[base[n] for n, _ in ngg.ngg_tree_args._fields_])


@pytest.mark.parametrize("over", [
    dict(dtype=ngg.NGG_FP8), dict(batch=0), dict(batch=1025), dict(tree=0), dict(tree=1025), dict(n_heads=5), dict(n_heads=0), dict(n_heads=2048),
    dict(max_pages=0), dict(max_pages=1 << 26), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None),
    dict(pages=None), dict(context_lens=None),
])
def test_tree_attention_refuses(lib, over):
    assert lib.ngg_tree_attention(pages(), tree_args(**over), 16, 1 << 40, None) == ngg.NGG_EINVAL


def test_tree_attention_asks_for_its_workspace(lib):
    need = C.c_int64(0)
    # one sequence of many pages is split
    assert lib.ngg_tree_attention_workspace(pages(k=None), tree_args(max_pages=512), need) == ngg.NGG_OK and need.value > 0
    for ws, size in ((None, need.value), (16, need.value - 1), (24, need.value)):
        assert lib.ngg_tree_attention(pages(), tree_args(max_pages=512), ws, size, None) == ngg.NGG_EINVAL
    assert lib.ngg_tree_attention(pages(dtype=ngg.NGG_F32), tree_args(), 16, 1 << 40, None) == ngg.NGG_EINVAL
    assert lib.ngg_tree_attention_workspace(pages(), None, need) == ngg.NGG_EINVAL


def score_args(**over):
    base = dict(logits=16, row_stride=100, dtype=ngg.NGG_F32, n_rows=2, vocab=100, scale=1.0, targets=16, n_targets=1, top_n=3, logprobs=16,
                entropy=None, lse=None, top_logprobs=16, top_ids=16)
    base.update(over)
    return ngg.ngg_score_args(*[base[n] for n, _ in ngg.ngg_score_args._fields_])


@pytest.mark.parametrize("over", [
    dict(dtype=ngg.NGG_FP8), dict(n_rows=-1), dict(vocab=0), dict(top_n=-1), dict(top_n=65), dict(vocab=2), dict(n_targets=65), dict(n_targets=-1),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(logits=None), dict(logits=18), dict(targets=None), dict(logprobs=None),
    dict(top_ids=None), dict(top_logprobs=None),
])
def test_token_logprobs_refuses(lib, over):
    assert lib.ngg_token_logprobs(score_args(**over), 16, 1 << 40, None) == ngg.NGG_EINVAL
    assert lib.ngg_token_logprobs(None, 16, 1 << 40, None) == ngg.NGG_EINVAL
    assert lib.ngg_token_logprobs(score_args(n_rows=0, logits=None), None, 0, None) == ngg.NGG_OK
