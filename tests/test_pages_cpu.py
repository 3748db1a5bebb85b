"""Host-side checks of a cache of 4 bits and of the calls on a cache's pages: sizes, and the refusals that come before any device work."""
import ctypes as C
import os

import pytest

import paper_2411_03786_amd as ngg


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ngg.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return ngg.load_library()


def pages(**over):
    base = dict(k=16, v=16, k_exp=16, v_exp=16, n_pages=12, page_size=64, n_kv_heads=2, head_dim=64, dtype=ngg.NGG_FP4)
    base.update(over)
    return ngg.ngg_kv_pages(*[base[n] for n, _ in ngg.ngg_kv_pages._fields_])


def table(**over):
    base = dict(pages=16, pages_seq=5, lens=16, refs=16, n_seqs=3, max_pages=5, n_pages=12, page_size=64)
    base.update(over)
    return ngg.ngg_page_table(*[base[n] for n, _ in ngg.ngg_page_table._fields_])


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_bytes_of_four_bits(lib, hd):
    v, e = C.c_int64(-1), C.c_int64(-1)
    assert lib.ngg_kv_bytes(pages(head_dim=hd, k=None, v=None, n_pages=1 << 20), v, e) == ngg.NGG_OK
    assert v.value == (1 << 20) * 64 * 2 * hd // 2 and e.value == (1 << 20) * 64 * 2 * hd // 32


@pytest.mark.parametrize("over,frag", [(dict(head_dim=48), "head_dim"), (dict(k=None), "null"), (dict(v=24), "aligned"), (dict(k_exp=None), "k_exp"),
                                       (dict(v_exp=8), "aligned"), (dict(dtype=3), "dtype"), (dict(dtype=5), "dtype")])
def test_pages_of_four_bits_are_checked_by_every_call(lib, over, frag):
    p, st = pages(**over), (C.c_int64 * 4)(128, 64, 128, 64)
    for call in (lambda: lib.ngg_kv_write(p, 16, 16, ngg.NGG_BF16, st, 16, 1, None, None, None),
                 lambda: lib.ngg_kv_read(p, 16, 1, ngg.NGG_BF16, 16, 16, st, None), lambda: lib.ngg_tree_attention(p, ngg.ngg_tree_args(), 16, 1 << 30, None),
                 lambda: lib.ngg_kv_move(p, 1, 16, 16, 1, 1, 1, 1, None), lambda: lib.ngg_kv_copy(p, 1, 16, 16, None, 1, None)):
        assert call() == ngg.NGG_EINVAL and frag in lib.ngg_last_error(None).decode()


def test_four_bits_are_no_type_of_tokens(lib):
    st = (C.c_int64 * 4)(128, 64, 128, 64)
    for dtype in (ngg.NGG_FP4, ngg.NGG_FP8, 3):
        assert lib.ngg_kv_write(pages(), 16, 16, dtype, st, 16, 1, None, None, None) == ngg.NGG_EINVAL
        assert lib.ngg_kv_read(pages(), 16, 1, dtype, 16, 16, st, None) == ngg.NGG_EINVAL
    assert lib.ngg_kv_write(pages(), None, None, ngg.NGG_BF16, st, None, 0, None, None, None) == ngg.NGG_OK


def test_moves_and_copies_refuse(lib):
    for layers in (0, -1, 5, 7, 13, 1 << 17):                            # 12 pages
        assert lib.ngg_kv_move(pages(), layers, 16, 16, 1, 1, 1, 1, None) == ngg.NGG_EINVAL
        assert lib.ngg_kv_copy(pages(), layers, 16, 16, None, 1, None) == ngg.NGG_EINVAL
    for src, dst, lists, n in ((None, 16, 1, 1), (16, None, 1, 1), (16, 16, -1, 1), (16, 16, 1, -1), (16, 16, 1, 1025)):
        assert lib.ngg_kv_move(pages(), 3, src, dst, 1, 1, lists, n, None) == ngg.NGG_EINVAL
    for src, dst, n in ((None, 16, 1), (16, None, 1), (16, 16, -1)):
        assert lib.ngg_kv_copy(pages(), 3, src, dst, None, n, None) == ngg.NGG_EINVAL
    for lists, n in ((0, 4), (4, 0)):
        assert lib.ngg_kv_move(pages(), 4, None, None, 0, 0, lists, n, None) == ngg.NGG_OK
    assert lib.ngg_kv_copy(pages(), 4, None, None, None, 0, None) == ngg.NGG_OK


@pytest.mark.parametrize("over", [dict(pages=None), dict(lens=None), dict(refs=None), dict(n_seqs=0), dict(n_seqs=1025), dict(max_pages=0),
                                  dict(max_pages=1 << 25), dict(pages_seq=4), dict(pages_seq=0), dict(n_pages=0), dict(n_pages=1 << 26), dict(page_size=0), dict(page_size=48)])
def test_tables_are_checked_by_every_call(lib, over):
    t = table(**over)
    assert lib.ngg_pages_fork(t, 16, 16, 1, None) == ngg.NGG_EINVAL
    assert lib.ngg_pages_reserve(t, 16, 16, 16, 16, 16, 16, 1 << 40, None) == ngg.NGG_EINVAL
    assert lib.ngg_pages_release(t, None, None) == ngg.NGG_EINVAL


def test_struct_size_matches_the_header():
    assert C.sizeof(ngg.ngg_page_table) == 4 * 8 + 4 * 4


def test_table_calls_refuse(lib):
    need = C.c_int64(0)
    assert lib.ngg_pages_reserve_workspace(table(), need) == ngg.NGG_OK and need.value >= 12 * 4
    assert lib.ngg_pages_reserve_workspace(None, need) == ngg.NGG_EINVAL and lib.ngg_pages_reserve_workspace(table(), None) == ngg.NGG_EINVAL
    ok = [table(), 16, 16, 16, 16, 16, 16, need.value, None]
    for at, bad in ((0, None), (1, None), (2, None), (3, None), (4, None), (5, None), (6, None), (6, 24), (7, need.value - 1)):
        args = list(ok)
        args[at] = bad
        assert lib.ngg_pages_reserve(*args) == ngg.NGG_EINVAL, at
    for sources, targets, n in ((None, 16, 1), (16, None, 1), (16, 16, -1), (16, 16, 1025)):
        assert lib.ngg_pages_fork(table(), sources, targets, n, None) == ngg.NGG_EINVAL
    assert lib.ngg_pages_fork(table(), None, None, 0, None) == ngg.NGG_OK
    assert lib.ngg_pages_release(None, None, None) == ngg.NGG_EINVAL


def test_a_pool_of_layers_refuses():
    for layers in (0, -2):
        with pytest.raises(ValueError):
            ngg.KVPages(4, 64, 2, 64, "fp4", layers=layers)
    with pytest.raises(ValueError):
        ngg.KVPages(4, 64, 2, 64, "int4")
    with pytest.raises(ngg.NggError):
        ngg.KVPages(1 << 20, 64, 2, 64, "fp4", layers=64)                # slots of all layers pass 32 bits
