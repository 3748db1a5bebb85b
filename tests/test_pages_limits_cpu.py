"""Sizes of a pool of pages that 32 bits do not hold: no GPU."""
import os

import pytest

import paper_2411_03786_amd as ngg


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(ngg.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()


@pytest.mark.parametrize("size", [dict(n_pages=(1 << 20) + 1, layers=4096), dict(n_pages=(1 << 32) + 8), dict(page_size=(1 << 32) + 32), dict(n_kv_heads=(1 << 32) + 1),
                                  dict(head_dim=(1 << 32) + 64), dict(n_pages=-(1 << 32) + 8)])
def test_sizes_beyond_32_bits_are_refused(size):
    """Cut to 32 bits these would be pools of a few pages, whose layers would be taken for larger ones than their memory."""
    with pytest.raises(ValueError, match="32 bits"):
        ngg.KVPages(**{**dict(n_pages=8, page_size=32, n_kv_heads=1, head_dim=64, cache="fp4"), **size})
