"""Corners of the operators' C entry points that need no GPU."""
import os

import pytest

import paper_2411_03786_amd as ngg


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ngg.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return ngg.load_library()


def test_rotary_of_no_tokens_needs_no_rows(lib):
    """Empty tensors have no address, so input and output are alike without being in place: slices of something wider, packed outputs."""
    rope, rows = ngg.ngg_rope(16, 16, 8, 64, 0), ngg.ngg_rotary_rows(None, None, 256, 64, 128, 64, 2)
    assert lib.ngg_rotary(rope, None, 0, 64, ngg.NGG_BF16, rows, None, 0, None) == ngg.NGG_OK
    assert lib.ngg_rotary(rope, None, 0, 64, ngg.NGG_BF16, rows, rows, 1, None) == ngg.NGG_OK
    assert lib.ngg_rotary(rope, 16, 1, 64, ngg.NGG_BF16, rows, None, 0, None) == ngg.NGG_EINVAL
    same = ngg.ngg_rotary_rows(16, 16, 256, 64, 128, 64, 2)
    assert lib.ngg_rotary(rope, 16, 1, 64, ngg.NGG_BF16, same, None, 0, None) == ngg.NGG_EINVAL
