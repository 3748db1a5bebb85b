"""Moves, copies and page lists beyond test_gpu_pages: fewer units than entries, long lists, many sequences that grow at once, what a call lacks.
Needs an MI355X.  Everything here is exact."""
import numpy as np
import pytest
import torch

import paper_2411_03786_amd as ngg
from test_gpu_operators import ints
from test_gpu_pages import CACHES, Lists, Pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_moves_of_more_entries_than_units(cache, hd):
    """One key head has as few as one unit of a kind: the lanes that have none still hold entries."""
    p = Pool(cache, 2, 3, 32, 1, hd)
    rng = np.random.default_rng(hd)
    for n in range(1, 17):
        mine = rng.permutation(p.n)
        src, dst = mine[:n], rng.permutation(mine[:2 * n])[:n]
        src[rng.random(n) < 0.2] = -1
        p.kv.move(ints(src), ints(dst))
        p.move([src], [dst])
        p.check()
