"""Defragmentation of a pool whose counts do not fit its tables: a listed block that counts as free is reported
wherever it lies, below the number of used blocks (where a used one is moved over it) or behind it."""
import numpy as np
import pytest

from oracle import draft as od
from tests.test_gpu_kv_pages import Pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("block", [0, 1, 2, 5, 7])
def test_a_listed_block_that_counts_as_free_is_flagged(block, in_place):
    # Two sequences on blocks 0, 1, 6 and 2, 5, 7; the block in question loses its count, and 5 used ones are left.
    pool = Pool(2, 10, 2, 8, 64, 3, 4)
    pool.table[0, :3] = 0, 1, 6
    pool.table[1, :3] = 2, 5, 7
    at = np.argwhere(pool.table == block)[0]
    pool.refs[[0, 1, 2, 5, 6, 7]] = 1
    pool.lens[:2] = 20, 24
    pool.refs[block] = 0
    pool.upload()
    assert od.defragment([], pool.table, pool.refs, pool.lens, 8)[3] == od.FLAG_POOL
    pool.defragment(in_place, f"block {block}")      # (compares the flags, the tables, the counts and the pages)
    assert pool.table[tuple(at)] == block            # the entry is left as it is, though another block lies there now
    assert pool.refs[:5].all() and not pool.refs[5:].any()


def test_counts_that_fit_are_not_flagged():
    pool = Pool(1, 10, 1, 8, 64, 2, 4)
    pool.table[0, :3] = 9, 1, 6
    pool.refs[[9, 1, 6]] = 1
    pool.lens[0] = 17
    pool.upload()
    pool.defragment(True)
    assert pool.table[0, :3].tolist() == [2, 1, 0] and pool.refs.tolist() == [1, 1, 1] + [0] * 7
