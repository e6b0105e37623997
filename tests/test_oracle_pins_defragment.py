"""The oracle of the defragmentation on counts that do not fit the tables."""
import numpy as np
import pytest

from oracle import draft as od


@pytest.mark.parametrize("block", [0, 1, 2, 5, 6, 7])
def test_a_listed_block_that_counts_as_free_is_flagged(block):
    table = np.array([[0, 1, 6], [2, 5, 7]], dtype=np.int32)
    refs = np.zeros(10, dtype=np.int32)
    refs[table.ravel()] = 1
    assert od.defragment([], table, refs, np.array([20, 24]), 8)[3] == 0
    refs[block] = 0
    new_table, new_refs, used, flags = od.defragment([], table, refs, np.array([20, 24]), 8)
    assert flags == od.FLAG_POOL and used == 5 and new_refs[:5].all() and not new_refs[5:].any()
    assert new_table.ravel()[table.ravel().tolist().index(block)] == block
