"""The workspace that tree attention asks for, without a GPU: it follows from the work there can be, not from the
GPU's size alone, and grows with it."""
import pytest

from paper_2409_04992_b200 import binding, build

TILE, ITEM_COST = 128, 4          # tokens per tile; what an item weighs more than its tiles


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.load()


@pytest.mark.parametrize("batch,nodes,q_heads,kv_heads,dim,longest", [
    (1, 32, 64, 8, 128, 128), (1, 8, 40, 40, 128, 128), (1, 128, 8, 1, 128, 300), (2, 64, 2, 1, 256, 1000), (1, 40, 1, 1, 64, 1)])
def test_little_work_asks_for_little(batch, nodes, q_heads, kv_heads, dim, longest):
    """A piece is a unit of the items' weight at least and leaves two partial results, each of an item's rows (at most
    two blocks of 128), at most.  The warp-level form's, which the same workspace has to hold, are a chunk's rows each, of 64
    tokens at least."""
    group = q_heads // kv_heads
    rows = nodes * group
    items = batch * kv_heads * -(-rows // (TILE // group * group))
    pieces = min(items * (-(-longest // TILE) + ITEM_COST), 148) + 1
    tcgen05 = 2 * pieces * min(rows, 2 * TILE) * (dim + 1) * 4 + 8 * items
    warp_level = batch * kv_heads * -(-longest // 64) * rows * (dim + 1) * 4
    assert 0 < binding.tree_workspace_bytes(batch, nodes, q_heads, kv_heads, dim, longest) <= max(tcgen05, warp_level) + 2048


@pytest.mark.parametrize("nodes,q_heads,kv_heads,dim", [(8, 40, 40, 128), (64, 40, 40, 128), (32, 64, 8, 128), (25, 15, 5, 256), (33, 6, 6, 64)])
def test_it_grows_with_the_batch_and_the_longest_length(nodes, q_heads, kv_heads, dim):
    """A workspace for the most that a program will have is enough for less."""
    lengths = [1, 100, 128, 129, 1000, 5000, 30000]
    sizes = [[binding.tree_workspace_bytes(b, nodes, q_heads, kv_heads, dim, n) for n in lengths] for b in (1, 2, 7, 16)]
    assert all(0 < s <= sizes[-1][-1] for row in sizes for s in row)
