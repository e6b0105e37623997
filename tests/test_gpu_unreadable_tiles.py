"""Whole tiles of blocks whose ids are out of range: no copy brings their zeros, the copying warp writes them, and
they have to be there when the tile is handed on.  The tiles before leave large values in the same slots."""
import numpy as np
import pytest
import torch

from oracle import draft as od
from paper_2409_04992_b200 import binding
from tests import gpu_util as gu
from tests.test_gpu_tree_attention import Case, compare, run

pytestmark = pytest.mark.gpu
LENS = [900, 300, 1300, 129]


def spoil(table, tokens, unreadable):
    """The table with the entries of positions [from, to) of each sequence out of range."""
    broken = table.copy()
    for b, (start, end) in enumerate(unreadable):
        for e in range(start // tokens, -(-end // tokens)):
            broken[b, e] = (-1, 1 << 30, -(1 << 31), len(table) * 10000)[e % 4]
    return broken


@pytest.mark.parametrize("tokens", [16, 32, 48, 64, 128])
@pytest.mark.parametrize("dim,nodes,group", [(128, 5, 1), (128, 40, 1), (128, 40, 3), (64, 6, 2), (64, 40, 1), (256, 20, 1), (256, 30, 3)])
def test_trees(tokens, dim, nodes, group):
    unreadable = [(256, 768), (0, 128), (384, 1280), (0, 0)]
    c = Case("paged", tokens, 2 * group, 2, dim, nodes, LENS, seed=dim + tokens)
    c.v[np.isfinite(c.v)] *= np.float16(50)
    broken = spoil(c.table, tokens, unreadable)
    first = None
    for _ in range(10):
        got, lse, flags = run(c, table=broken)
        assert flags == od.FLAG_BLOCK_RANGE
        first = first or (got, lse)
        assert np.array_equal(got.view(np.uint16), first[0].view(np.uint16)) and np.array_equal(lse, first[1])
    for cache in (c.k, c.v):
        cache[c.table[broken != c.table]] = 0
    compare(got, lse, od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale), "unreadable tiles", max(LENS))


@pytest.mark.parametrize("tokens", [16, 32, 64, 128])
@pytest.mark.parametrize("dim,group", [(128, 4), (256, 2), (64, 4)])
def test_grouped_steps(tokens, dim, group):
    c = Case("paged", tokens, 2 * group, 2, dim, 1, LENS, seed=dim + tokens)
    broken = spoil(c.table, tokens, [(256, 768), (0, 128), (384, 1280), (0, 0)])
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    q, k, v, table, lens = (put(a) for a in (c.q, c.k, c.v, broken, c.lens))
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
    ws = torch.empty(binding.grouped_workspace_bytes(len(LENS), 1, 2 * group, 2, dim, max(LENS)), dtype=torch.uint8, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    for cache in (c.k, c.v):
        cache[c.table[broken != c.table]] = 0
    want, want_lse, _, _ = od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale)
    for _ in range(10):
        binding.decode_attention_grouped(out, lse, q, k, v, table, lens, max(LENS), c.scale, ws, flags)
        torch.cuda.synchronize()
        assert int(flags.item()) == od.FLAG_BLOCK_RANGE
        assert np.abs(out.cpu().numpy().astype(np.float64) - want).max() <= gu.MAX_ABS
        assert np.allclose(lse.cpu().numpy(), want_lse, atol=gu.LSE_ATOL, rtol=gu.LSE_RTOL)
