"""Huge logits in the warp-level form of tree attention, which head size 64 with few rows, pages whose size
tcgen05 does not take and more than 128 heads a group get by default: past 2^24 a reference and the
weights' scale cannot be added exactly any more, and a weight that is off by that leaves the range of fp16.

The tolerances are the arithmetic's: a logit is off by at most dim 2^-22 of the largest sum of magnitudes
a row meets (see test_gpu_tree_attention), so a row whose two largest logits are further apart than twice
that, and 40 more for the exponential to vanish, is the value row of the largest one, rounded."""
import numpy as np
import pytest
import torch

from oracle import draft as od
from paper_2409_04992_b200 import binding
from tests.test_gpu_tree_attention import Case, run

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=[0, 1], ids=["automatic", "warp-mma"])
def path(request):
    binding.set_grouped_path(request.param)
    yield request.param
    binding.set_grouped_path(0)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("layout,tokens,dim,nodes,group", [
    ("contiguous", 0, 64, 8, 1), ("paged", 48, 64, 8, 2), ("contiguous", 0, 64, 1, 1), ("paged", 48, 128, 8, 1), ("paged", 48, 128, 40, 1),
    ("paged", 80, 256, 20, 1), ("contiguous", 0, 128, 2, 130)])
@pytest.mark.parametrize("reach", [11.0, 13.0])
def test_the_largest_logit_wins(layout, tokens, dim, nodes, group, sign, reach):
    c = Case(layout, tokens, group, 1, dim, nodes, [300, 140], seed=15)
    c.scale *= sign
    for b, n in enumerate(c.lens):
        sizes = 2.0 ** np.random.default_rng(b).uniform(-1, reach, n)
        for i in range(n):
            where = (b, slice(None), i) if c.table is None else (c.table[b, i // tokens], slice(None), i % tokens)
            c.k[where] = np.sign(c.k[where].astype(np.float32)) * 4 * sizes[i]
    c.q = (np.sign(c.q.astype(np.float32)) * 2.0 ** np.random.default_rng(5).uniform(4, 14, c.q.shape[:3])[..., None]).astype(np.float16)
    want = od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale)
    got, lse, flags = run(c)
    assert flags == 0 and np.isfinite(got).all() and np.isfinite(lse).all()
    assert want[3].max() > 2.0 ** 27
    assert (np.abs(lse - want[1]) <= dim * 2.0 ** -22 * want[3] + 16).all()
    clear = 0
    for b, n in enumerate(c.lens):
        k = od.rows_of(c.k, b, n, c.table)[0]
        for t in range(c.trees[b]):
            seen = [*range(n - c.trees[b]), *(n - c.trees[b] + j for j in range(c.trees[b]) if c.see[b, t, j])]
            for h in range(group):
                s = np.sort(k[seen] @ c.q[b, t, h].astype(np.float64) * c.scale)
                if s[-1] - s[-2] > 2 * dim * 2.0 ** -22 * want[3][b, t, h] + 40:
                    clear += 1
                    assert np.abs(got[b, t, h] - want[0][b, t, h]).max() <= 2.0 ** -10 * np.abs(want[0][b, t, h]).max()
    assert clear > 0


@pytest.mark.parametrize("top", [2 ** 20, 2 ** 24 - 64, 2 ** 24 + 64])
def test_small_steps_under_a_large_logit(top):
    """Logits of 2^20 to 2^24 that are 4, 200 and 4000 apart, whole numbers that 32 bits hold: what decides the
    weights is their differences, and those are exact.  The row is a mean of two value rows; its share of the second
    is read back from 64 dims, each rounded by at most 2^-11 of a value of a few units (2^-9 allowed)."""
    q, below = np.zeros(64), np.array([0, 4, 200, 4000])
    q[:3] = 2.0 ** 14, 2.0 ** 4, 1.0
    k, rest = np.zeros((4, 64)), top - below
    for i, step in enumerate(q[:3]):
        k[:, i] = rest // step
        rest = rest % step
    c = Case("contiguous", 0, 1, 1, 64, 1, [4], seed=3)
    c.scale = 1.0
    c.q[0, 0, 0], c.k[0, 0, :4] = q, k
    c.see[:] = True
    assert np.array_equal(c.k[0, 0, :4].astype(np.float64) @ c.q[0, 0, 0].astype(np.float64), top - below)
    got, lse, flags = run(c)
    assert flags == 0 and np.isfinite(got).all()
    first, second = c.v[0, 0, 0].astype(np.float64), c.v[0, 0, 1].astype(np.float64)
    share = ((got[0, 0, 0].astype(np.float64) - first) @ (second - first)) / ((second - first) @ (second - first))
    assert abs(share - np.exp(-4.0) / (1 + np.exp(-4.0))) < 2.0 ** -9
    assert abs(lse[0, 0, 0] - top) <= 2.0 ** -22 * top
