"""Verification in distribution: with children drawn independently from the draft's distributions, what is emitted
follows the target's, after any number of rejections and on every level.  A frequency over n draws has a standard
deviation of at most 0.5 / sqrt(n); five of them are allowed."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify import run

pytestmark = pytest.mark.gpu


def bound(n):
    return 2.5 / np.sqrt(n)


def choose(rng, rows):
    """One draw per row of probabilities."""
    edges = rows.cumsum(-1)
    return (rng.random(rows.shape[:-1])[..., None] * edges[..., -1:] >= edges).sum(-1).clip(0, rows.shape[-1] - 1).astype(np.int32)


@pytest.mark.parametrize("nodes", [3, 8, 64])
@pytest.mark.parametrize("q", [[0.1, 0.1, 0.2, 0.3, 0.3], [0.002, 0.008, 0.01, 0.38, 0.6]])
def test_a_star_of_any_width(nodes, q):
    """The second draft hardly ever proposes what the target wants: some ten rejections before a child is taken."""
    rng, steps = np.random.default_rng(nodes), 100000
    p, q = np.array([0.5, 0.2, 0.15, 0.1, 0.05]), np.array(q)
    tokens = choose(rng, np.broadcast_to(q, (steps, nodes, 5)))
    parents = np.zeros((steps, nodes), dtype=np.int32)
    parents[:, 0] = -1
    tile = lambda x: torch.from_numpy(np.tile(x.astype(np.float32), (steps, nodes, 1)))  # noqa: E731
    _, lens, said, flags = run(tile(p), tile(q), tokens, parents, None, rng.random((steps, nodes), dtype=np.float32))
    assert flags == 0
    assert np.abs(np.bincount(said[:, 0], minlength=5) / steps - p).max() < bound(steps)
    # behind a child that was taken, the next token is drawn from its row
    taken = lens == 2
    assert taken.any() and np.abs(np.bincount(said[taken, 1], minlength=5) / taken.sum() - p).max() < bound(taken.sum())


def test_trees_whose_rows_depend_on_the_tokens_before():
    """Three levels of three children each (40 nodes); a node's distributions are those of its token, so the joint
    frequencies of consecutive tokens tell whether the rows of the taken nodes decided."""
    rng, steps, V = np.random.default_rng(5), 60000, 4
    table_p, table_q = (rng.dirichlet(np.full(V, 1.5), V) for _ in range(2))
    parents = np.array([-1] + [(t - 1) // 3 for t in range(1, 40)], dtype=np.int32)
    tokens = np.zeros((steps, 40), dtype=np.int32)
    for t in range(1, 40):
        tokens[:, t] = choose(rng, table_q[tokens[:, parents[t]]])
    target, draft = (torch.from_numpy(x[tokens].astype(np.float32)) for x in (table_p, table_q))
    path, lens, said, flags = run(target, draft, tokens, np.tile(parents, (steps, 1)), None, rng.random((steps, 40), dtype=np.float32))
    assert flags == 0
    assert np.abs(np.bincount(said[:, 0], minlength=V) / steps - table_p[0]).max() < bound(steps)
    for level in (1, 2, 3):
        there = lens > level
        assert there.sum() > 1000
        for before in range(V):
            mine = there & (said[:, level - 1] == before)
            n = mine.sum()
            if n > 100:
                assert np.abs(np.bincount(said[mine, level], minlength=V) / n - table_p[before]).max() < bound(n), (level, before)
