"""The speculative-decoding oracle against closed forms, so that what the kernels are held to is itself
held to something."""
import numpy as np

from oracle import draft as od


def test_ancestors_and_their_words():
    see = od.ancestor_mask([-1, 0, 0, 1, 3, -1], 6, 6)
    assert [set(np.nonzero(r)[0]) for r in see] == [{0}, {0, 1}, {0, 2}, {0, 1, 3}, {0, 1, 3, 4}, {5}]
    words = od.pack_mask(np.eye(70, dtype=bool))
    assert words.shape == (70, 2) and words[3, 0] == 8 and words[66, 1] == 4 and words[63, 0] == np.iinfo(np.int64).min


def test_tree_attention_of_equal_keys_is_the_mean_of_what_is_seen():
    rng = np.random.default_rng(0)
    k = np.tile(rng.standard_normal(8), (1, 2, 10, 1))
    v = rng.standard_normal((1, 2, 10, 8))
    q = rng.standard_normal((1, 3, 4, 8))
    see = od.ancestor_mask([-1, 0, 0], 3, 3)[None]
    out, lse, size, _ = od.tree_attention(q, k, v, None, [9], [3], see, 0.3)
    for t, seen in enumerate(([*range(7)], [*range(8)], [*range(7), 8])):
        assert set(seen) == set(range(6)) | {6 + j for j in range(3) if see[0, t, j]}
        for h in range(4):
            assert np.allclose(out[0, t, h], v[0, h // 2, seen].mean(0))
            assert np.isclose(lse[0, t, h], 0.3 * k[0, 0, 0] @ q[0, t, h] + np.log(len(seen)))
    # a page table is only another way to lay the rows out
    table = np.array([[2, 0, 1]], dtype=np.int32)
    pages = np.zeros((3, 2, 4, 8))
    for i in range(10):
        pages[table[0, i // 4], :, i % 4] = v[0, :, i]
    assert np.array_equal(od.rows_of(pages, 0, 10, table), v[0])


def test_verification_follows_the_target():
    """Enumerated, not sampled: over a fine grid of uniforms the first emitted token's frequencies are p,
    for one and for two independent drafts."""
    p, q = np.array([0.5, 0.3, 0.2]), np.array([0.2, 0.2, 0.6])
    grid = (np.arange(60) + 0.5) / 60
    for drafts in (1, 2):
        mass = np.zeros(3)
        for x in np.ndindex(*(3,) * drafts):
            for us in np.ndindex(*(12,) * drafts):
                u = np.array([(i + 0.5) / 12 for i in us])
                B = len(grid)
                nodes = 1 + drafts
                target, draft = np.tile(p, (B, nodes, 1)), np.tile(q, (B, nodes, 1))
                tokens = np.tile([0, *x], (B, 1))
                parents = np.tile([-1] + [0] * drafts, (B, 1))
                uniforms = np.concatenate([grid[:, None], np.tile(u, (B, 1))], 1)
                _, _, said, _ = od.verify(target, draft, tokens, parents, [nodes] * B, uniforms)
                mass += np.bincount(said[:, 0], minlength=3) * np.prod(q[list(x)]) / 12 ** drafts / B
        assert np.abs(mass - p).max() < 0.03 * drafts          # the grids' steps: 1/12 and 1/60


def test_one_hot_drafts_and_a_dry_residual():
    p = np.array([[[0.6, 0.4, 0.0], [0.0, 0.0, 1.0]]])
    run = lambda u, x: od.verify(p, None, np.array([[0, x]]), np.array([[-1, 0]]), [2], np.array([[0.5, u]]))  # noqa: E731
    path, lens, said, flags = run(0.59, 0)
    assert path.tolist() == [[0, 1]] and lens.tolist() == [2] and said.tolist() == [[0, 2]] and flags == 0
    path, lens, said, _ = run(0.61, 0)                          # rejected: token 0 is out, 1 is all that is left
    assert lens.tolist() == [1] and said.tolist() == [[1, -1]]
    half = p * 0.5                                              # p <= q everywhere: the residual is empty, p stays
    _, _, said, _ = od.verify(half, p, np.array([[0, 0]]), np.array([[-1, 0]]), [2], np.array([[0.7, 0.9]]))
    assert said.tolist() == [[1, -1]]


def test_pool_histories_keep_counts_and_contents():
    """Whatever happens to the pool, a sequence reads back what was written to it."""
    rng = np.random.default_rng(2)
    B, M, T, P = 5, 4, 8, 14
    cache = np.zeros((P, 1, T, 1))
    table, refs, lens = np.full((B, M), -1), np.zeros(P, dtype=np.int64), np.zeros(B, dtype=np.int32)
    held = [[] for _ in range(B)]
    stamp = 0
    for _ in range(300):
        kind = rng.integers(0, 4)
        if kind == 0:
            s, d = rng.integers(0, B, 2)
            if not od.fork(table, refs, lens, [s], [d], T):
                held[d] = list(held[s])
        elif kind < 3:
            want = np.where(rng.random(B) < 0.5, lens, rng.integers(0, M * T + 1, B))
            new, _ = od.resize([cache], table, refs, lens, want, T)
            for b in range(B):
                held[b] = held[b][:new[b]]
                while len(held[b]) < new[b]:
                    i, stamp = len(held[b]), stamp + 1
                    assert refs[table[b, i // T]] == 1
                    cache[table[b, i // T], 0, i % T] = stamp
                    held[b].append(stamp)
            lens = new
        else:
            table, refs, used, flags = od.defragment([cache], table, refs, lens, T)
            assert flags == 0 and (refs[:used] > 0).all() and (refs[used:] == 0).all()
        for b in range(B):
            assert [cache[table[b, i // T], 0, i % T, 0] for i in range(lens[b])] == held[b]
        count = np.zeros(P, dtype=np.int64)
        for b in range(B):
            for e in range(od.blocks_for(lens[b], T)):
                count[table[b, e]] += 1
        assert np.array_equal(count, refs)


def test_keep_path_moves_and_refuses():
    k = np.arange(12).reshape(1, 1, 12, 1).copy()
    new, flags = od.keep_path([k], np.array([[0, 2, 5, -1, -1, -1]]), [3], [6], [10], None)
    assert new.tolist() == [7] and flags == 0
    assert k.ravel().tolist() == [0, 1, 2, 3, 4, 6, 9, 7, 8, 9, 10, 11]
    new, flags = od.keep_path([k], np.array([[0, 2, 2]]), [3], [3], [10], None)
    assert new.tolist() == [10] and flags == od.FLAG_TREE_RANGE
