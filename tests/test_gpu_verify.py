"""Verification of draft trees: every path and token equal to a plain loop's in 64 bits, for every
type, odd vocabularies and alignments, and the ancestors' masks."""
import numpy as np
import pytest
import torch

from oracle import draft as od
from paper_2409_04992_b200 import binding

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def random_parents(rng, nodes, shape):
    t = np.arange(nodes)
    back = {"mixed": rng.geometric(0.4, nodes), "chain": np.ones(nodes, dtype=int), "star": t,
            "pairs": t - (t - 1) // 2}[shape]
    return np.where(t == 0, -1, t - np.clip(back, 1, np.maximum(t, 1))).astype(np.int32)


def make(seed, batch, nodes, vocab, dtype, shape="mixed", noise=0.5, sharp=3.0):
    rng = np.random.default_rng(seed)
    logits = sharp * rng.standard_normal((batch, nodes, vocab))
    soft = lambda x: np.exp(x - x.max(-1, keepdims=True)) / np.exp(x - x.max(-1, keepdims=True)).sum(-1, keepdims=True)  # noqa: E731
    target = torch.from_numpy(soft(logits)).to(dtype)
    draft = torch.from_numpy(soft(logits + noise * rng.standard_normal(logits.shape))).to(dtype)
    parents = np.stack([random_parents(rng, nodes, shape) for _ in range(batch)])
    tokens = np.zeros((batch, nodes), dtype=np.int32)
    for b in range(batch):
        for t in range(nodes):
            p = draft[b, max(parents[b, t], 0)].double().numpy()
            tokens[b, t] = rng.choice(vocab, p=p / p.sum())
    uniforms = rng.random((batch, nodes), dtype=np.float32)
    return target, draft, tokens, parents, uniforms


def run(target, draft, tokens, parents, tree_lens, uniforms, stream=None):
    B, T, _ = target.shape
    new = lambda *s: torch.full(s, -9, dtype=torch.int32, device="cuda")  # noqa: E731
    path, lens, said, flags = new(B, T), new(B), new(B, T), torch.zeros(1, dtype=torch.int32, device="cuda")
    put = lambda a: None if a is None else (a if isinstance(a, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(a))).cuda()  # noqa: E731
    binding.verify_tree(path, lens, said, put(target), put(draft), put(tokens), put(parents), put(tree_lens), put(uniforms),
                        flags, stream)
    torch.cuda.synchronize()
    return path.cpu().numpy(), lens.cpu().numpy(), said.cpu().numpy(), int(flags.item())


def check(target, draft, tokens, parents, tree_lens, uniforms):
    got = run(target, draft, tokens, parents, tree_lens, uniforms)
    nodes = np.full(target.shape[0], target.shape[1]) if tree_lens is None else tree_lens
    want = od.verify(target.double().cpu().numpy(), None if draft is None else draft.double().cpu().numpy(), tokens, parents,
                     nodes, uniforms)
    for g, w, name in zip(got, want, ("path", "path_lens", "out_tokens", "flags")):
        assert np.array_equal(g, w), f"{name}\n{g}\n{w}"
    return want


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("batch,nodes,vocab,shape", [
    (3, 1, 1, "mixed"), (5, 2, 2, "chain"), (4, 7, 31, "mixed"), (3, 33, 257, "pairs"), (2, 64, 1000, "mixed"),
    (2, 65, 4099, "star"), (2, 128, 515, "mixed"), (1, 8, 32000, "mixed"), (2, 5, 50257, "star"), (2, 3, 100003, "star"), (1, 4, 131073, "pairs")])
def test_trees(dtype, batch, nodes, vocab, shape):
    for seed in range(3):
        target, draft, tokens, parents, uniforms = make(seed, batch, nodes, vocab, dtype, shape)
        check(target, draft, tokens, parents, None, uniforms)
        check(target, None, tokens, parents, None, uniforms)
        lens = np.array([(nodes * (b + 1)) // batch if b else 0 for b in range(batch)], dtype=np.int32)
        check(target, draft, tokens, parents, lens, uniforms)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_rows_of_a_padded_vocabulary(dtype):
    target, draft, tokens, parents, uniforms = make(5, 3, 6, 1003, dtype)
    wide = [torch.full((3, 6, 1017), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    for w, p in zip(wide, (target, draft)):
        w[:, :, :1003] = p.cuda()
    got = run(wide[0][:, :, :1003], wide[1][:, :, :1003], tokens, parents, None, uniforms)
    want = od.verify(target.double().numpy(), draft.double().numpy(), tokens, parents, [6] * 3, uniforms)
    for g, w in zip(got, want):
        assert np.array_equal(g, w)


def test_borders_and_ties():
    # u q Z against w where the two are equal: not taken; one step below: taken
    target = torch.tensor([[[0.25, 0.75], [0.5, 0.5]]])
    draft = torch.tensor([[[0.5, 0.5], [0.5, 0.5]]])
    tokens, parents = np.array([[0, 0]], dtype=np.int32), np.array([[-1, 0]], dtype=np.int32)
    half = np.float32(0.5)
    for u, count in ((half, 1), (np.nextafter(half, np.float32(0)), 2)):
        path, lens, said, _ = check(target, draft, tokens, parents, None, np.array([[0.0, u]], dtype=np.float32))
        assert lens[0] == count
    # the running sum has to exceed u_0 times the total: 0.25 of (0.25, 0.75) is not below 0.25
    one = np.array([[0]], dtype=np.int32)
    for u, token in ((0.0, 0), (np.nextafter(np.float32(0.25), np.float32(0)), 0), (0.25, 1), (1 - 2.0 ** -24, 1)):
        _, _, said, _ = check(target[:, :1], None, one, one - 1, None, np.array([[u]], dtype=np.float32))
        assert said[0, 0] == token
    # zeros around the only token
    p = torch.zeros(1, 1, 999)
    p[0, 0, 640] = 0.125
    for u in (0.0, 0.5, 1 - 2.0 ** -24):
        _, _, said, _ = check(p, None, one, one - 1, None, np.array([[u]], dtype=np.float32))
        assert said[0, 0] == 640


def test_equal_distributions_and_repeated_tokens():
    target, _, tokens, parents, uniforms = make(9, 4, 12, 130, torch.float32, "star")
    check(target, target, tokens, parents, None, uniforms)              # u q < p always: the first child is taken
    # a rejected child of the same distribution (p = q where w has no more left): the residual is empty
    zero = target.clone()
    zero[:, :, tokens[:, 1].max()] = 0
    uniforms[:] = np.float32(1 - 2.0 ** -24)
    check(zero, target, tokens, parents, None, uniforms)
    tokens[:, 1:] = tokens[:, 1:2]                                       # all siblings alike
    check(target, None, tokens, parents, None, uniforms)
    # p nowhere above q: every residual is empty, w stays p
    small = target * 0.25
    check(small, target, tokens, parents, None, uniforms)


def test_values_that_are_no_probabilities():
    target, draft, tokens, parents, uniforms = make(11, 6, 9, 77, torch.float32)
    target[0, :, ::3] = float("nan")
    target[1, :, 5] = float("inf")
    target[2, :, ::2] *= -1
    target[3] = 0
    draft[4, :, ::2] = float("nan")
    draft[5, :, 7] = float("inf")
    want = check(target, draft, tokens, parents, None, uniforms)
    assert want[3] == od.FLAG_TREE_RANGE and want[2][3, 0] == -1
    uniforms[:, 0] = np.nan                                              # no order against NaN: the last with any weight
    got = run(target, draft, tokens, parents, None, uniforms)
    assert np.all(got[2][:3, 0] >= 0)


def test_trees_that_are_none():
    target, draft, tokens, parents, uniforms = make(13, 5, 8, 50, torch.float16, "chain")
    parents[0, 3] = 3
    parents[1, 2] = -2
    tokens[2, 1] = 50
    tokens[3, 4] = -1
    uniforms[:] = 0                                                      # would take every child
    want = check(target, draft, tokens, parents, None, uniforms)
    assert want[3] == od.FLAG_TREE_RANGE and want[1].tolist() == [3, 2, 1, 4, 8]
    want = check(target, draft, tokens, parents, np.array([9, -1, 0, 8, 1], dtype=np.int32), uniforms)
    assert want[1].tolist() == [0, 0, 0, 4, 1]


def test_the_emitted_tokens_follow_the_target():
    """Two drafts a step from q; the first emitted token must be distributed as p.  200000 steps of one
    64-node star: with V = 5 each frequency's deviation is at most 0.5 / sqrt(200000) = 1.1e-3 (one
    standard deviation); five of them are allowed."""
    rng = np.random.default_rng(17)
    p, q, steps = np.array([0.5, 0.2, 0.15, 0.1, 0.05]), np.array([0.1, 0.1, 0.2, 0.3, 0.3]), 200000
    target = torch.from_numpy(np.tile(p, (steps, 3, 1))).float()
    draft = torch.from_numpy(np.tile(q, (steps, 3, 1))).float()
    tokens = rng.choice(5, (steps, 3), p=q).astype(np.int32)
    parents = np.tile(np.array([-1, 0, 0], dtype=np.int32), (steps, 1))
    _, _, said, flags = run(target, draft, tokens, parents, None, rng.random((steps, 3), dtype=np.float32))
    assert flags == 0
    assert np.abs(np.bincount(said[:, 0], minlength=5) / steps - p).max() < 5.5e-3


def test_other_streams_graphs_and_refusals():
    target, draft, tokens, parents, uniforms = make(19, 3, 10, 3001, torch.bfloat16)
    want = check(target, draft, tokens, parents, None, uniforms)
    side = torch.cuda.Stream()
    got = run(target, draft, tokens, parents, None, uniforms, side)
    assert all(np.array_equal(g, w) for g, w in zip(got, want))
    dev = [target.cuda(), draft.cuda(), torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda()]
    u = torch.from_numpy(uniforms).cuda()
    out = [torch.zeros(3, 10, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"),
           torch.zeros(3, 10, dtype=torch.int32, device="cuda")]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.verify_tree(*out, dev[0], dev[1], dev[2], dev[3], None, u)
    for seed in (1, 2):
        fresh = np.random.default_rng(seed).random((3, 10), dtype=np.float32)
        u.copy_(torch.from_numpy(fresh))
        graph.replay()
        torch.cuda.synchronize()
        want = od.verify(target.double().numpy(), draft.double().numpy(), tokens, parents, [10] * 3, fresh)
        assert all(np.array_equal(g.cpu().numpy(), w) for g, w in zip(out, want))
    with pytest.raises(binding.InstInferError):
        binding.verify_tree(*out, dev[0].cpu(), dev[1].cpu(), dev[2], dev[3], None, u)       # not on this device
    for bad in (dict(a=dev[0].double()), dict(b=dev[1].float()), dict(b=dev[1][:, :, :3000]), dict(a=dev[0].transpose(0, 1))):
        with pytest.raises(binding.InstInferError):
            binding.verify_tree(*out, bad.get("a", dev[0]), bad.get("b", dev[1]), dev[2], dev[3], None, u)


@pytest.mark.parametrize("nodes", [1, 2, 31, 64, 65, 128])
@pytest.mark.parametrize("shape", ["mixed", "chain", "star", "pairs"])
def test_masks(nodes, shape):
    rng = np.random.default_rng(nodes)
    parents = np.stack([random_parents(rng, nodes, shape) for _ in range(5)])
    lens = np.array([nodes, 0, nodes // 2, nodes, 1], dtype=np.int32)
    if nodes > 2:
        parents[3, 2] = -1                                               # a second root
    mask = torch.full((5, nodes, (nodes + 63) // 64), -1, dtype=torch.int64, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.tree_mask(mask, torch.from_numpy(parents).cuda(), torch.from_numpy(lens).cuda(), flags)
    want = od.pack_mask(np.stack([od.ancestor_mask(parents[b], lens[b], nodes) for b in range(5)]))
    torch.cuda.synchronize()
    assert int(flags.item()) == 0 and np.array_equal(mask.cpu().numpy(), want)
    parents[0, -1] = nodes
    lens[4] = nodes + 1
    binding.tree_mask(mask, torch.from_numpy(parents).cuda(), torch.from_numpy(lens).cuda(), flags)
    lens[4] = 0
    want = od.pack_mask(np.stack([od.ancestor_mask(parents[b], lens[b], nodes) for b in range(5)]))
    torch.cuda.synchronize()
    assert int(flags.item()) == od.FLAG_TREE_RANGE and np.array_equal(mask.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("vocab", [2047, 2048, 2049, 4095, 4097, 8191, 16385, 32767, 32769, 65535, 65537, 131071, 131072, 140001])
def test_vocabularies_at_the_borders_of_the_forms(dtype, vocab):
    target, draft, tokens, parents, uniforms = make(vocab, 2, 4, vocab, dtype, "star")
    uniforms[1] = np.float32(1 - 2.0 ** -24)         # the last tokens of the rows too
    check(target, draft, tokens, parents, None, uniforms)


def test_more_sequences_than_clusters_fit():
    target, draft, tokens, parents, uniforms = make(7, 200, 6, 9001, torch.float16, "mixed")
    lens = np.random.default_rng(1).integers(0, 7, 200).astype(np.int32)
    check(target, draft, tokens, parents, lens, uniforms)
