"""Attention of draft trees over the cache against a plain loop in 64 bits: types of layout, head sizes,
row counts from one to hundreds, ragged and empty trees, chunk borders, and what hidden nodes may hold.

The tolerance follows from the arithmetic.  A logit is D exact products added up in 32 bits, where
each addition (the tensor cores' included, which may truncate) is off by at most 2^-23 of the sum of
the magnitudes: D 2^-23 * spread.  A weight's relative error is that of its exponential's argument
(twice: the row's reference and sum carry it too), 2^-21 for the exponential and the two fp16 parts,
and each of the n additions of the row's sum and of its output is off by at most 2^-23; the chunk
merge repeats the exponential and a few additions.  Times the row's sum of weight * |value|, plus the
rounding to fp16 (half a step, 2^-11 of the value, 2^-25 below the normal range)."""
import itertools

import numpy as np
import pytest
import torch

from oracle import draft as od
from paper_2409_04992_b200 import binding
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=[2, 1], ids=["tcgen05", "warp-mma"])
def path(request):
    """Both implementations (shapes the tcgen05 form does not take fall back inside the library)."""
    binding.set_grouped_path(request.param)
    yield request.param
    binding.set_grouped_path(0)


def random_tree(rng, nodes, width):
    parents = np.full(width, -1, dtype=np.int32)
    for t in range(1, nodes):
        parents[t] = max(0, t - int(rng.geometric(0.4)))
    return parents


class Case:
    def __init__(self, layout, tokens, q_heads, kv_heads, dim, nodes, lens, trees=None, seed=0, see=None, q_scale=1.0):
        rng = np.random.default_rng(seed)
        B = len(lens)
        self.lens = np.array(lens, dtype=np.int32)
        self.trees = np.array(trees if trees is not None else [min(nodes, max(n, 0)) for n in lens], dtype=np.int32)
        if layout == "paged":
            per = max(1, max(od.blocks_for(n, tokens) for n in lens))
            blocks = B * per + 2
            self.table = rng.permutation(blocks)[:B * per].reshape(B, per).astype(np.int32)
            shape = (blocks, kv_heads, tokens, dim)
        else:
            self.table, shape = None, (B, kv_heads, max(1, max(lens)), dim)
        draw = lambda *s: rng.standard_normal(s, dtype=np.float32).astype(np.float16)  # noqa: E731
        self.q, self.k, self.v = draw(B, nodes, q_heads, dim) * np.float16(q_scale), draw(*shape), draw(*shape)
        self.scale = 1.0 / np.sqrt(dim)
        if see is None:
            see = np.stack([od.ancestor_mask(random_tree(rng, t, nodes), t, nodes) for t in self.trees])
        self.see = see
        self.poison_what_is_unused()

    def poison_what_is_unused(self):
        """Every slot that no sequence holds gets NaN."""
        used = np.zeros(self.k.shape[:1] + self.k.shape[2:3], dtype=bool)
        for b, n in enumerate(self.lens):
            for i in range(max(n, 0)):
                if self.table is None:
                    used[b, i] = True
                else:
                    T = self.k.shape[2]
                    used[self.table[b, i // T], i % T] = True
        for cache in (self.k, self.v):
            cache.transpose(0, 2, 1, 3)[~used] = np.nan

    def put(self, b, pos, k=None, v=None):
        where = (b, slice(None), pos) if self.table is None else \
            (self.table[b, pos // self.k.shape[2]], slice(None), pos % self.k.shape[2])
        if k is not None:
            self.k[where] = k
        if v is not None:
            self.v[where] = v


def run(c, trees="own", max_len=None, table="own", stream=None):
    put = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    B, T, Hq, D = c.q.shape
    out, lse = gu.Guarded((B, T, Hq, D), torch.float16), gu.Guarded((B, T, Hq), torch.float32)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    max_len = max_len or max(1, int(c.lens.max()))
    need = binding.tree_workspace_bytes(B, T, Hq, c.k.shape[1], D, max_len)
    ws = gu.Guarded((need,), torch.uint8)
    q, k, v, lens = put(c.q), put(c.k), put(c.v), put(c.lens)
    mask, nodes, blocks = put(od.pack_mask(c.see)), put(c.trees if isinstance(trees, str) else trees), put(c.table if isinstance(table, str) else table)
    torch.cuda.synchronize()
    binding.decode_attention_tree(out.view, lse.view, q, k, v, blocks, lens, nodes, mask, max_len, c.scale, ws.view, flags, stream)
    torch.cuda.synchronize()
    assert out.intact() and lse.intact() and ws.intact(), "a kernel wrote outside its buffers"
    return out.view.cpu().numpy(), lse.view.cpu().numpy(), int(flags.item())


def compare(got, got_lse, want, what="", n=1 << 11):
    """n: no row has more positions."""
    out, lse, size, spread = want
    dim = out.shape[-1]
    logit = dim * 2.0 ** -23 * spread + 2.0 ** -22 * np.where(np.isfinite(lse), np.abs(lse), 0.0)
    relative = 2 * logit + 2.0 ** -20 + 2 * n * 2.0 ** -23
    bound = relative[..., None] * size + 2.0 ** -11 * np.abs(out) + 2.0 ** -24
    got = got.astype(np.float64)
    assert np.isfinite(got[np.isfinite(out)]).all(), what
    with np.errstate(invalid="ignore"):
        off = np.abs(got - out) - bound
    assert (off[np.isfinite(out)] <= 0).all(), f"{what}: {np.nanmax(off)} over the bound"
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got_lse), empty), what
    assert (got[empty] == 0).all(), what
    live = np.isfinite(lse)
    lse_bound = logit + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -22 * np.abs(np.where(live, lse, 0))
    lse_off = np.abs(got_lse[live] - lse[live])
    assert (lse_off <= lse_bound[live]).all(), f"{what}: lse {lse_off.max()}"


def check(c, what="", **kw):
    got, got_lse, flags = run(c, **kw)
    assert flags == 0, what
    compare(got, got_lse, od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale), what, int(c.lens.max()))
    return got, got_lse


LAYOUTS = [("contiguous", 0), ("paged", 16), ("paged", 32), ("paged", 48), ("paged", 64), ("paged", 128), ("paged", 256)]
LENS = [1, 17, 127, 128, 129, 0, 300, 641, 64, 255]


@pytest.mark.parametrize("layout,tokens", LAYOUTS)
@pytest.mark.parametrize("dim,q_heads,kv_heads,nodes", [
    (128, 2, 2, 1), (128, 3, 1, 5), (128, 8, 2, 4), (128, 2, 2, 17), (128, 1, 1, 64), (128, 4, 2, 65), (128, 1, 1, 128),
    (128, 5, 1, 27), (128, 16, 2, 32), (128, 8, 1, 64), (64, 2, 2, 8), (64, 6, 2, 33), (64, 4, 1, 64), (256, 2, 1, 6),
    (256, 3, 1, 25), (256, 4, 2, 64), (256, 8, 1, 40)])
def test_shapes_and_layouts(layout, tokens, dim, q_heads, kv_heads, nodes):
    check(Case(layout, tokens, q_heads, kv_heads, dim, nodes, LENS, seed=dim + nodes), f"{layout} T={tokens} D={dim} nodes={nodes}")


@pytest.mark.parametrize("layout,tokens", [("contiguous", 0), ("paged", 32)])
@pytest.mark.parametrize("dim,group,nodes", [(128, 1, 40), (128, 5, 40), (64, 2, 100), (256, 3, 30)])
def test_long_sequences_are_cut_and_joined(layout, tokens, dim, group, nodes):
    # many pieces per sequence, cut at other places for every batch
    for lens in ([5000], [3001, 40, 2999], [129] * 40, [1, 0, 4000, 0, 128]):
        trees = [min(nodes, n) for n in lens]
        check(Case(layout, tokens, group, 1, dim, nodes, lens, trees, seed=len(lens)), f"{lens[:3]} D={dim}")


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("nodes,group", [(7, 1), (30, 2), (128, 2)])
def test_ragged_and_empty_trees(dim, nodes, group):
    lens = [300, 200, nodes, nodes + 1, 0, 131, nodes]
    trees = [nodes, 0, nodes, 1, nodes, max(1, nodes - 3), nodes // 2]
    c = Case("paged", 32, 2 * group, 2, dim, nodes, lens, trees, seed=3)
    got, lse = check(c, "ragged")
    assert (got[1] == 0).all() and np.isneginf(lse[1]).all() and (got[4] == 0).all()
    # rows that see nothing: the whole sequence is the tree and the mask hides it
    see = np.zeros((len(lens), nodes, nodes), dtype=bool)
    see[:, ::2] = np.random.default_rng(1).random((len(lens), (nodes + 1) // 2, nodes)) < 0.5
    c = Case("contiguous", 0, 2 * group, 2, dim, nodes, lens, trees, seed=4, see=see)
    got, lse = check(c, "any mask")
    assert np.isneginf(lse[2, 1::2]).all()
    # bits of nodes that a shorter tree does not have are ignored
    c = Case("contiguous", 0, 2 * group, 2, dim, nodes, lens, trees, seed=5, see=np.ones((len(lens), nodes, nodes), dtype=bool))
    check(c, "all bits")


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("layout,tokens", [("contiguous", 0), ("paged", 16), ("paged", 48)])
@pytest.mark.parametrize("nodes,group", [(6, 1), (40, 1), (40, 5)])
def test_hidden_nodes_may_hold_anything(dim, layout, tokens, nodes, group):
    """Infinities and NaN in keys and values: rows that do not see them are as the oracle has them, rows
    that see a NaN key are NaN, rows that see a value that is not finite have it where it is."""
    lens = [nodes, 150, 260, 133]
    c = Case(layout, tokens, group, 1, dim, nodes, lens, seed=6)
    bad = nodes - 2
    for b, n in enumerate(lens):
        base = n - nodes
        c.see[b, bad + 1, bad] = False
        c.see[b, 1, :] = False
        c.see[b, 1, 1] = True
    c.put(0, lens[0] - nodes + bad, v=np.nan)
    c.put(1, lens[1] - nodes + bad, k=np.nan)
    value = np.zeros(dim, dtype=np.float16)
    value[3], value[dim - 1] = np.inf, np.nan
    c.put(2, lens[2] - nodes + bad, v=value)
    c.put(3, lens[3] - nodes + bad, k=np.inf, v=-np.inf)
    c.put(3, lens[3] - nodes + 1, v=65504)               # the largest finite one is an ordinary value
    got, lse, flags = run(c)
    with np.errstate(all="ignore"):
        want = od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale)
    assert flags == 0
    seeing = c.see[:, :, bad]
    assert seeing.any() and not seeing.all()
    hidden = [x.copy() for x in want]
    compare(np.where(seeing[:, :, None, None], 0, got), np.where(seeing[:, :, None], -np.inf, lse),
            [np.where(seeing[:, :, None, None], 0, want[0]), np.where(seeing[:, :, None], -np.inf, want[1]),
             np.where(seeing[:, :, None, None], 0, hidden[2]), np.where(seeing[:, :, None], 0, hidden[3])], "rows that do not see it")
    assert np.isnan(got[0][seeing[0]]).all() and np.isfinite(lse[0][seeing[0]]).all()
    assert np.isnan(got[1][seeing[1]]).all() and np.isnan(lse[1][seeing[1]]).all()
    two = got[2][seeing[2]]
    assert np.isposinf(two[..., 3]).all() and np.isnan(two[..., dim - 1]).all()
    rest = [i for i in range(dim) if i not in (3, dim - 1)]
    assert np.isfinite(two[..., rest]).all()
    pick = lambda x: x[2][seeing[2]][..., rest][None, None]  # noqa: E731
    assert (np.abs(two[..., rest][None, None].astype(np.float64) - pick(want[0])) <= 0.01 * pick(want[2]) + 2.0 ** -24).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_peaked_and_moving_logits(dim):
    for nodes, group in ((3, 2), (50, 1), (50, 4)):
        c = Case("paged", 64, group, 1, dim, nodes, [900, 400], seed=7, q_scale=2.0)
        for b, n in enumerate((900, 400)):
            for pos, gain in ((n // 3, 2.0), (n // 2 + 5, 4.0), (n - nodes - 2, 6.0)):
                c.put(b, pos, k=(c.q[b, 1, 0].astype(np.float32) * gain / 2 * (128 / dim) ** 0.5).astype(np.float16))
        check(c, "moving reference")
    c = Case("contiguous", 0, 2, 1, dim, 20, [300, 77], seed=8)
    for scale in (0.0, -1.0 / np.sqrt(dim)):
        c.scale = scale
        check(c, f"scale {scale}")


@pytest.mark.parametrize("dim,nodes,group", [(128, 8, 1), (128, 40, 1), (128, 60, 2), (128, 60, 4), (64, 30, 1), (64, 90, 2), (256, 20, 1), (256, 90, 1)])
def test_huge_logits(path, dim, nodes, group):
    """Logits of 2^20 to 2^35, past where a reference and the weights' scale can be added exactly: the kernels
    end, and as the largest logit of a row is apart from the others by far more than their rounding, its
    value row is the result."""
    if path == 1:
        pytest.skip("the warp-level form's weights overflow there, as the grouped entry point's do")
    c = Case("contiguous", 0, group, 1, dim, nodes, [300, 140], seed=15)
    for b, n in enumerate(c.lens):
        sizes = 2.0 ** np.random.default_rng(b).uniform(-1, 13, n)
        c.k[b, 0, :n] = np.sign(c.k[b, 0, :n].astype(np.float32)) * 4 * sizes[:, None]
    c.q = (np.sign(c.q.astype(np.float32)) * 2.0 ** np.random.default_rng(5).uniform(4, 14, c.q.shape[:3])[..., None]).astype(np.float16)
    want = od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale)
    got, lse, flags = run(c)
    assert flags == 0 and np.isfinite(got).all() and np.isfinite(lse).all()
    assert want[3].max() > 2.0 ** 30
    assert (np.abs(lse - want[1]) <= dim * 2.0 ** -22 * want[3] + 16).all()
    # rows whose second largest logit is far below the largest one, in units of the logits' rounding
    clear = 0
    for b, n in enumerate(c.lens):
        for t in range(c.trees[b]):
            seen = [*range(n - c.trees[b]), *(n - c.trees[b] + j for j in range(c.trees[b]) if c.see[b, t, j])]
            for h in range(group):
                s = np.sort(c.k[b, 0, seen].astype(np.float64) @ c.q[b, t, h].astype(np.float64) * c.scale)
                if s[-1] - s[-2] > 2 * dim * 2.0 ** -22 * want[3][b, t, h] + 40:
                    clear += 1
                    assert np.abs(got[b, t, h] - want[0][b, t, h]).max() <= 2.0 ** -10 * np.abs(want[0][b, t, h]).max()
    assert clear > 0


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-30, -1e-30, -0.09, 2.0, -2.0])
@pytest.mark.parametrize("dim,nodes,group", [(128, 6, 1), (128, 40, 2), (128, 50, 3), (64, 70, 1), (256, 40, 1), (256, 80, 1)])
def test_other_scales(scale, dim, nodes, group):
    c = Case("contiguous", 0, group, 1, dim, nodes, [300, 131, 20], seed=18)
    c.scale = scale
    check(c, f"scale {scale}")


def test_a_cache_smaller_than_one_tile():
    for dim, nodes, group in ((128, 2, 1), (128, 2, 40), (64, 2, 20), (256, 1, 70), (128, 1, 128)):
        check(Case("contiguous", 0, group, 1, dim, nodes, [3], seed=16), f"three tokens, {group} heads")
        check(Case("paged", 16, 2 * group, 2, dim, nodes, [2, 3], seed=17), f"three tokens, {group} heads, paged")


def test_a_chain_agrees_with_the_grouped_entry_point():
    c = Case("paged", 32, 8, 2, 128, 4, [300, 64, 1000], seed=9)
    c.see[:] = np.tril(np.ones((4, 4), dtype=bool))
    got, lse, _ = run(c)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    out, other = torch.zeros(3, 4, 8, 128, dtype=torch.float16, device="cuda"), torch.zeros(3, 4, 8, device="cuda")
    ws = torch.empty(binding.grouped_workspace_bytes(3, 4, 8, 2, 128, 1000), dtype=torch.uint8, device="cuda")
    binding.decode_attention_grouped(out, other, put(c.q), put(c.k), put(c.v), put(c.table), put(c.lens), 1000, c.scale, ws)
    torch.cuda.synchronize()
    assert np.abs(out.cpu().numpy().astype(np.float64) - got).max() <= gu.MAX_ABS
    assert np.allclose(other.cpu().numpy(), lse, atol=gu.LSE_ATOL, rtol=gu.LSE_RTOL)


def test_trees_without_lengths_and_a_longer_bound():
    c = Case("paged", 16, 2, 1, 128, 9, [40, 100, 9], seed=10)
    want = od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale)
    got, lse, flags = run(c, trees=None, max_len=7 * 16)
    assert flags == 0
    compare(got, lse, want, "tree_lens None")


@pytest.mark.parametrize("nodes,group", [(8, 1), (48, 1), (48, 4)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_flags(nodes, group, dim):
    c = Case("paged", 32, group, 1, dim, nodes, [100, 90, 200, 77], seed=11)
    want = od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale)
    bad = c.trees.copy()
    bad[0], bad[1] = nodes + 1, -1
    got, lse, flags = run(c, trees=bad)
    assert flags == od.FLAG_TREE_RANGE and (got[:2] == 0).all() and np.isneginf(lse[:2]).all()
    compare(got[2:], lse[2:], [x[2:] for x in want], "others")
    got, lse, flags = run(c, max_len=100)                # 200 tokens are more than the call says
    assert flags == od.FLAG_SEQ_LEN_RANGE and (got[2] == 0).all()
    lens = c.lens.copy()
    c.lens[3] = nodes - 1                                # a tree longer than its sequence
    got, lse, flags = run(c, trees=np.full(4, nodes, dtype=np.int32))
    assert flags == od.FLAG_TREE_RANGE and (got[3] == 0).all()
    c.lens = lens
    table = c.table.copy()
    table[1, 1] = len(c.k) + 5                           # a block that is not there counts as zeros
    got, lse, flags = run(c, table=table)
    assert flags == od.FLAG_BLOCK_RANGE
    for cache in (c.k, c.v):
        cache[c.table[1, 1]] = 0
    compare(got, lse, od.tree_attention(c.q, c.k, c.v, c.table, c.lens, c.trees, c.see, c.scale), "zeroed block")


def test_the_result_does_not_depend_on_where_blocks_lie():
    c = Case("paged", 16, 4, 2, 128, 20, [500, 333, 64], seed=12)
    first, lse, _ = run(c)
    move = np.random.default_rng(2).permutation(len(c.k))
    c.k, c.v = c.k[np.argsort(move)], c.v[np.argsort(move)]
    c.table = move[c.table].astype(np.int32)
    again, other, _ = run(c)
    assert np.array_equal(first.view(np.uint16), again.view(np.uint16)) and np.array_equal(lse, other)


@pytest.mark.parametrize("nodes,group", [(4, 1), (30, 1), (60, 4)])
def test_streams_graphs_and_repeats(nodes, group):
    """On another stream, and two captured calls that share a workspace, replayed: the same bits."""
    c = Case("paged", 64, 2 * group, 2, 128, nodes, [700, 90, 1500], seed=13)
    want, want_lse, _ = run(c)
    got, lse, _ = run(c, stream=torch.cuda.Stream())
    assert np.array_equal(want.view(np.uint16), got.view(np.uint16)) and np.array_equal(want_lse, lse)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    B, T, Hq, D = c.q.shape
    dev = [put(x) for x in (c.q, c.k, c.v, c.table, c.lens, c.trees, od.pack_mask(c.see))]
    ws = torch.empty(binding.tree_workspace_bytes(B, T, Hq, 2, D, 1500), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros(B, T, Hq, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    graphs = []
    for out in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.decode_attention_tree(out, None, dev[0], dev[1], dev[2], dev[3], dev[4], dev[5], dev[6], 1500, c.scale, ws)
        graphs.append(graph)
    ws.fill_(0xFF)
    for graph in (graphs[0], graphs[1], graphs[0]):
        graph.replay()
    torch.cuda.synchronize()
    for out in outs:
        assert np.array_equal(out.cpu().numpy().view(np.uint16), want.view(np.uint16))


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes per cache: sequences at its two ends."""
    blocks, T, H, D, nodes = 40000, 64, 8, 128, 33
    k = torch.zeros(blocks, H, T, D, dtype=torch.float16, device="cuda")
    assert k.numel() * 2 > 1 << 32
    v = torch.zeros_like(k)
    small = Case("paged", T, H, H, D, nodes, [200, 150], seed=14)
    ids = np.array([[blocks - 1, 3, blocks - 7, blocks // 2], [0, blocks - 2, blocks - 3, 5]], dtype=np.int32)
    for b, e in itertools.product(range(2), range(small.table.shape[1])):
        k[int(ids[b, e])] = torch.from_numpy(small.k[small.table[b, e]]).cuda()
        v[int(ids[b, e])] = torch.from_numpy(small.v[small.table[b, e]]).cuda()
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    out, lse = torch.zeros(2, nodes, H, D, dtype=torch.float16, device="cuda"), torch.zeros(2, nodes, H, device="cuda")
    ws = torch.empty(binding.tree_workspace_bytes(2, nodes, H, H, D, 256), dtype=torch.uint8, device="cuda")
    binding.decode_attention_tree(out, lse, put(small.q), k, v, put(ids), put(small.lens), put(small.trees),
                                  put(od.pack_mask(small.see)), 256, small.scale, ws)
    torch.cuda.synchronize()
    compare(out.cpu().numpy(), lse.cpu().numpy(),
            od.tree_attention(small.q, small.k, small.v, small.table, small.lens, small.trees, small.see, small.scale), "far blocks")


@pytest.mark.parametrize("layout,tokens,dim,q_heads,kv_heads,nodes,lens", [
    ("paged", 32, 128, 40, 40, 64, [9000, 5003, 7777, 130, 64]),      # many items, each shorter than a long piece
    ("paged", 64, 128, 32, 4, 32, [60000, 33001, 40]),                # few items, longer than the pieces; two row blocks
    ("contiguous", 0, 64, 24, 24, 20, [30011, 17000]),
    ("paged", 128, 256, 12, 6, 40, [40000, 200, 33333]),
    ("paged", 16, 128, 16, 16, 7, [70001, 12345]),
    ("paged", 32, 64, 20, 2, 13, [60011, 50000, 1000])])
def test_large_batches_whose_pieces_are_drawn(path, layout, tokens, dim, q_heads, kv_heads, nodes, lens):
    """Enough tiles for pieces drawn from the ticket counter: every row against 64-bit attention on the
    GPU, one (sequence, KV head) at a time; twice, with the same bits."""
    if path == 1:
        pytest.skip("the cut into pieces belongs to the tcgen05 form")
    B, group = len(lens), q_heads // kv_heads
    g = torch.Generator(device="cuda").manual_seed(sum(lens))
    draw = lambda *s: torch.randn(*s, generator=g, device="cuda").half()  # noqa: E731
    rng = np.random.default_rng(3)
    trees = [nodes, max(1, nodes - 3), nodes, nodes, nodes][:B]
    see = np.stack([od.ancestor_mask(random_tree(rng, t, nodes), t, nodes) for t in trees])
    if layout == "paged":
        per = max(od.blocks_for(n, tokens) for n in lens)
        ids = rng.permutation(B * per)[:B * per].reshape(B, per).astype(np.int32)
        table = torch.from_numpy(ids).cuda()
        k, v = draw(B * per, kv_heads, tokens, dim), draw(B * per, kv_heads, tokens, dim)
    else:
        table, k, v = None, draw(B, kv_heads, max(lens), dim), draw(B, kv_heads, max(lens), dim)
    q = draw(B, nodes, q_heads, dim)
    put = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    scale, flags = dim ** -0.5, torch.zeros(1, dtype=torch.int32, device="cuda")
    need = binding.tree_workspace_bytes(B, nodes, q_heads, kv_heads, dim, max(lens))
    outs = []
    for _ in range(2):
        out, lse, ws = gu.Guarded(tuple(q.shape), torch.float16), gu.Guarded(tuple(q.shape[:3]), torch.float32), gu.Guarded((need,), torch.uint8)
        binding.decode_attention_tree(out.view, lse.view, q, k, v, table, put(lens), put(trees),
                                      torch.from_numpy(od.pack_mask(see)).cuda(), max(lens), scale, ws.view, flags)
        torch.cuda.synchronize()
        assert out.intact() and lse.intact() and ws.intact() and int(flags.item()) == 0
        outs.append((out.view.clone(), lse.view.clone()))
    assert torch.equal(outs[0][0].view(torch.int16), outs[1][0].view(torch.int16)) and torch.equal(outs[0][1], outs[1][1])
    got, got_lse = outs[0]
    for b, (n, t) in enumerate(zip(lens, trees)):
        hide = torch.zeros(t, n, dtype=torch.float64, device="cuda")
        hide[:, n - t:] = torch.where(torch.from_numpy(see[b, :t, :t]).cuda(), 0.0, -float("inf"))
        for h in range(kv_heads):
            if table is None:
                ks, vs = k[b, h, :n].double(), v[b, h, :n].double()
            else:
                pages = table[b, :od.blocks_for(n, tokens)].long()
                ks, vs = k[pages, h].flatten(0, 1)[:n].double(), v[pages, h].flatten(0, 1)[:n].double()
            rows = q[b, :t, h * group:(h + 1) * group].double()
            s = torch.einsum("tgd,nd->tgn", rows, ks) * scale
            spread = (torch.einsum("tgd,nd->tgn", rows.abs(), ks.abs()) * scale).amax(-1)
            s += hide[:, None]
            w = torch.softmax(s, -1)
            compare(got[b, :t, h * group:(h + 1) * group].cpu().numpy(), got_lse[b, :t, h * group:(h + 1) * group].cpu().numpy(),
                    [x.cpu().numpy() for x in (w @ vs, torch.logsumexp(s, -1), w @ vs.abs(), spread)], f"sequence {b} head {h}", n)
        assert (got[b, t:] == 0).all() and torch.isneginf(got_lse[b, t:]).all()


@pytest.mark.parametrize("layout,tokens,dim,q_heads,kv_heads,nodes", [
    ("contiguous", 0, 128, 128, 1, 32),       # 4096 rows: 32 blocks of rows of one node each
    ("paged", 16, 128, 100, 1, 8),            # a node's heads leave 28 rows of a block empty
    ("paged", 32, 256, 65, 1, 5), ("contiguous", 0, 256, 64, 1, 64), ("paged", 128, 64, 96, 1, 7),
    ("contiguous", 0, 128, 400, 2, 3),        # more heads than a block of rows: the warp-level form
    ("paged", 16, 64, 33, 1, 124)])
def test_many_rows(layout, tokens, dim, q_heads, kv_heads, nodes):
    lens = [300, 5, 129, 0]
    check(Case(layout, tokens, q_heads, kv_heads, dim, nodes, lens, [min(nodes, n) for n in lens], seed=nodes), f"{q_heads} heads, {nodes} nodes")


@pytest.mark.parametrize("layout,tokens", [("contiguous", 0), ("paged", 16)])
@pytest.mark.parametrize("dim,nodes,group", [(128, 3, 1), (128, 20, 2), (128, 30, 3), (64, 5, 4), (256, 5, 2)])
def test_large_batches_of_short_and_empty_sequences(layout, tokens, dim, nodes, group):
    lens = np.random.default_rng(nodes).choice([0, 0, 1, 2, 5, 40, 140, 270], 700)
    trees = [min(nodes, int(n)) for n in lens]
    trees[5:50:3] = [0] * 15
    check(Case(layout, tokens, group, 1, dim, nodes, lens.tolist(), trees, seed=19), f"700 sequences D={dim}")
    check(Case(layout, tokens, group, 1, dim, nodes, [0] * 699 + [300], seed=20), f"one of 700 D={dim}")


@pytest.mark.parametrize("dim,nodes,group", [(128, 3, 1), (128, 20, 2), (128, 30, 3), (64, 30, 1), (256, 5, 2)])
def test_without_log_sum_exps_and_flags(dim, nodes, group):
    c = Case("paged", 32, group, 1, dim, nodes, [300, 40, 0, 2000], [nodes, nodes, 0, 1], seed=21)
    want, want_lse, _ = run(c)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    out = gu.Guarded(c.q.shape, torch.float16)
    ws = torch.empty(binding.tree_workspace_bytes(4, nodes, group, 1, dim, 2000), dtype=torch.uint8, device="cuda")
    binding.decode_attention_tree(out.view, None, put(c.q), put(c.k), put(c.v), put(c.table), put(c.lens), put(c.trees),
                                  put(od.pack_mask(c.see)), 2000, c.scale, ws)
    torch.cuda.synchronize()
    assert out.intact() and np.array_equal(gu.bits(out.view), want.view(np.uint16))


@pytest.mark.parametrize("nodes,group", [(9, 1), (40, 1), (40, 4)])
def test_drawn_pieces_in_a_captured_call(path, nodes, group):
    """Replays, and an eager call between them on the same workspace, give the same bits: the counter that
    pieces are drawn from starts anew each time."""
    if path == 1:
        pytest.skip("the cut into pieces belongs to the tcgen05 form")
    B, H, D, n = 4, 8, 128, 16384
    g = torch.Generator(device="cuda").manual_seed(nodes)
    draw = lambda *s: torch.randn(*s, generator=g, device="cuda").half()  # noqa: E731
    k, v, q = draw(B, H, n, D), draw(B, H, n, D), draw(B, nodes, H * group, D)
    lens = torch.tensor([n, n - 77, n - 5000, n], dtype=torch.int32, device="cuda")
    see = np.stack([od.ancestor_mask(random_tree(np.random.default_rng(b), nodes, nodes), nodes, nodes) for b in range(B)])
    mask = torch.from_numpy(od.pack_mask(see)).cuda()
    ws = torch.full((binding.tree_workspace_bytes(B, nodes, H * group, H, D, n),), 255, dtype=torch.uint8, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    eager, captured = (torch.zeros_like(q) for _ in range(2))

    def call(out):
        binding.decode_attention_tree(out, None, q, k, v, None, lens, None, mask, n, D ** -0.5, ws, flags)

    call(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(captured)
    for _ in range(3):
        captured.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured.view(torch.int16), eager.view(torch.int16))
        call(eager)
    torch.cuda.synchronize()
    assert torch.equal(captured.view(torch.int16), eager.view(torch.int16)) and int(flags.item()) == 0
