"""Blocks of a shared pool (fork, resize with copy on write, defragment) and keeping a draft tree's
accepted path: bit for bit what plain loops do, the state's integers and every layer's pages."""
import numpy as np
import pytest
import torch

from oracle import draft as od
from paper_2409_04992_b200 import binding
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


def to_gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def same(gpu: torch.Tensor, cpu: np.ndarray):
    return np.array_equal(gpu.cpu().numpy(), cpu)


class Pool:
    """The same pool on both sides; every operation runs on both and is compared."""

    def __init__(self, layers, blocks, heads, tokens, dim, batch, per_seq, seed=0):
        rng = np.random.default_rng(seed)
        self.tokens, self.layers = tokens, layers
        self.caches = [rng.integers(0, 1 << 16, (blocks, heads, tokens, dim), dtype=np.uint16) for _ in range(2 * layers)]
        self.table = np.full((batch, per_seq), -7, dtype=np.int32)
        self.refs = np.zeros(blocks, dtype=np.int32)
        self.lens = np.zeros(batch, dtype=np.int32)
        self.gpu_caches = [to_gpu(c.view(np.float16)) for c in self.caches]
        self.upload()
        self.ws = gu.Guarded((max(binding.kv_resize_workspace_bytes(batch, blocks),
                                  binding.kv_defragment_workspace_bytes(blocks)),), torch.uint8)
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")

    def upload(self):
        self.gpu_table, self.gpu_refs, self.gpu_lens = to_gpu(self.table), to_gpu(self.refs), to_gpu(self.lens)

    @property
    def k(self):
        return self.gpu_caches[:self.layers]

    @property
    def v(self):
        return self.gpu_caches[self.layers:]

    def check(self, want_flags, what):
        torch.cuda.synchronize()
        got = int(self.flags.item())
        self.flags.zero_()
        assert got == want_flags, f"{what}: flags {got}, expected {want_flags}"
        assert same(self.gpu_lens, self.lens), f"{what}: lengths {self.gpu_lens.cpu().tolist()} {self.lens.tolist()}"
        assert same(self.gpu_refs, self.refs), f"{what}: counts"
        assert same(self.gpu_table, self.table), f"{what}: table"
        assert self.ws.intact(), what
        for i, (g, c) in enumerate(zip(self.gpu_caches, self.caches)):
            assert np.array_equal(gu.bits(g), c), f"{what}: cache {i}"

    def resize(self, want, what="resize"):
        want_gpu = ints(want)
        new, flags = od.resize(self.caches, self.table, self.refs, self.lens, want, self.tokens)
        self.lens = new
        binding.kv_resize(self.k, self.v, self.gpu_table, self.gpu_refs, self.gpu_lens, want_gpu, self.gpu_lens,
                          self.ws.view, self.flags)
        self.check(flags, what)
        return flags

    def fork(self, src, dst, what="fork"):
        flags = od.fork(self.table, self.refs, self.lens, src, dst, self.tokens)
        binding.kv_fork(self.gpu_table, self.gpu_refs, self.gpu_lens, ints(src), ints(dst), self.tokens, self.flags)
        self.check(flags, what)
        return flags

    def defragment(self, in_place, what="defragment"):
        table, refs, used, flags = od.defragment(self.caches, self.table, self.refs, self.lens, self.tokens)
        out_table = self.gpu_table if in_place else torch.full_like(self.gpu_table, 99)
        out_refs = self.gpu_refs if in_place else torch.full_like(self.gpu_refs, 99)
        count = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        binding.kv_defragment(self.k, self.v, self.gpu_table, self.gpu_refs, self.gpu_lens, out_table, out_refs, count,
                              self.ws.view, self.flags)
        torch.cuda.synchronize()
        assert int(count.item()) == used
        if not in_place:
            assert same(self.gpu_table, self.table) and same(self.gpu_refs, self.refs)      # inputs untouched
        self.table, self.refs, self.gpu_table, self.gpu_refs = table, refs, out_table, out_refs
        self.check(flags, what)


@pytest.mark.parametrize("layers,blocks,heads,tokens,dim,batch,per_seq", [
    (1, 40, 2, 16, 64, 6, 9), (3, 57, 3, 8, 128, 9, 12), (2, 33, 5, 24, 256, 5, 7), (2, 5000, 1, 8, 64, 40, 60)])
def test_random_histories(layers, blocks, heads, tokens, dim, batch, per_seq):
    rng = np.random.default_rng(blocks)
    pool = Pool(layers, blocks, heads, tokens, dim, batch, per_seq, seed=1)
    seen = 0
    for step in range(40):
        kind = rng.integers(0, 10)
        if kind < 6:
            want = np.where(rng.random(batch) < 0.5, pool.lens,
                            rng.integers(0, per_seq * tokens + 1, batch) * (rng.random(batch) < 0.8)).astype(np.int32)
            if kind < 3:        # small growth, as a decode step's
                want = np.minimum(pool.lens + rng.integers(0, 5, batch), per_seq * tokens).astype(np.int32)
            seen |= pool.resize(want, f"step {step} resize")
        elif kind < 9:
            n = int(rng.integers(1, batch + 1))
            seen |= pool.fork(rng.integers(-1, batch, n), rng.integers(0, batch + 1, n), f"step {step} fork")
        else:
            pool.defragment(bool(rng.integers(0, 2)), f"step {step} defragment")
    assert seen & od.FLAG_POOL                       # the histories do run into what is refused
    listed = np.zeros_like(pool.refs)
    for b in range(batch):
        for e in range(od.blocks_for(pool.lens[b], tokens)):
            listed[pool.table[b, e]] += 1
    assert np.array_equal(listed, pool.refs)         # counts say what the tables list


def test_the_last_of_the_writers_keeps_a_shared_block():
    pool = Pool(2, 30, 2, 16, 64, 6, 5)
    pool.resize([20, 0, 0, 0, 0, 0])
    pool.fork([0, 0, 0], [2, 3, 5])
    shared = int(pool.table[0, 1])
    pool.resize([25, 0, 25, 25, 0, 25])              # all four grow inside the block: three copies
    assert pool.table[5, 1] == shared and pool.refs[shared] == 1
    assert len({int(pool.table[b, 1]) for b in (0, 2, 3, 5)}) == 4
    pool.fork([5], [1])
    pool.resize([25, 26, 25, 25, 0, 25])             # one of two grows: it takes the copy
    assert pool.table[5, 1] == shared


def test_a_pool_that_runs_out_leaves_later_sequences_alone():
    pool = Pool(1, 6, 1, 8, 64, 5, 6)
    assert pool.resize([10, 10, 17, 8, 0]) == od.FLAG_POOL          # 2 + 2, then 3 of 2 left
    assert pool.lens.tolist() == [10, 10, 0, 0, 0]
    # the keeper of a shared block asks for nothing, but waits for the writers that could not be served
    pool = Pool(1, 3, 1, 8, 64, 4, 4)
    pool.resize([12, 0, 0, 0])
    pool.fork([0, 0], [1, 2])
    assert pool.resize([13, 13, 13, 0]) == od.FLAG_POOL
    assert pool.lens.tolist() == [13, 12, 12, 0]
    # what is freed in the call can be given out in it
    pool = Pool(1, 4, 1, 8, 64, 2, 4)
    pool.resize([32, 0])
    assert pool.resize([0, 32]) == 0


def test_bad_lengths_ids_and_counts_are_flagged():
    pool = Pool(1, 20, 1, 8, 64, 4, 4)
    pool.resize([20, 20, 0, 0])
    assert pool.resize([33, 25, -1, 0]) == od.FLAG_SEQ_LEN_RANGE
    assert pool.lens.tolist() == [20, 25, 0, 0]
    pool.table[0, 2] = 20                            # the partly filled block is not one
    pool.upload()
    assert pool.resize([21, 25, 0, 0]) == od.FLAG_BLOCK_RANGE
    assert pool.resize([0, 25, 0, 0]) == od.FLAG_BLOCK_RANGE
    pool.refs[pool.table[1, 0]] = 0                  # counted as free although it is listed
    pool.upload()
    pool.defragment(False)
    pool.refs[:] = 0
    pool.upload()
    assert pool.resize([0, 0, 0, 0]) == od.FLAG_POOL


def test_large_batches_and_empty_ones():
    # more sequences than the planner's shared memory holds by default
    pool = Pool(1, 9000, 1, 8, 64, 8192, 2)
    want = np.random.default_rng(3).integers(0, 17, 8192).astype(np.int32)
    new, flags = od.resize([], pool.table, pool.refs, pool.lens, np.zeros(8192, dtype=np.int32), 8)
    need = sum(od.blocks_for(n, 8) for n in want)
    while need > 9000:                               # keep the oracle's loop short: no refusals here
        want = want // 2
        need = sum(od.blocks_for(n, 8) for n in want)
    at = 0
    for b in range(8192):
        for e in range(od.blocks_for(want[b], 8)):
            pool.table[b, e] = at
            pool.refs[at] = 1
            at += 1
    pool.lens = want
    binding.kv_resize(pool.k, pool.v, pool.gpu_table, pool.gpu_refs, pool.gpu_lens, to_gpu(want), pool.gpu_lens,
                      pool.ws.view, pool.flags)
    pool.check(0, "8192 sequences")
    empty = ints([]).reshape(0, 2)
    binding.kv_resize(pool.k, pool.v, empty, pool.gpu_refs, ints([]), ints([]), ints([]), pool.ws.view, pool.flags)
    binding.kv_fork(pool.gpu_table, pool.gpu_refs, pool.gpu_lens, ints([]), ints([]), 8, pool.flags)
    pool.check(0, "empty calls")


def test_a_captured_step_replays():
    """Fork, grow and free in a graph: the children appear and are gone again, twice alike."""
    pool = Pool(2, 40, 2, 16, 128, 4, 6)
    pool.resize([40, 0, 0, 0])
    grown, want, base = ints([0] * 4), ints([40, 60, 60, 0]), ints([40, 0, 0, 0])
    src, dst = ints([0, 0]), ints([1, 2])

    def step():
        binding.kv_fork(pool.gpu_table, pool.gpu_refs, pool.gpu_lens, src, dst, 16, pool.flags)
        binding.kv_resize(pool.k, pool.v, pool.gpu_table, pool.gpu_refs, pool.gpu_lens, want, grown, pool.ws.view, pool.flags)
        binding.kv_resize(pool.k, pool.v, pool.gpu_table, pool.gpu_refs, grown, base, pool.gpu_lens, pool.ws.view, pool.flags)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        od.fork(pool.table, pool.refs, pool.lens, [0, 0], [1, 2], 16)
        pool.lens, _ = od.resize(pool.caches, pool.table, pool.refs, pool.lens, [40, 60, 60, 0], 16)
        assert pool.lens.tolist() == [40, 60, 60, 0]
        pool.lens, _ = od.resize(pool.caches, pool.table, pool.refs, pool.lens, [40, 0, 0, 0], 16)
    graph.replay()
    graph.replay()
    pool.check(0, "replayed")
    assert grown.cpu().tolist() == [40, 60, 60, 0]


def test_new_lengths_may_be_the_wanted_ones_and_flags_may_be_left_out():
    pool = Pool(1, 12, 2, 8, 64, 4, 4)
    pool.resize([20, 9, 0, 0])
    pool.fork([0], [2])
    pool.lens, flags = od.resize(pool.caches, pool.table, pool.refs, pool.lens, [24, 33, 21, 5], 8)
    assert flags == od.FLAG_SEQ_LEN_RANGE            # 33 is too long
    want = ints([24, 33, 21, 5])
    binding.kv_resize(pool.k, pool.v, pool.gpu_table, pool.gpu_refs, pool.gpu_lens, want, want, pool.ws.view)
    pool.gpu_lens = want
    pool.check(0, "no flags asked for")
    od.fork(pool.table, pool.refs, pool.lens, [1, 1], [3, 3], 8)
    binding.kv_fork(pool.gpu_table, pool.gpu_refs, pool.gpu_lens, ints([1, 1]), ints([3, 3]), 8)
    pool.check(0, "no flags asked for")


# ---------------------------------------------------------------- keeping a path
def keep_case(layout, tokens, layers, batch, heads, dim, nodes, lens, seed):
    rng = np.random.default_rng(seed)
    if layout == "paged":
        per = max(od.blocks_for(n, tokens) for n in lens) + 1
        blocks = batch * per + 3
        table = rng.permutation(blocks)[:batch * per].reshape(batch, per).astype(np.int32)
        shape = (blocks, heads, tokens, dim)
    else:
        table, shape = None, (batch, heads, max(lens) + 3, dim)
    return [rng.integers(0, 1 << 16, shape, dtype=np.uint16) for _ in range(2 * layers)], table


def run_keep(caches, table, path, path_lens, tree_lens, lens, what=""):
    layers = len(caches) // 2
    gpu = [to_gpu(c.view(np.float16)) for c in caches]
    flags, new = torch.zeros(1, dtype=torch.int32, device="cuda"), ints([-5] * len(lens))
    binding.kv_keep_path(gpu[:layers], gpu[layers:], to_gpu(path), ints(path_lens), None if tree_lens is None else ints(tree_lens),
                         ints(lens), new, None if table is None else to_gpu(table), flags)
    torch.cuda.synchronize()
    nodes = [path.shape[1]] * len(lens) if tree_lens is None else tree_lens
    want, want_flags = od.keep_path(caches, path, path_lens, nodes, lens, table)
    assert int(flags.item()) == want_flags, what
    assert same(new, want), what
    for g, c in zip(gpu, caches):
        assert np.array_equal(gu.bits(g), c), what
    return want_flags


@pytest.mark.parametrize("layout,tokens", [("contiguous", 0), ("paged", 8), ("paged", 16), ("paged", 48)])
@pytest.mark.parametrize("layers,heads,dim,nodes", [(1, 1, 64, 1), (2, 5, 128, 2), (3, 3, 256, 17), (2, 40, 128, 64), (1, 3, 64, 128)])
def test_kept_rows_move(layout, tokens, layers, heads, dim, nodes):
    rng = np.random.default_rng(nodes + tokens)
    lens = [nodes, nodes + 5, nodes + 130, nodes + 1, 0, nodes + 63]
    caches, table = keep_case(layout, tokens, layers, len(lens), heads, dim, nodes, lens, 4)
    path = np.full((len(lens), nodes), -1, dtype=np.int32)
    trees, counts = [], []
    for b, n in enumerate(lens):
        tree = [nodes, max(1, nodes // 2), nodes, 0, nodes, max(1, nodes - 1)][b]
        kept = [int(rng.integers(0, tree + 1)), tree, min(1, tree), 0, 1, int(rng.integers(0, tree + 1))][b]
        path[b, :kept] = np.sort(rng.choice(max(tree, 1), kept, replace=False))
        trees.append(tree)
        counts.append(kept)
    assert run_keep(caches, table, path, counts, trees, lens) == 0


def test_paths_out_of_range_leave_the_sequence_alone():
    lens, nodes = [40] * 9, 8
    caches, table = keep_case("paged", 16, 2, 9, 3, 128, nodes, lens, 5)
    path = np.tile(np.array([0, 2, 5, 7, -1, -1, -1, -1], dtype=np.int32), (9, 1))
    path[1, 1] = 0                                   # twice the same
    path[2, 2] = 1                                   # descending
    path[3, 3] = 8                                   # no such node
    path[4, 0] = -1
    trees = [8, 8, 8, 8, 8, 9, 7, 41, -1]
    assert run_keep(caches, table, path, [4, 4, 4, 4, 4, 4, 4, 4, 4], trees, lens) == od.FLAG_TREE_RANGE
    assert run_keep(caches, table, path[:2], [9, -1], [8, 8], lens[:2]) == od.FLAG_TREE_RANGE
    assert run_keep(caches, table, path[:2], [4, 4], None, [-3, 10000]) == od.FLAG_SEQ_LEN_RANGE
    broken = table.copy()
    broken[0, 2] = len(caches[0]) + 1                # positions 32.. of sequence 0
    assert run_keep(caches, broken, path[:1], [4], None, lens[:1]) == od.FLAG_BLOCK_RANGE


def test_keep_path_refuses_its_own_lengths_as_output():
    caches, _ = keep_case("contiguous", 0, 1, 1, 1, 64, 2, [4], 6)
    gpu = [to_gpu(c.view(np.float16)) for c in caches]
    lens = ints([4])
    with pytest.raises(binding.InstInferError):
        binding.kv_keep_path(gpu[:1], gpu[1:], ints([[0, 1]]), ints([2]), None, lens, lens)
    with pytest.raises(binding.InstInferError):
        binding.kv_keep_path(gpu[:1], [], ints([[0, 1]]), ints([2]), None, lens, ints([0]))
    with pytest.raises(binding.InstInferError):
        binding.kv_keep_path(gpu[:1], [gpu[1][:, :, :3]], ints([[0, 1]]), ints([2]), None, lens, ints([0]))
