"""Attention over a latent cache against the definition in 64 bits.  Tolerances: logits are 32-bit sums over the row's dims in
steps of 16, each off by 2^-23 of what is summed, so a logit is off by delta = 40 * 2^-23 * scale * max sum |q_d c_d|; a weight
by twice that; the result by 2 delta max |c| and half a step of its type (weights enter with 16 bits or more)."""
import math

import pytest
import torch

from paper_2409_04992_b200 import binding
from tests.test_gpu_rope_append import HALF_STEP, table_for

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, lens, N, H, T=0, dtype=torch.float16, L=512, nodes=None, parents=None, scale=None, seed=1, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.N, self.H, self.T, self.L, self.dtype, self.nodes = lens, N, H, T, L, dtype, nodes
        B, D = len(lens), L + 64
        self.scale = scale if scale is not None else 1 / math.sqrt(192)
        self.max_len = max(max(lens), 1)
        self.table, blocks = table_for(lens, T) if T else (None, 0)
        self.cache = torch.randn((blocks, T, D) if T else (B, self.max_len, D), generator=g, device="cuda").to(dtype)
        self.q = (spread * torch.randn(B, N, H, D, generator=g, device="cuda")).to(dtype)
        self.mask = None
        if parents is not None:
            self.mask = torch.zeros(B, N, (N + 63) // 64, dtype=torch.int64, device="cuda")
            binding.tree_mask(self.mask, parents.cuda())
        self.nodes_t = None if nodes is None else torch.tensor(nodes, dtype=torch.int32, device="cuda")
        self.lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.room = torch.full((binding.latent_workspace_bytes(B, N, H, L, 64, self.max_len) + 512,), 0x5A, dtype=torch.uint8, device="cuda")
        self.out = torch.full((B * N * H * L + 256,), 7.0, dtype=dtype, device="cuda")
        self.lse = torch.full((B * N * H + 64,), 7.0, device="cuda")

    def run(self, stream=None):
        B, size = len(self.lens), len(self.lens) * self.N * self.H
        out, lse = self.out[128:-128].view(B, self.N, self.H, self.L), self.lse[32:-32].view(B, self.N, self.H)
        binding.decode_attention_latent(out, lse, self.q, self.cache, self.table, self.lens_t, self.nodes_t, self.mask, self.max_len, self.scale,
                                        self.room[256:-256], self.flags, stream)
        return out, lse

    def rows(self, b):
        n = self.lens[b]
        if self.table is None:
            return self.cache[b, :n]
        return self.cache[self.table[b, :-(-n // self.T)].long()].flatten(0, 1)[:n]

    def check(self):
        out, lse = self.run()
        torch.cuda.synchronize()
        for guard in (self.out[:128], self.out[-128:], self.lse[:32], self.lse[-32:]):
            assert (guard == 7.0).all()
        assert (self.room[:256] == 0x5A).all() and (self.room[-256:] == 0x5A).all()
        for b, n in enumerate(self.lens):
            nodes = self.N if self.nodes is None else self.nodes[b]
            if n == 0:
                nodes = 0
            assert (out[b, nodes:] == 0).all() and (lse[b, nodes:] == -math.inf).all(), b
            if nodes == 0:
                continue
            c, q = self.rows(b).double(), self.q[b, :nodes].double()
            sees = torch.ones(nodes, n, dtype=torch.bool, device="cuda")
            j = torch.arange(nodes, device="cuda")
            if self.mask is None:
                sees[:, n - nodes:] = j[None, :] <= j[:, None]
            else:
                sees[:, n - nodes:] = (self.mask[b, :nodes][:, j // 64] >> (j % 64)[None]) & 1 != 0
            z = (torch.einsum("nhd,ld->nhl", q, c) * self.scale).masked_fill(~sees[:, None], -math.inf)
            want = torch.softmax(z, -1) @ c[:, :self.L]
            delta = 40 * 2.0 ** -23 * abs(self.scale) * float(torch.einsum("nhd,ld->nhl", q.abs(), c.abs()).max())
            bound = HALF_STEP[self.dtype] * want.abs() + 2 * delta * float(c.abs().max()) + 2.0 ** -25
            assert bool(((out[b, :nodes].double() - want).abs() <= bound).all()), (b, n)
            assert bool(((lse[b, :nodes].double() - torch.logsumexp(z, -1)).abs() <= delta + 2.0 ** -20 * (1 + z[sees[:, None].expand_as(z)].abs().max())).all()), (b, n)
        return out, lse


LENS = [0, 1, 63, 64, 65, 127, 128, 129, 300, 1000]


@pytest.mark.parametrize("H", [1, 16, 17, 32, 33, 64, 100, 128, 129, 300])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_rows_of_all_sizes(H, dtype):
    case = Case(LENS, 1, H, T=16, dtype=dtype)
    case.check()
    assert case.flags.item() == 0


@pytest.mark.parametrize("T", [0, 8, 24, 32, 48, 64, 128, 192])
@pytest.mark.parametrize("H", [16, 128])
def test_pages_of_all_sizes(T, H):
    Case(LENS[1:], 1, H, T=T).check()


@pytest.mark.parametrize("N,H", [(2, 5), (3, 16), (8, 16), (40, 8), (128, 3), (2, 128)])
def test_several_new_tokens(N, H):
    lens = [N, N + 1, N + 63, N + 64, 700 + N]
    Case(lens, N, H, T=16, nodes=[N, max(1, N // 2), 1, 0, N]).check()


@pytest.mark.parametrize("N,H", [(5, 3), (16, 4), (70, 2), (128, 1)])
def test_trees(N, H):
    g = torch.Generator().manual_seed(N)
    parents = torch.tensor([[-1] + [int(torch.randint(max(0, t - 4), t, (1,), generator=g)) for t in range(1, N)] for _ in range(4)], dtype=torch.int32)
    Case([N, N + 50, N + 128, 900], N, H, T=32, nodes=[N, N, N // 2 + 1, N], parents=parents, dtype=torch.bfloat16).check()


@pytest.mark.parametrize("H", [16, 128])
def test_many_sequences_and_long_ones(H):
    Case([(37 * i) % 500 for i in range(70)], 1, H, T=16).check()
    Case([20000, 3, 0, 9000], 1, H, T=64, dtype=torch.bfloat16).check()


@pytest.mark.parametrize("H", [8, 128])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_scales(H, scale):
    Case([200, 65], 1, H, scale=scale).check()


@pytest.mark.parametrize("H", [8, 128])
def test_peaked_weights(H):
    """Logits of some hundreds: references move often."""
    Case([1500, 700], 1, H, T=16, scale=1.0, spread=8.0).check()


@pytest.mark.parametrize("H", [4, 128])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_is_hidden_never_counts(H, value):
    case = Case([70, 200, 129], 4, H, T=48, nodes=[4, 2, 4])
    clean = [x.clone() for x in case.check()]
    for b, n in enumerate(case.lens):                                      # behind the sequence, in its last block
        if n % 48:
            case.cache[int(case.table[b, n // 48]), n % 48:] = value
    got = case.run()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    at = 70 - 2                                                            # new token 2 of sequence 0: hidden from tokens 0 and 1
    case.cache[int(case.table[0, at // 48]), at % 48, 3] = value
    out, lse = case.run()
    assert torch.equal(out[0, :2], clean[0][0, :2]) and torch.equal(out[1:], clean[0][1:]) and torch.equal(lse[0, :2], clean[1][0, :2])
    if math.isnan(value):
        assert out[0, 2:].isnan().all() and lse[0, 2:].isnan().all()


@pytest.mark.parametrize("H", [4, 128])
def test_bad_blocks_and_lengths(H):
    case = Case([100, 100, 300, 90], 1, H, T=16)
    case.table[1, 2] = 10 ** 6
    case.table[0, 0] = -1
    case.lens_t[2] = 301                                                   # beyond max_seq_len
    case.cache[0] = case.cache[0]
    out, lse = case.run()
    assert case.flags.item() == binding.FLAG_BLOCK_RANGE | binding.FLAG_SEQ_LEN_RANGE
    assert (out[2] == 0).all() and (lse[2] == -math.inf).all()
    rows = case.rows(3).double()
    want = torch.softmax(case.q[3, 0].double() @ rows.T * case.scale, -1) @ rows[:, :512]
    assert (out[3, 0].double() - want).abs().max() < 2e-3
    rows = case.cache[case.table[0].clamp(min=0).long()].flatten(0, 1)[:100].double()
    rows[:16] = 0                                                          # rows of zeros
    want = torch.softmax(case.q[0, 0].double() @ rows.T * case.scale, -1) @ rows[:, :512]
    assert (out[0, 0].double() - want).abs().max() < 2e-3
    bad = Case([5, 9], 3, H, nodes=[6, 3])
    out, _ = bad.run()
    assert bad.flags.item() == binding.FLAG_TREE_RANGE and (out[0] == 0).all() and (out[1] != 0).any()


@pytest.mark.parametrize("H", [16, 128])
def test_repeats_streams_and_graphs(H):
    a, b = Case([3000, 77, 512], 1, H, T=16, seed=1), Case([900, 2100, 5], 1, H, T=16, seed=2)
    want = [[x.clone() for x in case.check()] for case in (a, b)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for case, (out, lse) in zip((a, b), want):
        case.out.fill_(0)
        torch.cuda.synchronize()
        got = case.run(side)
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)
    size = max(a.room.numel(), b.room.numel())
    a.room = b.room = torch.zeros(size, dtype=torch.uint8, device="cuda")          # one workspace for both
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for case, graph in zip((a, b), graphs):
        with torch.cuda.graph(graph):
            case.run()
    for turn in range(6):
        graphs[turn % 2].replay()
        if turn == 2:
            a.run()
    torch.cuda.synchronize()
    for case, (out, lse) in zip((a, b), want):
        assert torch.equal(case.out[128:-128].view_as(out), out) and torch.equal(case.lse[32:-32].view_as(lse), lse)


def test_whole_blocks_of_a_latent_pool_are_shared_and_grown():
    """Latent pools as pools of nine heads of 64, one layer as K and one as V pool: a fork that grows gets its own last block."""
    pools = [torch.randn(12, 16, 576, device="cuda").half() for _ in range(2)]
    table = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    table[0, :2] = torch.tensor([5, 6])
    refs = torch.zeros(12, dtype=torch.int32, device="cuda")
    refs[[5, 6]] = 1
    lens = torch.tensor([20, 0], dtype=torch.int32, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.kv_fork(table, refs, lens, torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda"), 16, flags)
    want = torch.tensor([20, 21], dtype=torch.int32, device="cuda")
    room = torch.empty(binding.kv_resize_workspace_bytes(2, 12), dtype=torch.uint8, device="cuda")
    binding.kv_resize([pools[0].view(12, 9, 16, 64)], [pools[1].view(12, 9, 16, 64)], table, refs, lens, want, lens, room, flags)
    torch.cuda.synchronize()
    mine, other = int(table[1, 1]), int(table[0, 1])
    assert flags.item() == 0 and lens.tolist() == [20, 21] and mine != other and int(table[1, 0]) == 5
    for pool in pools:
        assert torch.equal(pool[mine], pool[other])
