"""Speculative decoding as a server runs it: sequences forked from a shared prompt, then steps of make
room, append a tree's K and V, attend in every layer, verify, keep the accepted path and give the rest
back, with a defragmentation on the way.  Everything is held to the oracle after every step: tables,
counts, lengths and all layers' pages bit for bit, the attention of sampled rows in 64 bits, the tokens
exactly; and the cache reads back what the accepted tokens wrote."""
import numpy as np
import pytest
import torch

from oracle import draft as od
from paper_2409_04992_b200 import binding
from tests import gpu_util as gu
from tests.test_gpu_tree_attention import compare, random_tree

pytestmark = pytest.mark.gpu
LAYERS, HEADS, Q_HEADS, DIM, T, VOCAB = 2, 2, 4, 128, 16, 211


def to_gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("nodes,captured", [(5, False), (24, False), (24, True)])
def test_steps(nodes, captured):
    rng = np.random.default_rng(nodes)
    B, M, P = 6, 20, 70
    caches = [rng.standard_normal((P, HEADS, T, DIM), dtype=np.float32).astype(np.float16) for _ in range(2 * LAYERS)]
    table, refs = np.full((B, M), -1, dtype=np.int32), np.zeros(P, dtype=np.int32)
    lens = np.zeros(B, dtype=np.int32)
    # one prompt of 37 tokens, forked into four continuations; another sequence of its own
    lens, flags = od.resize([], table, refs, lens, [37, 0, 0, 0, 0, 50], T)
    assert flags == 0
    gpu = [to_gpu(c) for c in caches]
    k, v = gpu[:LAYERS], gpu[LAYERS:]
    gt, gr, gl = to_gpu(table), to_gpu(refs), to_gpu(lens)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(binding.kv_resize_workspace_bytes(B, P), binding.kv_defragment_workspace_bytes(P),
                         binding.tree_workspace_bytes(B, nodes, Q_HEADS, HEADS, DIM, M * T)), dtype=torch.uint8, device="cuda")
    assert od.fork(table, refs, lens, [0, 0, 0], [1, 2, 3], T) == 0
    binding.kv_fork(gt, gr, gl, to_gpu(np.array([0, 0, 0], dtype=np.int32)), to_gpu(np.array([1, 2, 3], dtype=np.int32)), T, status)

    new = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    buf = dict(want=new(B), trees=new(B), parents=new(B, nodes), tokens=new(B, nodes), u=new(B, nodes, dtype=torch.float32),
               q=new(LAYERS, B, nodes, Q_HEADS, DIM, dtype=torch.float16), kn=new(2 * LAYERS, B, nodes, HEADS, DIM, dtype=torch.float16),
               p=new(B, nodes, VOCAB, dtype=torch.float32), d=new(B, nodes, VOCAB, dtype=torch.float32),
               mask=new(B, nodes, 1, dtype=torch.int64), out=new(LAYERS, B, nodes, Q_HEADS, DIM, dtype=torch.float16),
               lse=new(LAYERS, B, nodes, Q_HEADS, dtype=torch.float32), path=new(B, nodes), count=new(B), said=new(B, nodes), kept=new(B))

    def step():
        binding.kv_resize(k, v, gt, gr, gl, buf["want"], gl, ws, status)
        binding.tree_mask(buf["mask"], buf["parents"], buf["trees"], status)
        for layer in range(LAYERS):
            binding.kv_append_bulk(k[layer], v[layer], buf["kn"][layer], buf["kn"][LAYERS + layer], gl, buf["trees"], gt, status)
            binding.decode_attention_tree(buf["out"][layer], buf["lse"][layer], buf["q"][layer], k[layer], v[layer], gt, gl, buf["trees"],
                                          buf["mask"], M * T, DIM ** -0.5, ws, status)
        binding.verify_tree(buf["path"], buf["count"], buf["said"], buf["p"], buf["d"], buf["tokens"], buf["parents"], buf["trees"],
                            buf["u"], status)
        binding.kv_keep_path(k, v, buf["path"], buf["count"], buf["trees"], gl, buf["kept"], gt, status)
        binding.kv_resize(k, v, gt, gr, gl, buf["kept"], gl, ws, status)

    graph = None
    if captured:
        # (a first call outside: nothing of it is kept, want = the present lengths and no trees)
        buf["want"].copy_(gl)
        with torch.cuda.stream(torch.cuda.Stream()):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for turn in range(5):
        trees = np.array([nodes if n else 0 for n in lens], dtype=np.int32)
        trees[5] = max(1, nodes - turn)
        parents = np.stack([random_tree(rng, t, nodes) for t in trees])
        logits = 2.0 * rng.standard_normal((B, nodes, VOCAB))
        soft = lambda x: (np.exp(x) / np.exp(x).sum(-1, keepdims=True)).astype(np.float32)  # noqa: E731
        p, d = soft(logits), soft(logits + 0.5 * rng.standard_normal(logits.shape))
        tokens = np.array([[rng.choice(VOCAB, p=d[b, max(parents[b, t], 0)] / d[b, max(parents[b, t], 0)].astype(np.float64).sum())
                            for t in range(nodes)] for b in range(B)], dtype=np.int32)
        u = rng.random((B, nodes), dtype=np.float32)
        q = rng.standard_normal((LAYERS, B, nodes, Q_HEADS, DIM), dtype=np.float32).astype(np.float16)
        kn = rng.standard_normal((2 * LAYERS, B, nodes, HEADS, DIM), dtype=np.float32).astype(np.float16)
        for name, value in dict(want=lens + trees, trees=trees, parents=parents, tokens=tokens, u=u, q=q, kn=kn, p=p, d=d).items():
            buf[name].copy_(to_gpu(value))
        graph.replay() if graph else step()
        torch.cuda.synchronize()

        # the same on the CPU
        lens, flags = od.resize(caches, table, refs, lens, lens + trees, T)
        assert flags == 0 and int(status.item()) == 0
        for c, rows in zip(caches, kn):
            for b in range(B):
                for t in range(trees[b]):
                    at = lens[b] - trees[b] + t
                    assert refs[table[b, at // T]] == 1               # nobody else sees what is written
                    c[table[b, at // T], :, at % T] = rows[b, t]
        see = np.stack([od.ancestor_mask(parents[b], trees[b], nodes) for b in range(B)])
        for layer in range(LAYERS):
            want = od.tree_attention(q[layer], caches[layer], caches[LAYERS + layer], table, lens, trees, see, DIM ** -0.5)
            compare(buf["out"][layer].cpu().numpy(), buf["lse"][layer].cpu().numpy(), want, f"turn {turn} layer {layer}", int(lens.max()))
        path, count, said, flags = od.verify(p.astype(np.float64), d.astype(np.float64), tokens, parents, trees, u)
        assert flags == 0
        for name, value in dict(path=path, count=count, said=said).items():
            assert np.array_equal(buf[name].cpu().numpy(), value), (turn, name)
        kept, flags = od.keep_path(caches, path, count, trees, lens, table)
        assert flags == 0
        lens, flags = od.resize(caches, table, refs, lens, kept, T)
        assert flags == 0
        if turn == 2 and not captured:
            table, refs, used, flags = od.defragment(caches, table, refs, lens, T)
            count_gpu = new(1)
            binding.kv_defragment(k, v, gt, gr, gl, gt, gr, count_gpu, ws, status)
            assert flags == 0 and int(count_gpu.item()) == used
        torch.cuda.synchronize()
        assert np.array_equal(gl.cpu().numpy(), lens) and np.array_equal(gr.cpu().numpy(), refs)
        for b in range(B):                                            # (entries behind a sequence's end are anything)
            held = od.blocks_for(lens[b], T)
            assert np.array_equal(gt.cpu().numpy()[b, :held], table[b, :held])
        assert lens[4] == 0 and int(status.item()) == 0
    whole = [gu.bits(g) for g in gpu]
    for i, c in enumerate(caches):
        for b in range(B):
            rows = [(table[b, at // T], at % T) for at in range(lens[b])]
            assert all(np.array_equal(whole[i][r, :, s], c[r, :, s].view(np.uint16)) for r, s in rows)
