"""A whole speculative step over latent caches of several layers: room, append, tree attention in every layer, logits to probabilities,
verification, the accepted path's rows moved into place, the blocks given back."""
import math

import pytest
import torch

from paper_2409_04992_b200 import binding
from tests.test_gpu_rope_append import table_for

pytestmark = pytest.mark.gpu


def as_heads(cache):
    """A latent cache or pool as the calls that move rows and blocks take it: one head, 16-bit values whatever their type."""
    return cache.view(torch.float16).unsqueeze(1)


def halves(caches):
    """Layers as K and V caches, half of them each; with an odd number the last one is in both lists, at the same place."""
    heads = [as_heads(c) for c in caches]
    return heads[::2], heads[1::2] + heads[len(heads) // 2 * 2:]


@pytest.mark.parametrize("layers", [1, 2, 3])
@pytest.mark.parametrize("T", [0, 8, 48])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_the_kept_rows_are_the_accepted_ones(layers, T, dtype):
    torch.manual_seed(layers)
    lens, nodes, N = [70, 9, 0, 140], [9, 3, 0, 6], 9
    paths, kept = [[0, 2, 5, 8], [0, 1, 2], [], [1, 5]], [4, 3, 0, 2]
    table, blocks = table_for(lens, T) if T else (None, 0)
    caches = [torch.randn((blocks, T, 576) if T else (4, 150, 576), device="cuda").to(dtype) for _ in range(layers)]
    caches[0].view(torch.int16)[0, 0, :4] = torch.tensor([0x7C01, -1, 0x7F81, -32768], dtype=torch.int16, device="cuda")     # bit copies
    before = [c.clone() for c in caches]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    path = torch.full((4, N), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p)
    new_lens, flags = ints([0] * 4), ints([0])
    k, v = halves(caches)
    binding.kv_keep_path(k, v, path.cuda(), ints(kept), ints(nodes), ints(lens), new_lens, table, flags)
    torch.cuda.synchronize()
    assert flags.item() == 0 and new_lens.tolist() == [n - t + len(p) for n, t, p in zip(lens, nodes, paths)]
    for now, old in zip(caches, before):
        want = old.clone()
        place = lambda b, at: (b, at) if table is None else (int(table[b, at // T]), at % T)  # noqa: E731
        for b, p in enumerate(paths):
            for i, node in enumerate(p):
                want[place(b, lens[b] - nodes[b] + i)] = old[place(b, lens[b] - nodes[b] + node)]
        assert torch.equal(now.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("layers,H", [(3, 16), (2, 128)])
def test_a_speculative_step(layers, H):
    torch.manual_seed(H)
    B, N, T, L, P, V = 3, 6, 16, 512, 60, 300
    parents = torch.tensor([[-1, 0, 0, 1, 1, 2]] * B, dtype=torch.int32)
    depth = torch.tensor([0, 1, 1, 2, 2, 2])
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pools = [torch.randn(P, T, L + 64, device="cuda").bfloat16() for _ in range(layers)]
    k, v = halves(pools)
    table, refs, lens, flags = torch.zeros(B, 20, dtype=torch.int32, device="cuda"), ints([0] * P), ints([0] * B), ints([0])
    room = torch.empty(binding.kv_resize_workspace_bytes(B, P), dtype=torch.uint8, device="cuda")
    before = [40, 7, 100]
    binding.kv_resize(k, v, table, refs, lens, ints(before), lens, room, flags)
    binding.kv_resize(k, v, table, refs, lens, ints([n + N for n in before]), lens, room, flags)
    f, m = binding.rope_frequencies(64)
    mask = torch.zeros(B, N, 1, dtype=torch.int64, device="cuda")
    binding.tree_mask(mask, parents.cuda())
    positions = (torch.tensor(before)[:, None] + depth[None]).int().cuda()
    work = torch.empty(binding.latent_workspace_bytes(B, N, H, L, 64, 320), dtype=torch.uint8, device="cuda")
    for pool in pools:
        new, q = torch.randn(B, N, L + 64, device="cuda").bfloat16(), torch.randn(B, N, H, L + 64, device="cuda").bfloat16()
        binding.latent_append(q, pool, q[..., L:].clone(), new[..., :L], new[..., L:], f, lens, None, table, positions=positions, magnitude=m,
                              status_flags=flags)
        out = torch.zeros(B, N, H, L, dtype=torch.bfloat16, device="cuda")
        binding.decode_attention_latent(out, None, q, pool, table, lens, None, mask, 320, 1 / math.sqrt(192), work, flags)
        assert out.isfinite().all() and (out != 0).any(-1).all()
    logits, tokens = torch.randn(B, N, V, device="cuda"), torch.randint(0, V, (B, N), device="cuda").int()
    # (what the tokens of nodes 2 and 5 are is all but certain behind nodes 0 and 2: the path is theirs)
    for parent, node in ((0, 2), (2, 5)):
        logits[torch.arange(B), parent, tokens[:, node].long()] = 60.0
    probs = torch.zeros(B, N, V, device="cuda")
    binding.process_logits(probs, logits, draft_tokens=tokens, mask=mask, status_flags=flags)
    path, path_lens, emitted, kept = torch.zeros(B, N, dtype=torch.int32, device="cuda"), ints([0] * B), torch.zeros(B, N, dtype=torch.int32, device="cuda"), ints([0] * B)
    binding.verify_tree(path, path_lens, emitted, probs, None, tokens, parents.cuda(), None, torch.rand(B, N, device="cuda"), flags)
    rows = [[pool[table[b, :-(-(n + N) // T)].long()].flatten(0, 1)[:n + N].clone() for b, n in enumerate(before)] for pool in pools]
    binding.kv_keep_path(k, v, path, path_lens, None, lens, kept, table, flags)
    binding.kv_resize(k, v, table, refs, lens, kept, lens, room, flags)
    torch.cuda.synchronize()
    assert flags.item() == 0 and path_lens.tolist() == [3] * B and path[:, :3].tolist() == [[0, 2, 5]] * B
    assert lens.tolist() == [n + 3 for n in before] and int(refs.sum()) == sum(-(-(n + 3) // T) for n in before)
    for pool, old in zip(pools, rows):
        for b, n in enumerate(before):
            now = pool[table[b, :-(-(n + 3) // T)].long()].flatten(0, 1)[:n + 3]
            assert torch.equal(now, old[b][torch.tensor(list(range(n)) + [n, n + 2, n + 5], device="cuda")])


@pytest.mark.parametrize("layers", [1, 3])
def test_blocks_of_an_odd_number_of_layers_are_shared_and_tidied(layers):
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pools = [torch.randn(12, 16, 576, device="cuda").half() for _ in range(layers)]
    k, v = halves(pools)
    table, refs = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), ints([0] * 12)
    table[0, :2] = ints([9, 6])
    refs[[9, 6]] = 1
    lens, flags = ints([20, 0]), ints([0])
    binding.kv_fork(table, refs, lens, ints([0]), ints([1]), 16, flags)
    room = torch.empty(max(binding.kv_resize_workspace_bytes(2, 12), binding.kv_defragment_workspace_bytes(12)), dtype=torch.uint8, device="cuda")
    rows = lambda b, n: [pool[table[b, :-(-n // 16)].long()].flatten(0, 1)[:n].clone() for pool in pools]  # noqa: E731
    old = rows(0, 20)
    binding.kv_resize(k, v, table, refs, lens, ints([20, 21]), lens, room, flags)
    assert flags.item() == 0 and int(table[1, 1]) != int(table[0, 1])
    assert all(torch.equal(a, b) for a, b in zip(rows(1, 20), old)) and all(torch.equal(a, b) for a, b in zip(rows(0, 20), old))
    used = ints([0])
    binding.kv_defragment(k, v, table, refs, lens, table, refs, used, room, flags)
    assert flags.item() == 0 and used.item() == 3 and int(table[0, 0]) < 3
    assert all(torch.equal(a, b) for a, b in zip(rows(1, 20), old)) and all(torch.equal(a, b) for a, b in zip(rows(0, 20), old))
