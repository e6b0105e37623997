"""The operators as they are used: a speculative step over K and V caches (turned and appended drafts at their depths' positions,
tree attention, logits to probabilities, verification, the kept path), and a step over a latent cache."""
import math

import pytest
import torch

from paper_2409_04992_b200 import binding
from tests.test_gpu_rope_append import table_for, turned

pytestmark = pytest.mark.gpu


def test_a_speculative_step_with_rotary_positions():
    torch.manual_seed(0)
    B, N, Hq, H, D, T, V = 3, 6, 8, 4, 128, 16, 1000
    parents = torch.tensor([[-1, 0, 0, 1, 1, 2]] * B, dtype=torch.int32)
    depth = torch.tensor([0, 1, 1, 2, 2, 2])
    before = [40, 7, 100]
    lens = [n + N for n in before]
    table, blocks = table_for(lens, T)
    kc, vc = (torch.randn(blocks, H, T, D, device="cuda").half() for _ in range(2))
    q, k, v = (torch.randn(B, N, h, D, device="cuda").bfloat16() for h in (Hq, H, H))
    f, m = binding.rope_frequencies(D)
    positions = torch.tensor(before)[:, None] + depth[None]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lens_t, flags = ints(lens), torch.zeros(1, dtype=torch.int32, device="cuda")
    turned_q = torch.zeros(B, N, Hq, D, dtype=torch.float16, device="cuda")
    binding.rope_append(turned_q, kc, vc, q, k, v, f, lens_t, None, table, positions=positions.int().cuda(), magnitude=m, status_flags=flags)
    mask = torch.zeros(B, N, 1, dtype=torch.int64, device="cuda")
    binding.tree_mask(mask, parents.cuda())
    out, max_len = torch.zeros_like(turned_q), max(lens)
    room = torch.empty(binding.tree_workspace_bytes(B, N, Hq, H, D, max_len), dtype=torch.uint8, device="cuda")
    binding.decode_attention_tree(out, None, turned_q, kc, vc, table, lens_t, None, mask, max_len, 1 / math.sqrt(D), room, flags)
    want_q = turned(q, positions.cuda(), f, 1.0, False)
    for b in range(B):
        pages = table[b, :-(-lens[b] // T)].long()
        keys, values = (c[pages].permute(1, 0, 2, 3).flatten(1, 2)[:, :lens[b]].double() for c in (kc, vc))
        keys[:, before[b]:] = turned(k[b:b + 1], positions[b:b + 1].cuda(), f, 1.0, False)[0].transpose(0, 1)
        sees = torch.ones(N, lens[b], dtype=torch.bool, device="cuda")
        sees[:, before[b]:] = torch.stack([(mask[b, :, 0] >> j) & 1 for j in range(N)], -1) != 0
        z = torch.einsum("nhd,hld->hnl", want_q[b], keys.repeat_interleave(2, 0)) / math.sqrt(D)
        want = torch.softmax(z.masked_fill(~sees, -math.inf), -1) @ values.repeat_interleave(2, 0)
        # keys and queries were rounded to fp16: logits off by some 2^-10, weights and the result by twice that
        assert (out[b].double().transpose(0, 1) - want).abs().max() < 2.0 ** -7
    logits = torch.randn(B, N, V, device="cuda") * 3
    tokens = torch.randint(0, V, (B, N), device="cuda").int()
    history, probs = torch.randint(0, V, (B, 50), device="cuda").int(), torch.zeros(B, N, V, device="cuda")
    binding.process_logits(probs, logits, tokens=history, penalties=torch.tensor([[1.3, 0.1, 0.2]] * B, device="cuda"), draft_tokens=tokens, mask=mask,
                           temperatures=torch.full((B,), 0.8, device="cuda"), status_flags=flags)
    assert (probs.sum(-1) - 1).abs().max() < 1e-5
    path, path_lens, emitted = (torch.zeros(*s, dtype=torch.int32, device="cuda") for s in ((B, N), (B,), (B, N)))
    binding.verify_tree(path, path_lens, emitted, probs, None, tokens, parents.cuda(), None, torch.rand(B, N, device="cuda"), flags)
    new_lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    binding.kv_keep_path([kc], [vc], path, path_lens, ints([N] * B), lens_t, new_lens, table, flags)
    torch.cuda.synchronize()
    assert flags.item() == 0
    assert new_lens.tolist() == [n + p for n, p in zip(before, path_lens.tolist())] and bool((path_lens >= 1).all())


@pytest.mark.parametrize("H", [16, 128])
def test_a_step_over_a_latent_cache(H):
    torch.manual_seed(1)
    B, N, T, L = 4, 2, 32, 512
    before = [0, 31, 64, 500]
    lens = [n + N for n in before]
    table, blocks = table_for(lens, T)
    cache = torch.randn(blocks, T, L + 64, device="cuda").bfloat16()
    new, q = torch.randn(B, N, L + 64, device="cuda").bfloat16(), torch.randn(B, N, H, 192, device="cuda").bfloat16()
    up = (torch.randn(H, 128, L, device="cuda") / 10).bfloat16()            # what makes a head's keys of the latent vector, absorbed by its query
    absorbed = torch.zeros(B, N, H, L + 64, dtype=torch.bfloat16, device="cuda")
    absorbed[..., :L] = torch.einsum("bnhd,hdl->bnhl", q[..., :128], up)
    f, m = binding.rope_frequencies(64, scaling="linear", factor=4)
    lens_t, flags = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.latent_append(absorbed, cache, q[..., 128:], new[..., :L], new[..., L:], f, lens_t, None, table, interleaved=True, magnitude=m,
                          status_flags=flags)
    out = torch.zeros(B, N, H, L, dtype=torch.bfloat16, device="cuda")
    room = torch.empty(binding.latent_workspace_bytes(B, N, H, L, 64, max(lens)), dtype=torch.uint8, device="cuda")
    binding.decode_attention_latent(out, None, absorbed, cache, table, lens_t, None, None, max(lens), 1 / math.sqrt(192), room, flags)
    torch.cuda.synchronize()
    assert flags.item() == 0
    for b in range(B):
        rows = cache[table[b, :-(-lens[b] // T)].long()].flatten(0, 1)[:lens[b]].double()
        assert torch.equal(rows[-N:, :L], new[b, :, :L].double())
        z = torch.einsum("nhd,ld->nhl", absorbed[b].double(), rows) / math.sqrt(192)
        z[0, :, -1] = -math.inf
        want = torch.softmax(z, -1) @ rows[:, :L]
        assert bool(((out[b].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3).all())
