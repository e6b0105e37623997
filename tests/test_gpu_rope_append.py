"""Rotary appends against the definition in 64 bits.  A turned value is two 32-bit products of inputs with a sine that is off by
2^-22 at most, added, then rounded once to 16 bits: half a step of the result and 2^-20 of the inputs' size cover it."""
import math

import pytest
import torch

from paper_2409_04992_b200 import binding

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
CASES = [  # batch, tokens, q heads, kv heads, head size, rotary dims, page, type, interleaved, first position
    (1, 1, 40, 40, 128, 128, 0, torch.float16, False, 0), (3, 1, 8, 2, 64, 16, 8, torch.bfloat16, True, 0),
    (5, 7, 6, 3, 256, 256, 16, torch.float32, False, 1 << 20), (4, 33, 4, 4, 128, 64, 48, torch.float16, True, 1 << 24),
    (2, 900, 8, 1, 128, 128, 64, torch.bfloat16, False, 0), (700, 1, 2, 1, 64, 64, 16, torch.float16, False, -5), (1, 1, 0, 1, 64, 32, 0, torch.float32, True, 0)]


def turned(x, positions, f, magnitude, interleaved):
    half = f.numel()
    angle = positions.double()[:, :, None, None] * f
    cos, sin = angle.cos() * magnitude, angle.sin() * magnitude
    part = x.double()[..., :2 * half]
    a, b = (part[..., ::2], part[..., 1::2]) if interleaved else (part[..., :half], part[..., half:])
    new = (a * cos - b * sin, a * sin + b * cos)
    return torch.cat((torch.stack(new, -1).flatten(-2) if interleaved else torch.cat(new, -1), x.double()[..., 2 * half:]), -1)


def near(got, want, size, dtype):
    error = (got.double() - want).abs()
    return bool((error <= HALF_STEP[dtype] * want.abs() + 2.0 ** -20 * size + 2.0 ** -25).all())


def table_for(lens, T, device="cuda"):
    blocks = sum(-(-n // T) for n in lens) + 3
    ids = torch.randperm(blocks)
    table, at = torch.full((len(lens), max(1, -(-max(lens) // T))), -7, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        need = -(-n // T)
        table[b, :need] = ids[at:at + need]
        at += need
    return table.to(device), blocks


def place(cache, table, b, at, T):
    return cache[b, :, at] if table is None else cache[int(table[b, at // T]), :, at % T]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("given", [False, True])
def test_turned_and_appended(case, given):
    B, N, Hq, H, D, R, T, dtype, interleaved, first = case
    torch.manual_seed(3)
    fresh = [max(0, N - b % 3) for b in range(B)]
    lens = [fresh[b] + b % 5 for b in range(B)]
    x = torch.randn(B, N, Hq + 2 * H, D, device="cuda").to(dtype)
    q, k, v = x.split([Hq, H, H], dim=2)
    table, blocks = table_for(lens, T) if T else (None, 0)
    shape = (blocks, H, T, D) if T else (B, H, max(max(lens), 1), D)
    kc, vc = (torch.full(shape, 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    q_out = torch.full((B, N, Hq, D), 5.0, dtype=torch.float16, device="cuda")
    f, magnitude = binding.rope_frequencies(R, scaling="by_parts", factor=8, trained_len=4096)
    cache_at = torch.tensor(lens)[:, None] - torch.tensor(fresh)[:, None] + torch.arange(N)[None]
    positions = (cache_at + first).int().cuda() if given else None
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.tensor(fresh, dtype=torch.int32, device="cuda"), table)
    binding.rope_append(q_out if Hq else None, kc, vc, q if Hq else None, k, v, f, *args, positions=positions, interleaved=interleaved,
                        magnitude=magnitude, status_flags=flags)
    torch.cuda.synchronize()
    assert flags.item() == 0
    at = (cache_at + (first if given else 0)).cuda()
    want_q, want_k = turned(q, at, f, magnitude, interleaved), turned(k, at, f, magnitude, interleaved)
    written_k, written_v = (torch.zeros(shape[:3], dtype=torch.bool, device="cuda") for _ in range(2))
    for b in range(B) if B < 50 else list(range(20)) + [B - 1]:
        for t in range(fresh[b]):
            assert near(place(kc, table, b, int(cache_at[b, t]), T), want_k[b, t], 10, torch.float16), (b, t)
            assert torch.equal(place(vc, table, b, int(cache_at[b, t]), T), v[b, t].half())
        if Hq:
            assert near(q_out[b, :fresh[b]], want_q[b, :fresh[b]], 10, torch.float16)
            assert (q_out[b, fresh[b]:] == 5.0).all()                     # rows of tokens that there are not stay
    assert int((kc != 9.0).any(-1).sum()) <= sum(fresh) * H and int((vc != 9.0).any(-1).sum()) <= sum(fresh) * H


@pytest.mark.parametrize("case", [(1, 1, 16, 512, 0, torch.float16, False), (5, 3, 7, 512, 8, torch.bfloat16, True), (40, 1, 128, 512, 64, torch.bfloat16, False),
                                  (3, 600, 1, 512, 48, torch.float16, True), (2, 4, 0, 512, 16, torch.float16, False)])
def test_latent_rows(case):
    B, N, H, L, T, dtype, interleaved = case
    torch.manual_seed(4)
    fresh = [max(0, N - b % 2) for b in range(B)]
    lens = [fresh[b] + b % 7 for b in range(B)]
    new = torch.randn(B, N, L + 64, device="cuda").to(dtype)
    q = torch.randn(B, N, H, 192, device="cuda").to(dtype)
    table, blocks = table_for(lens, T) if T else (None, 0)
    cache = torch.full((blocks, T, L + 64) if T else (B, max(max(lens), 1), L + 64), 9.0, dtype=dtype, device="cuda")
    q_out = torch.full((B, N, H, L + 64), 5.0, dtype=dtype, device="cuda")
    f, _ = binding.rope_frequencies(64)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.latent_append(q_out if H else None, cache, q[..., 128:] if H else None, new[..., :L], new[..., L:], f,
                          torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.tensor(fresh, dtype=torch.int32, device="cuda"), table,
                          interleaved=interleaved, status_flags=flags)
    torch.cuda.synchronize()
    assert flags.item() == 0
    at = (torch.tensor(lens)[:, None] - torch.tensor(fresh)[:, None] + torch.arange(N)[None]).cuda()
    want_q, want_k = turned(q[..., 128:], at, f, 1.0, interleaved), turned(new[..., L:][:, :, None], at, f, 1.0, interleaved)[:, :, 0]
    for b in range(B):
        for t in range(fresh[b]):
            p = int(at[b, t])
            row = cache[b, p] if table is None else cache[int(table[b, p // T]), p % T]
            assert torch.equal(row[:L], new[b, t, :L]) and near(row[L:], want_k[b, t], 10, dtype)
        if H:
            assert near(q_out[b, :fresh[b], :, L:], want_q[b, :fresh[b]], 10, dtype)
            assert (q_out[b, fresh[b]:] == 5.0).all() and (q_out[b, :, :, :L] == 5.0).all()
    assert int((cache != 9.0).any(-1).sum()) == sum(fresh)


def test_a_plain_append_without_turning_equals_the_append():
    """Frequencies of 0: the same bits as instinfer_kv_append_bulk's."""
    k, v = (torch.randn(3, 5, 4, 128, device="cuda").half() for _ in range(2))
    lens, fresh = torch.tensor([5, 9, 4], dtype=torch.int32, device="cuda"), torch.tensor([5, 2, 0], dtype=torch.int32, device="cuda")
    caches = [torch.zeros(3, 4, 16, 128, dtype=torch.float16, device="cuda") for _ in range(4)]
    binding.kv_append_bulk(caches[0], caches[1], k, v, lens, fresh)
    binding.rope_append(None, caches[2], caches[3], None, k, v, torch.zeros(64, dtype=torch.float64, device="cuda"), lens, fresh)
    assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])


def test_in_place_and_without_new_lens():
    q, k, v = (torch.randn(4, 1, h, 64, device="cuda").half() for h in (8, 2, 2))
    lens = torch.tensor([3, 0, 16, 1], dtype=torch.int32, device="cuda")
    f, _ = binding.rope_frequencies(64)
    kc, vc = (torch.zeros(4, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    apart, same = torch.zeros_like(q), q.clone()
    binding.rope_append(apart, kc, vc, q, k, v, f, lens)
    binding.rope_append(same, kc, vc, same, k, v, f, lens)
    assert torch.equal(apart[[0, 2, 3]], same[[0, 2, 3]]) and torch.equal(same[1], q[1])      # length 0: not a token
    assert kc[1].abs().sum() == 0


def test_lengths_and_blocks_out_of_range():
    q, k, v = (torch.randn(5, 2, h, 64, device="cuda").half() for h in (2, 1, 1))
    f, _ = binding.rope_frequencies(32)
    table = torch.tensor([[0, 1], [2, 3], [99, 4], [5, 6], [7, 8]], dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros(9, 1, 8, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    out = torch.zeros_like(q)
    lens = torch.tensor([2, 17, 2, -1, 1], dtype=torch.int32, device="cuda")
    fresh = torch.tensor([2, 2, 2, 1, 2], dtype=torch.int32, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.rope_append(out, kc, vc, q, k, v, f, lens, fresh, table, status_flags=flags)
    assert flags.item() == binding.FLAG_SEQ_LEN_RANGE | binding.FLAG_BLOCK_RANGE
    assert out[0].abs().sum() > 0 and out[2].abs().sum() > 0 and out[[1, 3, 4]].abs().sum() == 0
    assert kc[0].abs().sum() > 0 and kc[1:].abs().sum() == 0 and vc[1:].abs().sum() == 0


def test_values_beyond_fp16_become_infinities():
    k = torch.full((1, 1, 1, 64), 1e6, device="cuda")
    kc, vc = (torch.zeros(1, 1, 1, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    binding.rope_append(None, kc, vc, None, k, -k, torch.zeros(8, dtype=torch.float64, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"))
    assert (kc == math.inf).all() and (vc == -math.inf).all()
