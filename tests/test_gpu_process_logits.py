"""Logits to probabilities against the definition in 64 bits.  In 32 bits a probability is off by the rounding of its exponent
(2^-23 of (max z - z) / T, some tens at most, and of the penalties' arithmetic) and of the sum: 2^-16 of its value covers it,
and half a step of the output's type; what is below 2^-126 may be 0, and fp16 steps end at 2^-24."""
import math

import pytest
import torch

from paper_2409_04992_b200 import binding

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def reference(z, history, lens, prompts, penalties, drafts, sees, bias_tokens, bias, allowed, hot, probabilities=True):
    B, N, V = z.shape
    z = z.double().cpu().clone()
    out = torch.zeros(B, N, V, dtype=torch.float64)
    for b in range(B):
        for t in range(N):
            x = z[b, t].clone()
            if penalties is not None:
                count, asked = torch.zeros(V, dtype=torch.float64), torch.zeros(V, dtype=torch.bool)
                if history is not None:
                    h = history[b, :lens[b]].long().cpu()
                    ok = (h >= 0) & (h < V)
                    asked[h[:prompts[b]][ok[:prompts[b]]]] = True
                    count += torch.bincount(h[prompts[b]:][ok[prompts[b]:]], minlength=V).double()
                if drafts is not None:
                    for j in range(N):
                        if sees[b, t, j]:
                            count[int(drafts[b, j])] += 1
                r, f, p = penalties[b].double().tolist()
                said = asked | (count > 0)
                x = torch.where(said, torch.where(x > 0, x / r, x * r), x)
                x = x - f * count - p * (count > 0)
            if bias_tokens is not None:
                for token, value in zip(bias_tokens[b].tolist(), bias[b].double().tolist()):
                    if 0 <= token < V:
                        x[token] += value
            if allowed is not None:
                bits = (allowed[b, t].cpu().long()[:, None] >> torch.arange(32)) & 1
                x = x.masked_fill(bits.flatten()[:V] == 0, -math.inf)
            T = float(hot[b]) if hot is not None else 1.0
            if not probabilities:
                out[b, t] = x / T if T > 0 else x
            elif x.max() == -math.inf:
                pass
            elif T > 0:
                out[b, t] = torch.softmax((x - x.max()) / T, -1)
            else:
                out[b, t, int((x == x.max()).nonzero()[0])] = 1.0
    return out


def make(B, N, V, M, dtype, seed, bias=0, mask=True, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    whole = (4 * torch.randn(B, N, V + pad, generator=g, device="cuda")).to(dtype)
    history = (torch.rand(B, max(M, 1), generator=g, device="cuda").pow(3) * V).int().clamp(max=V - 1)
    lens = torch.tensor([max(0, M - 3 * b) for b in range(B)], dtype=torch.int32)
    s = dict(logits=whole[..., :V], tokens=history, token_lens=lens.cuda(), prompt_lens=(lens // 3).cuda(),
             penalties=torch.tensor([[1.0 + 0.1 * (b % 4), 0.25 * (b % 3), 0.5 * (b % 2)] for b in range(B)], device="cuda"),
             temperatures=torch.tensor([0.0 if b % 4 == 3 else 0.5 + 0.25 * b % 2 for b in range(B)], device="cuda"),
             status_flags=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if N > 1:
        parents = torch.tensor([[-1] + [int(torch.randint(0, t, (1,))) for t in range(1, N)] for _ in range(B)], dtype=torch.int32, device="cuda")
        s["mask"] = torch.zeros(B, N, (N + 63) // 64, dtype=torch.int64, device="cuda")
        binding.tree_mask(s["mask"], parents)
        s["draft_tokens"] = (torch.rand(B, N, generator=g, device="cuda").pow(3) * V).int().clamp(max=V - 1)
    if bias:
        s["bias_tokens"] = torch.randint(0, V, (B, bias), generator=g, device="cuda").int()
        s["bias_tokens"][:, -1] = -1
        if bias > 2:
            s["bias_tokens"][:, 1] = s["bias_tokens"][:, 0]                # listed twice
        s["bias_values"] = torch.randn(B, bias, generator=g, device="cuda") * 3
    if mask:
        s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (B, N, (V + 31) // 32), generator=g, device="cuda").int()
        s["allowed"][:, :, 0] |= 1
    return s


def want_of(s, **kw):
    B, N, V = s["logits"].shape
    j = torch.arange(N)
    sees = None
    if "draft_tokens" in s:
        m = s["mask"].cpu()
        sees = torch.stack([(m[:, :, k // 64] >> (k % 64)) & 1 for k in range(N)], -1) != 0
    return reference(s["logits"], s.get("tokens"), s["token_lens"].tolist(), s["prompt_lens"].tolist(), s.get("penalties"),
                     s.get("draft_tokens"), sees, s.get("bias_tokens"), s.get("bias_values"), s.get("allowed"), s.get("temperatures"), **kw)


def close(got, want, dtype):
    error = (got.double().cpu() - want).abs()
    return bool((error <= (HALF[dtype] + 2.0 ** -16) * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126)).all())


@pytest.mark.parametrize("V", [1, 2, 3, 31, 33, 1000, 4097, 16385, 50257, 131071, 262144])
@pytest.mark.parametrize("kinds", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float16, torch.bfloat16), (torch.bfloat16, torch.float16)])
def test_vocabularies_and_types(V, kinds):
    s = make(3, 1, V, 200, kinds[0], V, bias=5 if V > 5 else 0)
    out = torch.zeros(3, 1, V, dtype=kinds[1], device="cuda")
    binding.process_logits(out, **s)
    assert close(out, want_of(s), kinds[1]) and s["status_flags"].item() == 0


@pytest.mark.parametrize("B,N,V", [(2, 7, 999), (3, 32, 4096), (1, 128, 513), (40, 4, 2049), (300, 1, 101)])
@pytest.mark.parametrize("in_place", [False, True])
def test_trees_and_batches(B, N, V, in_place):
    s = make(B, N, V, 90, torch.float32, 5, bias=3)
    want = want_of(s)
    out = s["logits"] if in_place else torch.zeros(B, N, V, device="cuda")
    binding.process_logits(out, **s)
    assert close(out, want, torch.float32)


@pytest.mark.parametrize("pad,out_pad", [(0, 1), (3, 0), (47, 47), (1, 1)])
def test_padded_rows(pad, out_pad):
    s = make(5, 3, 997, 50, torch.bfloat16, 6, pad=pad)
    whole = torch.full((5, 3, 997 + out_pad), 9.0, device="cuda")
    binding.process_logits(whole[..., :997], **s)
    assert close(whole[..., :997], want_of(s), torch.float32) and (whole[..., 997:] == 9.0).all()


@pytest.mark.parametrize("V", [100, 40001])
def test_logits_out(V):
    s = make(4, 2, V, 60, torch.float32, 7, bias=4)
    out = torch.zeros(4, 2, V, device="cuda")
    binding.process_logits(out, probabilities=False, **s)
    want = want_of(s, probabilities=False)
    got = out.double().cpu()
    left = want > -math.inf
    assert torch.equal(left, got > -math.inf) and bool(((got - want)[left].abs() <= 2.0 ** -20 * (1 + want[left].abs())).all())


def test_nothing_given_is_a_softmax():
    z = torch.randn(7, 1, 3001, device="cuda")
    out = torch.zeros_like(z)
    binding.process_logits(out, z)
    assert close(out, torch.softmax(z.double(), -1).cpu(), torch.float32)


@pytest.mark.parametrize("V", [64, 9000])
def test_nothing_left_infinities_and_nan(V):
    z = torch.randn(6, 1, V, device="cuda")
    allowed = torch.full((6, 1, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    allowed[0] = 0                                                         # a grammar that leaves nothing
    z[1, 0, 5], z[2, 0, 5], z[3, 0, 5] = math.nan, math.inf, math.nan
    allowed[1, 0, 0] &= ~(1 << 5)                                          # a NaN that is not allowed
    z[4] = -math.inf
    hot = torch.tensor([1.0, 1.0, 1.0, 1.0, 1.0, 0.0], device="cuda")
    z[5, 0, 40] = z[5, 0, 50] = 99.0                                       # greedy: the lower one of two
    z[5, 0, 60] = math.nan
    out = torch.full_like(z, 7.0)
    binding.process_logits(out, z, allowed=allowed, temperatures=hot)
    assert (out[0] == 0).all() and (out[4] == 0).all() and out[2].isnan().all() and out[3].isnan().all()
    rest = z[1, 0].double().clone()
    rest[5] = -math.inf
    assert close(out[1, 0], torch.softmax(rest, -1).cpu(), torch.float32)
    assert int(out[5, 0].argmax()) == 40 and out[5].sum() == 1


def test_rows_that_there_are_not_stay_and_ranges_are_flagged():
    s = make(3, 4, 500, 20, torch.float32, 8)
    s["tree_lens"] = torch.tensor([4, 2, 5], dtype=torch.int32, device="cuda")
    out = torch.full((3, 4, 500), 7.0, device="cuda")
    binding.process_logits(out, **s)
    assert s["status_flags"].item() == binding.FLAG_TREE_RANGE
    assert close(out[0], want_of(s)[0], torch.float32) and close(out[1, :2], want_of(s)[1, :2], torch.float32)
    assert (out[1, 2:] == 7.0).all() and (out[2] == 7.0).all()
    s = make(2, 1, 500, 20, torch.float32, 9)
    s["tokens"][0, 3], s["tokens"][1, 2] = -1, 500
    out = torch.zeros(2, 1, 500, device="cuda")
    binding.process_logits(out, **s)
    assert s["status_flags"].item() == binding.FLAG_TOKEN_RANGE and close(out, want_of(s), torch.float32)


def test_a_long_history_of_one_token():
    V, M = 2000, 100000
    z = torch.zeros(1, 1, V, device="cuda")
    tokens = torch.full((1, M), 7, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(z)
    binding.process_logits(out, z, tokens=tokens, penalties=torch.tensor([[1.0, 1e-5, 0.0]], device="cuda"))
    want = torch.zeros(V, dtype=torch.float64)
    want[7] = -float(torch.tensor(1e-5)) * M
    assert close(out[0, 0], torch.softmax(want, -1), torch.float32)


def test_captured_and_replayed():
    s = make(70, 3, 5001, 300, torch.bfloat16, 10, bias=4)
    out = torch.zeros(70, 3, 5001, device="cuda")
    binding.process_logits(out, **s)
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.process_logits(out, **s)
    out.zero_()
    for _ in range(3):
        graph.replay()
    assert torch.equal(out, first)
