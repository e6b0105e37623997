"""Calls of the decode step's operators that the header allows: optional arguments in every combination, rows in place whatever their
alignment, offsets beyond 32 bits, many sequences with some out of range, two streams at once, a first call that is captured."""
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2409_04992_b200 import binding
from tests import test_gpu_process_logits as logits
from tests.test_gpu_latent_attention import Case
from tests.test_gpu_rope_append import near, turned

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OPTIONS = ["tokens", "token_lens", "prompt_lens", "penalties", "draft_tokens", "mask", "bias", "allowed", "temperatures"]


@pytest.mark.parametrize("combination", range(0, 1 << len(OPTIONS), 3))
def test_every_combination_of_what_is_given(combination):
    B, N, V = 3, 5, (700, 4099, 20001)[combination % 7 % 3]
    s = logits.make(B, N, V, 40, (torch.float32, torch.bfloat16, torch.float16)[combination % 3], combination, bias=3, pad=combination % 5)
    given = {name for i, name in enumerate(OPTIONS) if combination >> i & 1}
    sees = torch.tril(torch.ones(N, N, dtype=torch.bool)).expand(B, N, N)
    if "mask" in given:
        sees = torch.stack([(s["mask"][:, :, 0].cpu() >> j) & 1 for j in range(N)], -1) != 0
    args = dict(s)
    for name in OPTIONS:
        if name not in given:
            for key in (("bias_tokens", "bias_values") if name == "bias" else (name,)):
                args.pop(key)
    has = lambda name: s[name] if name in given else None  # noqa: E731
    lens = s["token_lens"].tolist() if "token_lens" in given else [40] * B
    prompts = s["prompt_lens"].tolist() if "prompt_lens" in given else [0] * B
    if "tokens" not in given:
        lens, prompts = [0] * B, [0] * B
    bias = (s["bias_tokens"], s["bias_values"]) if "bias" in given else (None, None)
    args.pop("logits")
    if "tokens" not in given:                                     # (lengths of a history that there is not are not looked at)
        args.pop("token_lens", None)
        args.pop("prompt_lens", None)
    want = logits.reference(s["logits"], has("tokens"), lens, prompts, has("penalties"), has("draft_tokens"), sees, *bias, has("allowed"), has("temperatures"))
    out = torch.full((B, N, V), 7.0, device="cuda")
    binding.process_logits(out, s["logits"], **args)
    assert s["status_flags"].item() == 0 and logits.close(out, want, torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("V,pad", [(997, 0), (997, 3), (50257, 0), (131071, 2), (4096, 5)])
def test_in_place_between_boundaries(dtype, V, pad):
    s = logits.make(2, 3, V, 50, dtype, V + pad, bias=2, pad=pad)
    whole = s["logits"]._base if s["logits"]._base is not None else s["logits"]
    behind = whole[..., V:].clone()
    want = logits.want_of(s)
    binding.process_logits(s["logits"], **s)
    assert logits.close(s["logits"], want, dtype) and torch.equal(whole[..., V:], behind)


def test_logits_beyond_32_bits():
    rows, V = 17000, 131073                                        # 2.2e9 values
    z = torch.zeros(rows, 1, V, dtype=torch.bfloat16, device="cuda")
    at = torch.arange(rows, device="cuda") * 7 % V
    z[torch.arange(rows, device="cuda"), 0, at] = 12.0
    out = torch.full_like(z, 3.0)
    binding.process_logits(out, z)
    top = math.exp(12) / (math.exp(12) + V - 1)
    peak = out[torch.arange(rows, device="cuda"), 0, at].double()
    assert bool(((peak - top).abs() <= (2.0 ** -8 + 2.0 ** -16) * top).all())
    out[torch.arange(rows, device="cuda"), 0, at] = 0
    rest = torch.tensor((1 - top) / (V - 1)).bfloat16()
    assert out.view(torch.int16).amax() <= rest.view(torch.int16) + 1 and bool((out[-3:].double().sum(-1) > 0.5 * (1 - top)).all())


def test_appends_and_latent_attention_beyond_32_bits():
    P, T = 60000, 64                                               # 2.2e9 values of latent rows
    pool = torch.zeros(P, T, 576, dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([[P - 1, 0], [P - 2, P - 3]], dtype=torch.int32, device="cuda")
    lens, flags = torch.tensor([70, 100], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    new, q = torch.randn(2, 100, 576, device="cuda").bfloat16(), torch.randn(2, 1, 16, 576, device="cuda").bfloat16()
    f, _ = binding.rope_frequencies(64)
    binding.latent_append(None, pool, None, new[..., :512], new[..., 512:], f, lens, lens, table, status_flags=flags)
    out = torch.zeros(2, 1, 16, 512, dtype=torch.bfloat16, device="cuda")
    room = torch.empty(binding.latent_workspace_bytes(2, 1, 16, 512, 64, 128), dtype=torch.uint8, device="cuda")
    binding.decode_attention_latent(out, None, q, pool, table, lens, None, None, 128, 0.07, room, flags)
    at = torch.arange(100, device="cuda")
    for b, n in enumerate((70, 100)):
        rows = pool[table[b].long()].flatten(0, 1)[:n]
        assert torch.equal(rows[:, :512], new[b, :n, :512])
        assert near(rows[:, 512:], turned(new[b:b + 1, :n, 512:][:, :, None], at[None, :n], f, 1.0, False)[0, :, 0], 10, torch.bfloat16)
        want = torch.softmax(q[b, 0].double() @ rows.double().T * 0.07, -1) @ rows[:, :512].double()
        assert (out[b, 0].double() - want).abs().max() < 2.0 ** -8 * want.abs().max() + 1e-4
    del pool
    P, H, D = 16500, 8, 256                                        # 2.2e9 values of keys
    k, v = (torch.zeros(P, H, T, D, dtype=torch.float16, device="cuda") for _ in range(2))
    x = torch.randn(2, 100, H, D, device="cuda").half()
    table = torch.tensor([[P - 1, 0], [P - 2, P - 3]], dtype=torch.int32, device="cuda")
    binding.rope_append(None, k, v, None, x, x, torch.zeros(D // 2, dtype=torch.float64, device="cuda"), lens, lens, table, status_flags=flags)
    for b, n in enumerate((70, 100)):
        for cache in (k, v):
            assert torch.equal(cache[table[b].long()].transpose(1, 2).flatten(0, 1)[:n], x[b, :n])
    assert flags.item() == 0


@pytest.mark.parametrize("H", [8, 128])
def test_many_sequences_of_which_some_are_out_of_range(H):
    B = 90
    case = Case([50 + 3 * b for b in range(B)], 2, H, T=16, nodes=[2] * B)
    clean = [x.clone() for x in case.run()]
    assert case.flags.item() == 0
    case.lens_t[40], case.nodes_t[77], case.lens_t[5] = case.max_len + 1, 3, -1
    out, lse = case.run()
    assert case.flags.item() == binding.FLAG_SEQ_LEN_RANGE | binding.FLAG_TREE_RANGE
    for b in (5, 40, 77):
        assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
    good = torch.tensor([b for b in range(B) if b not in (5, 40, 77)], device="cuda")
    # (other cuts of the work: other roundings of the 32-bit sums)
    assert (out[good].double() - clean[0][good].double()).abs().max() < 2.0 ** -9 and (lse[good] - clean[1][good]).abs().max() < 1e-5


@pytest.mark.parametrize("H", [16, 128])
def test_two_streams_at_once(H):
    cases = [Case([3000, 77, 512], 1, H, T=16, seed=1), Case([900, 2100, 5], 1, H, T=16, seed=2)]
    rows = [logits.make(8, 3, 30001, 100, torch.bfloat16, i, bias=3) for i in (1, 2)]
    outs = [torch.zeros(8, 3, 30001, device="cuda") for _ in rows]
    want = []
    for case, s, out in zip(cases, rows, outs):
        case.run()
        binding.process_logits(out, **s)
        want.append((case.out.clone(), case.lse.clone(), out.clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for turn in range(20):
        for case, s, out, stream in zip(cases, rows, outs, streams):
            case.run(stream)
            binding.process_logits(out, **s, stream=stream)
    torch.cuda.synchronize()
    for case, out, (o, lse, probs) in zip(cases, outs, want):
        assert torch.equal(case.out, o) and torch.equal(case.lse, lse) and torch.equal(out, probs)


FIRST = """
import torch
from paper_2409_04992_b200 import binding
from tests.test_gpu_latent_attention import Case
from tests import test_gpu_process_logits as logits
s = logits.make(30, 2, 131072, 100, torch.bfloat16, 1, bias=3)
out = torch.zeros(30, 2, 131072, device="cuda")
cases = [Case([300, 5, 0], 1, H, T=16) for H in (16, 128)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    binding.process_logits(out, **s)
    for case in cases:
        case.run()
for _ in range(2):
    graph.replay()
torch.cuda.synchronize()
first, rows = out.clone(), [c.out.clone() for c in cases]
binding.process_logits(out, **s)
for case in cases:
    case.check()
assert torch.equal(out, first) and all(torch.equal(c.out, r) for c, r in zip(cases, rows)) and logits.close(out, logits.want_of(s), torch.float32)
print("captured first")
"""


def test_a_first_call_that_is_captured():
    done = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert done.returncode == 0 and "captured first" in done.stdout, done.stdout[-2000:] + done.stderr[-2000:]
