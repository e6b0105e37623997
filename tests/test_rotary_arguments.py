"""Arguments of the rotary appends: frequencies between 8-byte boundaries are refused, queries whose heads lie head after head are taken.

As in test_abi.py, made-up device addresses are only handed over in a process that sees no CUDA device."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2409_04992_b200 import binding
from tests.test_decode_step_abi import FAKE, call, lib  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
fake_pointers = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: run in the GPU-less child instead")


@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU here: the tests below run in this process")
def test_they_pass_in_a_child_that_sees_no_gpu():
    done = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-p", "no:cacheprovider", "-m", "not gpu"],
                          cwd=ROOT, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""), capture_output=True, text=True, timeout=600)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-2000:]
    assert " passed" in done.stdout


@fake_pointers
@pytest.mark.parametrize("name", ["instinfer_rope_append", "instinfer_latent_append"])
def test_frequencies_between_boundaries_are_refused(lib, name):  # noqa: F811
    assert call(lib, name, frequencies=FAKE + 4) == binding.ERR_INVALID_ARG


@fake_pointers
def test_queries_head_after_head_are_within_the_checks(lib):  # noqa: F811
    """Strides of q_rope [heads, batch * tokens, 64]: a call without work passes with those that are apart, overlapping parts are refused."""
    name, heads, tokens = "instinfer_latent_append", 4, 2 * 3
    work = dict(batch=2, max_new=3)
    for good in (dict(q_stride=64, q_head_stride=tokens * 64), dict(q_stride=72, q_head_stride=5 * 72 + 64), dict(q_stride=heads * 64, q_head_stride=64)):
        assert call(lib, name, **good, max_new=0) == binding.OK
    for bad in (dict(q_stride=64, q_head_stride=(tokens - 1) * 64 + 56), dict(q_stride=72, q_head_stride=5 * 72 + 56), dict(q_stride=56, q_head_stride=1 << 20)):
        assert call(lib, name, **bad, **work) == binding.ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("B,N,H", [(1, 1, 16), (5, 3, 7), (40, 1, 128), (2, 90, 1)])
def test_queries_head_after_head_are_turned_alike(B, N, H):
    torch.manual_seed(B)
    q = torch.randn(H, B * N, 64, device="cuda").bfloat16().view(H, B, N, 64).permute(1, 2, 0, 3)      # as a product batched over the heads leaves it
    new = torch.randn(B, N, 576, device="cuda").bfloat16()
    f, _ = binding.rope_frequencies(64)
    lens, flags = torch.full((B,), N + 4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    outs = []
    for given in (q, q.contiguous()):
        cache, out = torch.zeros(B, N + 4, 576, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, N, H, 576, dtype=torch.bfloat16, device="cuda")
        binding.latent_append(out, cache, given, new[..., :512], new[..., 512:], f, lens, status_flags=flags)
        outs.append((out, cache))
    assert flags.item() == 0 and all(torch.equal(a, b) for a, b in zip(*outs)) and (outs[0][0][..., 512:] != 0).any(-1).all()
