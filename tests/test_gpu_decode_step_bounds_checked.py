"""Rotary appends, the latent cache and the logits in the bounds-checking build of the library: no kernel computes an offset outside what the
call's shapes imply.  The cases here assert the status word themselves; the operators' own tests run in that build too."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2409_04992_b200 import binding, build
from tests import test_gpu_process_logits as logits
from tests.test_gpu_latent_attention import Case
from tests.test_gpu_rope_append import table_for

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join("tests", os.path.basename(__file__))
CASES = ["tests/test_gpu_rope_append.py", "tests/test_gpu_latent_attention.py", "tests/test_gpu_process_logits.py",
         "tests/test_gpu_decode_step_operators.py", "tests/test_gpu_latent_speculative_step.py", HERE]
in_the_child = "DECODE_STEP_BOUNDS" in os.environ


@pytest.mark.skipif(in_the_child, reason="this is the child")
def test_no_bounds_flag_in_the_checked_build():
    library = build.build(checked=True)
    done = subprocess.run([sys.executable, "-m", "pytest", *CASES, "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider"], cwd=ROOT,
                          env=dict(os.environ, INSTINFER_LIBRARY=str(library), DECODE_STEP_BOUNDS="1"), capture_output=True, text=True, timeout=1800)
    assert done.returncode == 0, done.stdout[-4000:] + done.stderr[-2000:]
    assert " passed" in done.stdout


@pytest.mark.parametrize("B,N,D,T", [(1, 1, 64, 0), (5, 7, 128, 0), (3, 200, 256, 24), (90, 1, 128, 8), (2, 2500, 64, 64)])
def test_rotary_appends(B, N, D, T):
    lens = [N + 5 * (b % 4) for b in range(B)]
    table, blocks = table_for(lens, T) if T else (None, 0)
    k, v, q = (torch.randn(B, N, h, D, device="cuda").half() for h in (2, 2, 6))
    caches = [torch.zeros((blocks, 2, T, D) if T else (B, 2, max(lens), D), dtype=torch.float16, device="cuda") for _ in range(2)]
    latent, pool = torch.randn(B, N, 576, device="cuda").half(), torch.zeros((blocks, T, 576) if T else (B, max(lens), 576), dtype=torch.float16, device="cuda")
    turned = torch.zeros(B, N, 3, 576, dtype=torch.float16, device="cuda")
    lens_t, flags = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.rope_append(torch.zeros_like(q), *caches, q, k, v, binding.rope_frequencies(D)[0], lens_t, None, table, status_flags=flags)
    binding.latent_append(turned, pool, torch.randn(B, N, 3, 64, device="cuda").half(), latent[..., :512], latent[..., 512:],
                          binding.rope_frequencies(64)[0], lens_t, None, table, status_flags=flags)
    assert flags.item() == 0


@pytest.mark.parametrize("lens,N,H,T", [([1], 1, 1, 0), ([5, 70, 1000], 3, 16, 0), ([9, 64, 129, 4000], 8, 16, 8), ([300, 8] * 20, 2, 7, 24),
                                        ([40, 700, 4100], 40, 16, 16), ([128, 129, 130], 128, 128, 64)])
def test_latent_attention(lens, N, H, T):
    case = Case(lens, N, H, T=T, nodes=[max(1, min(N, n) - b % 3) for b, n in enumerate(lens)])
    case.check()
    assert case.flags.item() == 0


@pytest.mark.parametrize("B,N,V,pad", [(1, 1, 1, 0), (3, 1, 33, 2), (2, 5, 999, 1), (40, 3, 4097, 0), (4, 2, 50257, 0), (1, 1, 262144, 0), (3, 1, 262143, 0),
                                       (1, 7, 131071, 1)])
def test_logits(B, N, V, pad):
    s = logits.make(B, N, V, 60, torch.bfloat16, V, bias=4 if V > 4 else 0, pad=pad)
    for out_pad in (0, 1, pad):
        whole = torch.full((B, N, V + out_pad), 7.0, device="cuda")
        binding.process_logits(whole[..., :V], **s)
        assert s["status_flags"].item() == 0 and (whole[..., V:] == 7.0).all()
    assert logits.close(whole[..., :V], logits.want_of(s), torch.float32)
