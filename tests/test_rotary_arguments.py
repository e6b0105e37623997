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
