"""The calls that move rows and blocks, for latent caches, without a GPU: one head of the row's width, or refused.

As in test_abi.py, made-up device addresses are only handed over in a process that sees no CUDA device."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2409_04992_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000
fake_pointers = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: run in the GPU-less child instead")


@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU here: the test below runs in this process")
def test_it_passes_in_a_child_that_sees_no_gpu():
    done = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-p", "no:cacheprovider"],
                          cwd=ROOT, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""), capture_output=True, text=True, timeout=600)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-2000:]
    assert " passed" in done.stdout


@fake_pointers
def test_one_head_of_the_rows_width_is_taken():
    build.build()
    lib = binding.load()
    pools = (ctypes.c_void_p * 1)(FAKE)
    keep = lambda heads, dim: lib.instinfer_kv_keep_path(pools, pools, 1, FAKE, FAKE, None, FAKE, 2 * FAKE, None, 0, 0, 0, 0, 8,  # noqa: E731
                                                         heads, dim, 64, None, None)
    resize = lambda heads, dim: lib.instinfer_kv_resize(pools, pools, 1, FAKE, FAKE, FAKE, FAKE, FAKE, 4, 16, 9, 0, heads, dim, FAKE,  # noqa: E731
                                                        1 << 20, None, None)
    tidy = lambda heads, dim: lib.instinfer_kv_defragment(pools, pools, 1, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 4, 16, 9, 0, heads, dim,  # noqa: E731
                                                          FAKE, 1 << 20, None, None)
    for call in (keep, resize, tidy):
        assert call(1, 576) == call(9, 64) == binding.OK
        assert call(2, 576) == call(1, 512) == call(1, 320) == call(1, 560) == binding.ERR_UNSUPPORTED
        assert call(0, 576) == binding.ERR_INVALID_ARG


@fake_pointers
def test_a_cache_at_two_places_of_the_lists_is_refused():
    build.build()
    lib = binding.load()

    def keep(k, v):
        lists = [(ctypes.c_void_p * len(x))(*(FAKE * i for i in x)) for x in (k, v)]
        return lib.instinfer_kv_keep_path(*lists, len(k), FAKE, FAKE, None, FAKE, 2 * FAKE, None, 0, 0, 0, 1 << 24, 8, 1, 576, 64, None, None)

    for k, v in (([1, 1], [2, 3]), ([1, 2], [3, 3]), ([1, 2], [2, 3]), ([1, 2], [3, 1]), ([1, 2, 3], [4, 5, 1])):
        assert keep(k, v) == binding.ERR_INVALID_ARG, (k, v)
