"""Rotary appends, the latent cache and logits without a GPU: what the entry points refuse before anything is enqueued, the
sizes they report, the rotary frequencies, and that the binding's signatures and limits are the header's.

As in test_abi.py, made-up device addresses are only handed over in a process that sees no CUDA device."""
import ctypes
import math
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_2409_04992_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000
E = binding
NEW = ["instinfer_rope_frequencies", "instinfer_rope_append", "instinfer_latent_append", "instinfer_decode_attention_latent",
       "instinfer_latent_workspace_bytes", "instinfer_process_logits"]

fake_pointers = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: run in the GPU-less child instead")


@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU here: the tests below run in this process")
def test_refusals_pass_in_a_child_that_sees_no_gpu():
    done = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-p", "no:cacheprovider"],
                          cwd=ROOT, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""), capture_output=True, text=True, timeout=600)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-2000:]
    assert " passed" in done.stdout


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "instinfer.h")).read(), flags=re.S)


def parameters(name):
    found = re.search(r"(\w+)\s+%s\s*\((.*?)\);" % name, header(), flags=re.S)
    return found.group(1), [" ".join(p.split()) for p in found.group(2).split(",")]


def test_the_binding_has_the_headers_signatures(lib):
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "double": ctypes.c_double, "size_t": ctypes.c_size_t}
    for name in NEW:
        result, given = parameters(name)
        assert getattr(lib, name).argtypes == [ctypes.c_void_p if "*" in p else kinds[p.split()[0]] for p in given], name
        assert getattr(lib, name).restype == (ctypes.c_size_t if result == "size_t" else ctypes.c_int), name


def test_limits_are_the_headers():
    text = open(os.path.join(ROOT, "include", "instinfer.h")).read()
    value = lambda name: int(re.search(r"#define\s+INSTINFER_%s\s+(\d+)" % name, text).group(1))  # noqa: E731
    for name in ("MAX_LATENT_ROWS", "MAX_VOCAB", "MAX_BIAS", "FLAG_TOKEN_RANGE"):
        assert getattr(E, name) == value(name)
    assert E.ROPE_SCALINGS == {"plain": value("ROPE_PLAIN"), "linear": value("ROPE_LINEAR"), "by_parts": value("ROPE_BY_PARTS")}
    assert {str(t): n for t, n in E._TYPES.items()} == {"torch.float32": value("F32"), "torch.float16": value("F16"), "torch.bfloat16": value("BF16")}


ROPE = dict(q_out=FAKE, k_cache=FAKE, v_cache=FAKE, q=FAKE, k_new=FAKE, v_new=FAKE, type=1, q_stride=512, k_stride=256, v_stride=256,
            frequencies=FAKE, rope_dim=128, interleaved=0, magnitude=1.0, positions=None, seq_lens=FAKE, new_lens=None, block_table=FAKE,
            max_blocks_per_seq=8, block_tokens=16, num_phys_blocks=100, batch=2, max_new=3, q_heads=4, kv_heads=2, head_dim=128, s_max=0,
            status_flags=None, cuda_stream=None)
LATENT_APPEND = dict(q_out=FAKE, cache=FAKE, q_rope=FAKE, latent_new=FAKE, rope_new=FAKE, type=2, q_stride=4 * 192, q_head_stride=192,
                     latent_stride=576, rope_stride=576, frequencies=FAKE, interleaved=0, magnitude=1.0, positions=None, seq_lens=FAKE,
                     new_lens=None, block_table=FAKE, max_blocks_per_seq=8, block_tokens=16, num_phys_blocks=100, batch=2, max_new=3,
                     q_heads=4, latent_dim=512, rope_dim=64, s_max=0, status_flags=None, cuda_stream=None)
LATENT = dict(out=FAKE, lse=None, q=FAKE, cache=FAKE, block_table=FAKE, seq_lens=FAKE, tree_lens=None, tree_mask=None, type=1, batch=2,
              q_tokens=1, q_heads=16, latent_dim=512, rope_dim=64, s_max=0, block_tokens=16, max_blocks_per_seq=8, num_phys_blocks=100,
              max_seq_len=128, scale=0.1, workspace=FAKE, workspace_bytes=1 << 40, status_flags=None, cuda_stream=None)
LOGITS = dict(out=FAKE, out_type=0, out_stride=1000, logits=FAKE, logits_type=2, row_stride=1000, tokens=FAKE, token_lens=None,
              prompt_lens=None, max_tokens=10, penalties=FAKE, draft_tokens=None, tree_mask=None, tree_lens=None, bias_tokens=FAKE,
              bias_values=FAKE, max_bias=4, allowed=None, temperatures=None, probabilities=1, batch=2, tree_tokens=1, vocab=1000,
              status_flags=None, cuda_stream=None)
CALLS = {"instinfer_rope_append": ROPE, "instinfer_latent_append": LATENT_APPEND, "instinfer_decode_attention_latent": LATENT,
         "instinfer_process_logits": LOGITS}


def call(lib, name, **changed):
    base = CALLS[name]
    given = [p.split()[-1].lstrip("*") for p in parameters(name)[1]]
    assert given == list(base)
    return getattr(lib, name)(*{**base, **changed}.values())


BAD = {
    "instinfer_rope_append": [
        (E.ERR_INVALID_ARG, [dict(q_heads=-1), dict(kv_heads=0), dict(head_dim=0), dict(rope_dim=0), dict(rope_dim=256), dict(batch=-1),
                             dict(max_new=-1), dict(magnitude=math.inf), dict(q_stride=511), dict(k_stride=255), dict(k_stride=260), dict(v_stride=128),
                             dict(block_tokens=0), dict(num_phys_blocks=0), dict(max_blocks_per_seq=0), dict(block_table=None), dict(q=None),
                             dict(q_out=None), dict(k_cache=None), dict(v_cache=FAKE + 8), dict(k_new=FAKE + 2), dict(v_new=None),
                             dict(frequencies=None), dict(seq_lens=None)]),
        (E.ERR_UNSUPPORTED, [dict(head_dim=96, rope_dim=64), dict(rope_dim=24), dict(type=3), dict(type=-1), dict(block_tokens=12)])],
    "instinfer_latent_append": [
        (E.ERR_INVALID_ARG, [dict(q_heads=-1), dict(latent_dim=0), dict(rope_dim=0), dict(batch=-1), dict(max_new=-1), dict(q_stride=3 * 192 + 56),
                             dict(q_head_stride=60), dict(latent_stride=504), dict(rope_stride=56), dict(rope_stride=575), dict(block_table=None),
                             dict(cache=None), dict(q_rope=None), dict(q_out=None), dict(latent_new=FAKE + 8), dict(rope_new=None), dict(frequencies=None),
                             dict(seq_lens=None), dict(magnitude=math.nan)]),
        (E.ERR_UNSUPPORTED, [dict(latent_dim=384), dict(latent_dim=256), dict(rope_dim=32), dict(type=0), dict(block_tokens=4)])],
    "instinfer_decode_attention_latent": [
        (E.ERR_INVALID_ARG, [dict(q_tokens=0), dict(q_heads=0), dict(latent_dim=0), dict(rope_dim=-1), dict(batch=-1), dict(max_seq_len=0),
                             dict(max_seq_len=129), dict(scale=math.inf), dict(block_tokens=0), dict(num_phys_blocks=0), dict(block_table=None),
                             dict(out=None), dict(q=FAKE + 8), dict(cache=None), dict(seq_lens=None), dict(tree_mask=FAKE + 8)]),
        (E.ERR_UNSUPPORTED, [dict(latent_dim=384), dict(latent_dim=256), dict(rope_dim=128), dict(type=0), dict(q_tokens=129), dict(q_heads=16385), dict(block_tokens=20),
                             dict(num_phys_blocks=1 << 28)]),
        (E.ERR_WORKSPACE, [dict(workspace=None), dict(workspace=FAKE + 8), dict(workspace_bytes=1000)])],
    "instinfer_process_logits": [
        (E.ERR_INVALID_ARG, [dict(batch=-1), dict(tree_tokens=0), dict(vocab=0), dict(max_tokens=-1), dict(max_bias=-1), dict(row_stride=999),
                             dict(out_stride=999), dict(out=None), dict(logits=FAKE + 2), dict(tokens=None), dict(bias_values=None), dict(tree_mask=FAKE + 8)]),
        (E.ERR_UNSUPPORTED, [dict(tree_tokens=129), dict(vocab=262145, row_stride=262145, out_stride=262145), dict(max_bias=257), dict(out_type=3),
                             dict(logits_type=-1)])],
}


@fake_pointers
@pytest.mark.parametrize("name", CALLS)
def test_refusals(lib, name):
    for status, changes in BAD[name]:
        for changed in changes:
            assert call(lib, name, **changed) == status, (name, changed)


@fake_pointers
@pytest.mark.parametrize("name", CALLS)
def test_empty_calls(lib, name):
    assert call(lib, name, batch=0) == E.OK
    if "append" in name:
        assert call(lib, name, max_new=0) == E.OK


def test_workspace_sizes(lib):
    for batch, tokens, heads, length in ((1, 1, 1, 1), (64, 1, 16, 16384), (32, 1, 128, 8192), (7, 8, 16, 30000), (300, 1, 5, 100)):
        for latent in (512,):
            need = E.latent_workspace_bytes(batch, tokens, heads, latent, 64, length)
            assert need > 0 and need % 256 == 0
            # two partial results per block (or pair) at most, for a GPU of up to 160 SMs, and a few bytes per item
            assert need <= 2 * 160 * min(128, tokens * heads) * (latent + 1) * 4 + batch * tokens * heads * 8 + 1024
    assert E.latent_workspace_bytes(1, 1, 1, 512, 32, 100) == 0 and E.latent_workspace_bytes(1, 129, 1, 512, 64, 100) == 0
    assert E.latent_workspace_bytes(0, 1, 16, 512, 64, 100) == 256


@pytest.mark.parametrize("dim", [2, 16, 64, 128])
def test_frequencies(lib, dim):
    plain = [10000.0 ** (-2 * i / dim) for i in range(dim // 2)]
    f, m = E.rope_frequencies(dim, device="cpu")
    assert m == 1.0 and f.dtype == torch.float64 and torch.allclose(f, torch.tensor(plain, dtype=torch.float64), rtol=1e-14)
    f, m = E.rope_frequencies(dim, base=500000.0, scaling="linear", factor=4, device="cpu")
    assert m == 1.0 and torch.allclose(f, torch.tensor([500000.0 ** (-2 * i / dim) / 4 for i in range(dim // 2)], dtype=torch.float64), rtol=1e-14)
    f, m = E.rope_frequencies(dim, scaling="by_parts", factor=8, trained_len=4096, slow_turns=1, fast_turns=32, device="cpu")
    for got, p in zip(f.tolist(), plain):
        turns = 4096 * p / (2 * math.pi)
        share = min(1.0, max(0.0, (turns - 1) / 31))
        assert math.isclose(got, share * p + (1 - share) * p / 8, rel_tol=1e-13)
    assert math.isclose(m, 0.1 * math.log(8) + 1, rel_tol=2 ** -23)


def test_frequencies_refused(lib):
    for bad in (dict(rope_dim=3), dict(rope_dim=0), dict(rope_dim=64, base=0.0), dict(rope_dim=64, base=math.inf),
                dict(rope_dim=64, scaling="linear", factor=0.5), dict(rope_dim=64, scaling="by_parts", factor=2, trained_len=0),
                dict(rope_dim=64, scaling="by_parts", factor=2, trained_len=100, slow_turns=4, fast_turns=4),
                dict(rope_dim=64, scaling="by_parts", factor=math.nan, trained_len=100)):
        with pytest.raises(E.InstInferError) as error:
            E.rope_frequencies(device="cpu", **bad)
        assert error.value.status == E.ERR_INVALID_ARG
    with pytest.raises(E.InstInferError) as error:
        E.rope_frequencies(64, scaling="other", device="cpu")
    assert error.value.status == E.ERR_UNSUPPORTED
