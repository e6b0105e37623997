"""Tensors of the rotary appends, the latent cache and the logits whose layout is not the one that the kernels read, without a GPU (the
library is the stub of test_decode_step_binding.py): those that would be read wrongly or out of range are refused."""
import pytest
import torch

from paper_2409_04992_b200 import binding
from tests.test_decode_step_binding import B, CALLS, N, STREAM, lib, refused  # noqa: F401


@pytest.mark.parametrize("call", ["process_logits", "decode_attention_latent"])
def test_a_mask_whose_rows_are_not_one_after_the_other_is_refused(lib, call):  # noqa: F811
    words = torch.zeros(B, N, 2, dtype=torch.int64)
    refused(lib, call, dict(CALLS[call](), mask=words[..., :1]))                    # every other word: other nodes' bits would be read
    refused(lib, call, dict(CALLS[call](), mask=words[:1, :, :1].contiguous().expand(B, N, 1)))     # one tree for all: memory behind it would be
    getattr(binding, call)(**dict(CALLS[call](), mask=words[:1, :, :1].expand(B, N, 1).contiguous()), stream=STREAM)


@pytest.mark.parametrize("call,name,shape", [
    ("process_logits", "penalties", (B, 4)), ("process_logits", "draft_tokens", (B, N + 1)), ("process_logits", "allowed", (B, N, 3)),
    ("process_logits", "allowed", (B, N + 1, 2)), ("process_logits", "mask", (B, N, 2)), ("process_logits", "mask", (B, N + 1, 1)),
    ("process_logits", "temperatures", (B, 1)), ("process_logits", "tree_lens", (B, 2)), ("process_logits", "tokens", (B * 7,)),
    ("decode_attention_latent", "mask", (B, N, 2)), ("decode_attention_latent", "mask", (B, N + 1, 1))])
def test_rows_of_another_length_are_refused(lib, call, name, shape):  # noqa: F811
    args = CALLS[call]()
    refused(lib, call, dict(args, **{name: torch.zeros(shape, dtype=args[name].dtype)}))


def test_more_sequences_than_the_batch_has_are_taken(lib):  # noqa: F811
    for call, names in (("process_logits", ("penalties", "draft_tokens", "allowed", "mask", "temperatures", "tokens", "token_lens")),
                        ("decode_attention_latent", ("mask", "seq_lens"))):
        args = CALLS[call]()
        for name in names:
            args[name] = torch.zeros(B + 2, *args[name].shape[1:], dtype=args[name].dtype)
        getattr(binding, call)(**args, stream=STREAM)


def test_an_empty_history_and_no_biases_are_taken(lib):  # noqa: F811
    empty = dict(tokens=torch.zeros(B, 0, dtype=torch.int32), bias_tokens=torch.zeros(B, 0, dtype=torch.int32), bias_values=torch.zeros(B, 0))
    binding.process_logits(**dict(CALLS["process_logits"](), **empty), stream=STREAM)
    assert lib.args[9] == 0 and lib.args[16] == 0


@pytest.mark.parametrize("call", ["rope_append", "latent_append"])
@pytest.mark.parametrize("batch,tokens", [(B, 0), (0, N), (0, 0), (1, 0)])
def test_no_new_tokens_are_a_call_without_work(lib, call, batch, tokens):  # noqa: F811
    args = CALLS[call]()
    for name in ("q_out", "q", "k_new", "v_new", "q_rope", "latent_new", "rope_new", "positions"):
        if name in args:
            args[name] = torch.zeros(batch, tokens, *args[name].shape[2:], dtype=args[name].dtype)
    getattr(binding, call)(**args, stream=STREAM)
    assert lib.called == ["instinfer_" + call]
