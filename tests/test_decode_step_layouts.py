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
