"""What the binding of the rotary appends, the latent cache and the logits lets through to the library, without a GPU: the
devices of CPU tensors are made up, and the library is a stub that notes it was called."""
import types

import pytest
import torch

from paper_2409_04992_b200 import binding

B, N, V, HQ, H, D, M, P, T = 3, 2, 50, 4, 2, 64, 5, 20, 16
STREAM = types.SimpleNamespace(cuda_stream=1)


class Stub:
    def __init__(self):
        self.called, self.args, self.elsewhere = [], None, set()

    def __getattr__(self, name):
        def call(*args):
            self.called.append(name)
            self.args = args
            return 0 if name != "instinfer_status_string" else b"refused"
        return call


@pytest.fixture
def lib(monkeypatch):
    stub = Stub()
    monkeypatch.setattr(binding, "load", lambda: stub)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1 if id(t) in stub.elsewhere else 0)
    return stub


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def halves(*shape):
    return torch.zeros(*shape, dtype=torch.float16)


def doubles(n):
    return torch.zeros(n, dtype=torch.float64)


CALLS = {
    "rope_append": lambda: dict(q_out=halves(B, N, HQ, D), k_cache=halves(P, H, T, D), v_cache=halves(P, H, T, D), q=halves(B, N, HQ, D),
                                k_new=halves(B, N, H, D), v_new=halves(B, N, H, D), frequencies=doubles(D // 2), seq_lens=ints(B),
                                new_lens=ints(B), block_table=ints(B, M), positions=ints(B, N), status_flags=ints(1)),
    "latent_append": lambda: dict(q_out=halves(B, N, HQ, 576), cache=halves(P, T, 576), q_rope=halves(B, N, HQ, 64), latent_new=halves(B, N, 512),
                                  rope_new=halves(B, N, 64), frequencies=doubles(32), seq_lens=ints(B), new_lens=ints(B),
                                  block_table=ints(B, M), positions=ints(B, N), status_flags=ints(1)),
    "decode_attention_latent": lambda: dict(out=halves(B, N, HQ, 512), lse=torch.zeros(B, N, HQ), q=halves(B, N, HQ, 576), cache=halves(P, T, 576),
                                            block_table=ints(B, M), seq_lens=ints(B), tree_lens=ints(B),
                                            mask=torch.zeros(B, N, 1, dtype=torch.int64), max_seq_len=M * T, scale=0.1,
                                            workspace=torch.zeros(1000, dtype=torch.uint8), status_flags=ints(1)),
    "process_logits": lambda: dict(out=torch.zeros(B, N, V), logits=halves(B, N, V), tokens=ints(B, 7), token_lens=ints(B), prompt_lens=ints(B),
                                   penalties=torch.zeros(B, 3), draft_tokens=ints(B, N), mask=torch.zeros(B, N, 1, dtype=torch.int64),
                                   tree_lens=ints(B), bias_tokens=ints(B, 3), bias_values=torch.zeros(B, 3), allowed=ints(B, N, 2),
                                   temperatures=torch.zeros(B), status_flags=ints(1)),
}
TENSORS = [(call, name) for call, make in CALLS.items() for name, value in make().items() if isinstance(value, torch.Tensor)]
OPTIONAL = {"rope_append": ("new_lens", "positions", "status_flags"), "latent_append": ("new_lens", "positions", "status_flags"),
            "decode_attention_latent": ("lse", "tree_lens", "mask", "status_flags"),
            "process_logits": ("tokens", "token_lens", "prompt_lens", "penalties", "draft_tokens", "mask", "tree_lens", "bias_tokens",
                               "bias_values", "allowed", "temperatures", "status_flags")}


def refused(lib, call, args, status=binding.ERR_INVALID_ARG):
    lib.called.clear()
    with pytest.raises(binding.InstInferError) as error:
        getattr(binding, call)(**args, stream=STREAM)
    assert error.value.status == status
    assert "instinfer_" + call not in lib.called


@pytest.mark.parametrize("call", CALLS)
def test_good_arguments_pass(lib, call):
    getattr(binding, call)(**CALLS[call](), stream=STREAM)
    assert lib.called == ["instinfer_" + call]
    getattr(binding, call)(**{k: None if k in OPTIONAL[call] else v for k, v in CALLS[call]().items()}, stream=STREAM)
    assert lib.called == ["instinfer_" + call] * 2


@pytest.mark.parametrize("call,name", TENSORS)
def test_a_tensor_of_another_device_is_refused(lib, call, name):
    args = CALLS[call]()
    lib.elsewhere.add(id(args[name]))
    refused(lib, call, args)


@pytest.mark.parametrize("call,name", [(c, n) for c, n in TENSORS if n not in ("workspace", "status_flags", "logits", "out", "q", "k_new", "latent_new")
                                       or (c, n) == ("rope_append", "q")])
def test_a_tensor_of_another_type_is_refused(lib, call, name):
    args = CALLS[call]()
    args[name] = args[name].to(torch.int16)
    refused(lib, call, args)


@pytest.mark.parametrize("call,name", [("rope_append", "k_new"), ("latent_append", "latent_new"), ("decode_attention_latent", "q"),
                                       ("process_logits", "logits"), ("process_logits", "out")])
def test_types_that_no_kernel_takes_are_unsupported(lib, call, name):
    args = CALLS[call]()
    args[name] = args[name].double()
    refused(lib, call, args, binding.ERR_UNSUPPORTED)


@pytest.mark.parametrize("call,name", [("rope_append", n) for n in ("k_cache", "v_cache", "k_new", "v_new", "q", "q_out", "positions")] +
                         [("latent_append", n) for n in ("cache", "q_out", "q_rope", "rope_new", "positions")] +
                         [("decode_attention_latent", n) for n in ("cache", "lse")] + [("process_logits", "out")])
def test_a_tensor_of_another_shape_is_refused(lib, call, name):
    args = CALLS[call]()
    shape = list(args[name].shape)
    shape[-1] += 1
    args[name] = torch.zeros(*shape, dtype=args[name].dtype)
    refused(lib, call, args)


@pytest.mark.parametrize("call,name", [("rope_append", "seq_lens"), ("rope_append", "new_lens"), ("rope_append", "block_table"),
                                       ("latent_append", "block_table"), ("decode_attention_latent", "seq_lens"),
                                       ("decode_attention_latent", "block_table"), ("process_logits", "temperatures"), ("process_logits", "tokens"),
                                       ("process_logits", "allowed"), ("process_logits", "penalties")])
def test_too_few_sequences_are_refused(lib, call, name):
    args = CALLS[call]()
    args[name] = args[name][:B - 1]
    refused(lib, call, args)


def test_slices_of_a_projection_keep_their_strides(lib):
    whole = halves(B, N, HQ + 2 * H, D)
    q, k, v = whole.split([HQ, H, H], dim=2)
    args = dict(CALLS["rope_append"](), q=q, k_new=k, v_new=v)
    binding.rope_append(**args, stream=STREAM)
    assert lib.args[7:10] == ((HQ + 2 * H) * D,) * 3
    args = CALLS["rope_append"]()
    args["k_new"] = halves(B, N + 1, H, D)[:, :N]          # sequences further apart than their tokens
    refused(lib, "rope_append", args)
    args["k_new"] = halves(B, N, D, H).transpose(2, 3)
    refused(lib, "rope_append", args)
    padded = halves(B, N, 64)[..., :V]
    binding.process_logits(**dict(CALLS["process_logits"](), logits=padded), stream=STREAM)
    assert lib.args[5] == 64
    refused(lib, "process_logits", dict(CALLS["process_logits"](), logits=halves(B, N, 2 * V)[..., ::2]))


def test_queries_and_their_place_come_together(lib):
    for call, name in (("rope_append", "q"), ("rope_append", "q_out"), ("latent_append", "q_rope"), ("latent_append", "q_out")):
        refused(lib, call, dict(CALLS[call](), **{name: None}))
    binding.rope_append(**dict(CALLS["rope_append"](), q=None, q_out=None), stream=STREAM)
    binding.latent_append(**dict(CALLS["latent_append"](), q_rope=None, q_out=None), stream=STREAM)
