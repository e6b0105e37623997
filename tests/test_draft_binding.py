"""What the binding of the speculative-decoding calls lets through to the library, without a GPU: the devices
of CPU tensors are made up, and the library is a stub that notes it was called.  Every tensor of every call,
the optional ones and all layers' too, has to be on the current device."""
import types

import pytest
import torch

from paper_2409_04992_b200 import binding

B, T, V, HQ, HKV, D, M, P, PAGE, LAYERS = 3, 8, 50, 4, 2, 64, 5, 20, 16, 3
STREAM = types.SimpleNamespace(cuda_stream=1)


class Stub:
    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        def call(*args):
            self.called.append(name)
            return 0 if name != "instinfer_status_string" else b"refused"
        return call


@pytest.fixture
def lib(monkeypatch):
    """The stub; tensors are on device 0 except those in lib.elsewhere."""
    stub = Stub()
    stub.elsewhere = set()
    monkeypatch.setattr(binding, "load", lambda: stub)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1 if id(t) in stub.elsewhere else 0)
    return stub


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def halves(*shape):
    return torch.zeros(*shape, dtype=torch.float16)


def pools():
    return [halves(P, HKV, PAGE, D) for _ in range(LAYERS)]


def flags():
    return ints(1)


CALLS = {
    "tree_mask": lambda: dict(mask=torch.zeros(B, T, 1, dtype=torch.int64), parents=ints(B, T), tree_lens=ints(B), status_flags=flags()),
    "decode_attention_tree": lambda: dict(
        out=halves(B, T, HQ, D), lse=torch.zeros(B, T, HQ), q=halves(B, T, HQ, D), k_cache=halves(P, HKV, PAGE, D),
        v_cache=halves(P, HKV, PAGE, D), block_table=ints(B, M), seq_lens=ints(B), tree_lens=ints(B),
        mask=torch.zeros(B, T, 1, dtype=torch.int64), max_seq_len=M * PAGE, scale=0.1, workspace=torch.zeros(1000, dtype=torch.uint8),
        status_flags=flags()),
    "verify_tree": lambda: dict(
        path=ints(B, T), path_lens=ints(B), out_tokens=ints(B, T), target_probs=torch.zeros(B, T, V), draft_probs=torch.zeros(B, T, V),
        tokens=ints(B, T), parents=ints(B, T), tree_lens=ints(B), uniforms=torch.zeros(B, T), status_flags=flags()),
    "kv_keep_path": lambda: dict(
        k_caches=pools(), v_caches=pools(), path=ints(B, T), path_lens=ints(B), tree_lens=ints(B), seq_lens=ints(B), new_lens=ints(B),
        block_table=ints(B, M), status_flags=flags()),
    "kv_fork": lambda: dict(block_table=ints(B, M), block_refs=ints(P), seq_lens=ints(B), src=ints(2), dst=ints(2), block_tokens=PAGE,
                            status_flags=flags()),
    "kv_resize": lambda: dict(
        k_pools=pools(), v_pools=pools(), block_table=ints(B, M), block_refs=ints(P), seq_lens=ints(B), want_lens=ints(B),
        new_lens=ints(B), workspace=torch.zeros(1000, dtype=torch.uint8), status_flags=flags()),
    "kv_defragment": lambda: dict(
        k_pools=pools(), v_pools=pools(), block_table=ints(B, M), block_refs=ints(P), seq_lens=ints(B), new_block_table=ints(B, M),
        new_block_refs=ints(P), blocks_used=ints(1), workspace=torch.zeros(1000, dtype=torch.uint8), status_flags=flags()),
}
TENSORS = [(call, name) for call, make in CALLS.items() for name, value in make().items() if isinstance(value, torch.Tensor)]
LAYERED = [(call, name) for call, make in CALLS.items() for name, value in make().items() if isinstance(value, list)]


def refused(lib, call, args):
    lib.called.clear()
    with pytest.raises(binding.InstInferError) as error:
        getattr(binding, call)(**args, stream=STREAM)
    assert error.value.status == binding.ERR_INVALID_ARG
    assert "instinfer_" + call not in lib.called


@pytest.mark.parametrize("call", CALLS)
def test_good_arguments_pass(lib, call):
    getattr(binding, call)(**CALLS[call](), stream=STREAM)
    assert lib.called == ["instinfer_" + call]
    args = {name: value for name, value in CALLS[call]().items()
            if name not in ("lse", "tree_lens", "draft_probs", "status_flags")}
    if call in ("decode_attention_tree", "kv_keep_path"):
        args["block_table"] = None
        for name in ("k_cache", "v_cache", "k_caches", "v_caches"):
            if name in args:
                args[name] = halves(B, HKV, 100, D) if name.endswith("cache") else [halves(B, HKV, 100, D) for _ in range(LAYERS)]
    for name in ("lse", "tree_lens", "draft_probs"):
        if name in CALLS[call]():
            args[name] = None
    getattr(binding, call)(**args, stream=STREAM)


@pytest.mark.parametrize("call,name", TENSORS)
def test_a_tensor_of_another_device_is_refused(lib, call, name):
    args = CALLS[call]()
    lib.elsewhere.add(id(args[name]))
    refused(lib, call, args)


@pytest.mark.parametrize("call,name", LAYERED)
@pytest.mark.parametrize("layer", range(LAYERS))
def test_a_layer_of_another_device_is_refused(lib, call, name, layer):
    args = CALLS[call]()
    lib.elsewhere.add(id(args[name][layer]))
    refused(lib, call, args)


@pytest.mark.parametrize("call,name", LAYERED)
@pytest.mark.parametrize("layer", range(LAYERS))
def test_a_layer_of_another_type_or_size_is_refused(lib, call, name, layer):
    for bad in (torch.zeros(P, HKV, PAGE, D), torch.zeros(P, HKV, PAGE, D, dtype=torch.int64), halves(P - 1, HKV, PAGE, D),
                halves(P, HKV, D, PAGE).transpose(2, 3)):
        args = CALLS[call]()
        args[name][layer] = bad
        refused(lib, call, args)


@pytest.mark.parametrize("call,name", LAYERED)
def test_pools_of_another_type_or_number_are_refused(lib, call, name):
    other = name.replace("k_", "v_") if name.startswith("k_") else name.replace("v_", "k_")
    args = CALLS[call]()
    args[name] = args[name][1:]
    refused(lib, call, args)
    args = CALLS[call]()
    args[name], args[other] = ([x.float() for x in args[n]] for n in (name, other))
    refused(lib, call, args)
    args = CALLS[call]()
    args[name] = [halves(P, PAGE, HKV, D) for _ in range(LAYERS)]        # as many elements, another layout
    refused(lib, call, args)


def test_what_belongs_together_has_to_fit(lib):
    for call in ("kv_resize", "kv_defragment"):
        refused(lib, call, dict(CALLS[call](), block_refs=ints(P - 1)))
    refused(lib, "kv_defragment", dict(CALLS["kv_defragment"](), new_block_refs=ints(P - 1)))
    for shape in ((B - 1, M), (B, M - 1), (B, M + 1)):
        refused(lib, "kv_defragment", dict(CALLS["kv_defragment"](), new_block_table=ints(*shape)))
    for src, dst in ((2, 1), (1, 2)):
        refused(lib, "kv_fork", dict(CALLS["kv_fork"](), src=ints(src), dst=ints(dst)))
    refused(lib, "decode_attention_tree", dict(CALLS["decode_attention_tree"](), v_cache=halves(P, PAGE, HKV, D)))
    refused(lib, "decode_attention_tree", dict(CALLS["decode_attention_tree"](), v_cache=halves(P - 1, HKV, PAGE, D)))
    # caches, tables and masks of fewer sequences than the call's, of other heads, or of fewer nodes
    tree, keep = CALLS["decode_attention_tree"], CALLS["kv_keep_path"]
    refused(lib, "decode_attention_tree", dict(tree(), block_table=ints(B - 1, M)))
    refused(lib, "decode_attention_tree", dict(tree(), block_table=None, k_cache=halves(B - 1, HKV, 100, D), v_cache=halves(B - 1, HKV, 100, D)))
    refused(lib, "decode_attention_tree", dict(tree(), k_cache=halves(P, HKV, PAGE, 2 * D), v_cache=halves(P, HKV, PAGE, 2 * D)))
    refused(lib, "decode_attention_tree", dict(tree(), mask=torch.zeros(B - 1, T, 1, dtype=torch.int64)))
    wide = dict(tree(), q=halves(B, 65, HQ, D), out=halves(B, 65, HQ, D), lse=torch.zeros(B, 65, HQ))
    refused(lib, "decode_attention_tree", dict(wide, mask=torch.zeros(B, 65, 1, dtype=torch.int64)))
    refused(lib, "kv_keep_path", dict(keep(), block_table=ints(B - 1, M)))
    few = [halves(B - 1, HKV, 100, D) for _ in range(LAYERS)]
    refused(lib, "kv_keep_path", dict(keep(), block_table=None, k_caches=few, v_caches=few))


def test_buffers_may_be_larger_and_rows_further_apart(lib):
    binding.decode_attention_tree(**dict(CALLS["decode_attention_tree"](), seq_lens=ints(B + 5), status_flags=ints(4)), stream=STREAM)
    binding.kv_resize(**dict(CALLS["kv_resize"](), seq_lens=ints(B + 1), new_lens=ints(B + 3), block_refs=ints(P + 1)), stream=STREAM)
    wide = [torch.zeros(B, T, V + 3)[:, :, :V] for _ in range(2)]
    binding.verify_tree(**dict(CALLS["verify_tree"](), target_probs=wide[0], draft_probs=wide[1]), stream=STREAM)
