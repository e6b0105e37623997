"""Every tensor of the speculative-decoding calls left on the host in turn: refused before anything is enqueued."""
import pytest
import torch

from paper_2409_04992_b200 import binding
from tests.test_draft_binding import CALLS

pytestmark = pytest.mark.gpu


def moved(value):
    return [x.cuda() for x in value] if isinstance(value, list) else value.cuda() if isinstance(value, torch.Tensor) else value


@pytest.mark.parametrize("call", CALLS)
def test_a_tensor_of_the_host_is_refused(call, monkeypatch):
    on_gpu = {name: moved(value) for name, value in CALLS[call]().items()}
    before = {name: [x.clone() for x in value] if isinstance(value, list) else value.clone()
              for name, value in on_gpu.items() if not isinstance(value, (int, float))}
    reached = []

    class Nothing:                       # (should a call not be refused, it ends here and not on the GPU)
        def __getattr__(self, name):
            return (lambda *args: b"refused") if name == "instinfer_status_string" else (lambda *args: reached.append(name) or 0)
    monkeypatch.setattr(binding, "load", lambda: Nothing())
    for name, value in on_gpu.items():
        hosts = []
        if isinstance(value, list):
            hosts = [value[:i] + [value[i].cpu()] + value[i + 1:] for i in range(len(value))]
        elif isinstance(value, torch.Tensor):
            hosts = [value.cpu()]
        for host in hosts:
            with pytest.raises(binding.InstInferError) as error:
                getattr(binding, call)(**dict(on_gpu, **{name: host}))
            assert error.value.status == binding.ERR_INVALID_ARG
    assert reached == []
    getattr(binding, call)(**on_gpu)
    assert reached == ["instinfer_" + call]
    for name, value in before.items():
        now = on_gpu[name]
        assert all(torch.equal(x, y) for x, y in zip(value, now)) if isinstance(value, list) else torch.equal(value, now)
