"""Logits out (no probabilities): z / T is one division, rounded once, and once more to the output's type, so the results are those of the
host's division bit by bit; where the temperature is 0 or less, z itself."""
import math

import pytest
import torch

from paper_2409_04992_b200 import binding

pytestmark = pytest.mark.gpu
TEMPERATURES = [0.7, 1.0, 1.3, 3.0, 1e-3, 1e-12, 1e-38, 3e-39, 1e-40, 1e-45, 1e30, 0.0, -1.0]


@pytest.mark.parametrize("V", [1000, 1001, 50257, 131072])
@pytest.mark.parametrize("kinds", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float16, torch.bfloat16)])
def test_quotients_are_rounded_once(V, kinds):
    g = torch.Generator(device="cuda").manual_seed(V)
    hot = torch.tensor(TEMPERATURES)
    z = (4 * torch.randn(len(hot), 2, V, generator=g, device="cuda")).to(kinds[0])
    z[:, :, ::7] = 0.0
    z[:, 1, 3] = -math.inf
    allowed = torch.randint(-2 ** 31, 2 ** 31, (len(hot), 2, (V + 31) // 32), generator=g, device="cuda").int()
    out = torch.full(z.shape, 7.0, dtype=kinds[1], device="cuda")
    binding.process_logits(out, z, allowed=allowed, temperatures=hot.cuda(), probabilities=False)
    which = torch.arange(V)
    left = (allowed.cpu()[:, :, which // 32] >> (which % 32)) & 1 != 0
    t = hot[:, None, None]
    want = torch.where(t > 0, z.float().cpu() / torch.where(t > 0, t, 1.0), z.float().cpu())
    assert torch.equal(out.cpu(), want.masked_fill(~left, -math.inf).to(kinds[1]))
