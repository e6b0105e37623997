"""Probabilities at small temperatures, of huge logits and of masks of the type's lowest value, against the definition in 64 bits.

Tolerance: with x = (z - max z) / T log2 e, z - max z is rounded once, the rate log2 e / T twice and their product once, so x is off by
4 * 2^-24 of itself and the exponential by ln 2 times that, and by 2^-21 of its own; a sum of at most 2^18 terms goes through fewer than
96 additions a term, 2^-24 each.  Where x is above -30 that stays below 2^-16, the bound of the other tests of these calls."""
import math

import pytest
import torch

from paper_2409_04992_b200 import binding

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TEMPERATURES = [0.1, 0.05, 1e-2, 1e-3, 1e-4, 1e-6, 1e-8, 1e-9, 1e-10, 1e-12, 1e-30, 1e-38, 1e-45]
VOCABS = [1000, 16384, 50257, 131072, 262144]          # one block a row, several, eight, rows that start between boundaries


def check(out, z, hot):
    z, t = z.double().cpu(), hot.double().cpu()[:, None, None]
    x = (z - z.amax(-1, keepdim=True)) / t
    want = torch.softmax(x, -1)
    error, x = (out.double().cpu() - want).abs(), (x * math.log2(math.e)).clamp(min=-200)
    relative = 96 * 2.0 ** -24 + 2.0 ** -21 - x * math.log(2) * 2.0 ** -22
    assert bool((relative[x > -30] < 2.0 ** -16).all())
    floor = 2.0 ** -25 if out.dtype == torch.float16 else 2.0 ** -126
    assert bool((error <= (HALF[out.dtype] + relative) * want + floor).all()), float((error / want.clamp(min=1e-30)).max())


def rivals(B, V, dtype, size, hot, seed):
    """Logits of about `size` whose largest have close rivals, some in other parts of the row, some equal to the largest."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(B, 1, V, generator=g, device="cuda") * size / 10
    top = (size * (1 + 0.01 * torch.arange(B, device="cuda")))[:, None]
    places = torch.linspace(0, V - 1, 16, device="cuda").long()
    near = top - hot[:, None].clamp(max=1.0) * torch.arange(16, device="cuda") * 0.75
    near[:, 9] = top[:, 0]
    z[:, 0, places] = near
    return z.to(dtype)


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("size", [30.0, 1e4])
def test_small_temperatures(V, size):
    hot = torch.tensor(TEMPERATURES, device="cuda")
    z = rivals(len(hot), V, torch.float32, size, hot, V)
    out = torch.full_like(z, 7.0)
    binding.process_logits(out, z, temperatures=hot)
    check(out, z, hot)


@pytest.mark.parametrize("kinds", [(torch.bfloat16, torch.float32), (torch.float16, torch.bfloat16), (torch.bfloat16, torch.float16)])
@pytest.mark.parametrize("V", [1000, 50257])
def test_small_temperatures_of_16_bit_logits(kinds, V):
    hot = torch.tensor(TEMPERATURES * 40, device="cuda")          # more rows than clusters: runs of rows
    z = rivals(len(hot), V, kinds[0], 8.0, hot, 3)
    out = torch.zeros(z.shape, dtype=kinds[1], device="cuda")
    binding.process_logits(out, z, temperatures=hot)
    check(out, z, hot)


@pytest.mark.parametrize("V", [1000, 131072])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_lowest_and_largest_values(V, dtype):
    """Masked by the type's lowest value: one token left, nothing but masked ones (all alike), and the largest value beside the lowest."""
    lowest, largest = torch.finfo(dtype).min, torch.finfo(dtype).max
    z = torch.full((4, 1, V), lowest, device="cuda", dtype=dtype)
    z[0, 0, V // 2] = 1.0
    z[2, 0, :: 2] = largest
    z[3, 0, V - 1] = -math.inf
    for t in (1.0, 1e-3, 1e3):
        hot = torch.full((4,), t, device="cuda")
        out = torch.full((4, 1, V), 7.0, device="cuda")
        binding.process_logits(out, z, temperatures=hot)
        check(out, z, hot)
