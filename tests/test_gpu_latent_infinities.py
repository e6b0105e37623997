"""Attention over a latent cache: rows that see a value which is not finite, by the sign of what it makes of their logits.  Tolerances as in
test_gpu_latent_attention.py, with the values that count."""
import math

import pytest
import torch

from tests.test_gpu_latent_attention import Case
from tests.test_gpu_rope_append import HALF_STEP

pytestmark = pytest.mark.gpu
T = 48


def expected(case, b, left_out):
    """Sequence b without the position left_out: outputs, log-sum-exps and the bounds of both, [tokens, heads, ..]."""
    n, N = case.lens[b], case.N
    keep = torch.arange(n, device="cuda") != left_out
    c, q = case.rows(b).double()[keep], case.q[b].double()
    position, j = torch.arange(n, device="cuda")[keep], torch.arange(N, device="cuda")
    sees = position[None, :] <= n - N + j[:, None]
    z = (torch.einsum("nhd,ld->nhl", q, c) * case.scale).masked_fill(~sees[:, None], -math.inf)
    want = torch.softmax(z, -1) @ c[:, :case.L]
    delta = 40 * 2.0 ** -23 * abs(case.scale) * float(torch.einsum("nhd,ld->nhl", q.abs(), c.abs()).max())
    bound = HALF_STEP[case.dtype] * want.abs() + 2 * delta * float(c.abs().max()) + 2.0 ** -25
    lse = torch.logsumexp(z, -1)
    return want, bound, lse, delta + 2.0 ** -20 * (1 + float(z[sees[:, None].expand_as(z)].abs().max()))


@pytest.mark.parametrize("H", [4, 40, 128])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dim", [3, 300, 540])               # in the vector's two halves and in the turned part
@pytest.mark.parametrize("new", [True, False])
def test_rows_by_the_sign_of_their_logit(H, dtype, value, dim, new):
    case = Case([70, 200, 129], 4, H, T=T, dtype=dtype, seed=dim)
    clean = [x.clone() for x in case.run()]
    b, n = 1, 200
    at = n - 3 if new else 77                                # (a new token that the first one does not see, or one before them)
    case.cache[int(case.table[b, at // T]), at % T, dim] = value
    out, lse = case.run()
    torch.cuda.synchronize()
    for other in (0, 2):
        assert torch.equal(out[other], clean[0][other]) and torch.equal(lse[other], clean[1][other])
    want, bound, want_lse, lse_bound = expected(case, b, at)
    sign = torch.sign(case.q[b, :, :, dim].double() * value * case.scale)
    for t in range(4):
        for h in range(H):
            if new and t == 0:
                assert torch.equal(out[b, t, h], clean[0][b, t, h]) and torch.equal(lse[b, t, h], clean[1][b, t, h])
            elif sign[t, h] == -1:                           # its logit is -infinity: it counts nothing
                counts = torch.ones(512, dtype=torch.bool, device="cuda")
                if not new and dim < 512:
                    counts[dim] = False                      # (0 times an infinity: NaN, or the others' value)
                    got, ref = out[b, t, h, dim].double(), want[t, h, dim]
                    assert bool(got.isnan()) or abs(float(got - ref)) <= float(bound[t, h, dim])
                assert bool(((out[b, t, h].double() - want[t, h]).abs() <= bound[t, h])[counts].all()), (t, h)
                assert abs(float(lse[b, t, h].double() - want_lse[t, h])) <= lse_bound
            else:                                            # +infinity, or NaN (an infinity times 0 too)
                assert out[b, t, h].isnan().all() and lse[b, t, h].isnan(), (t, h)


@pytest.mark.parametrize("H", [4, 128])
def test_nothing_but_left_out_tokens_is_an_empty_row(H):
    case = Case([3, 2], 2, H, T=T)
    case.q[0, 1, :, 7] = case.q[0, 1, :, 7].abs() + 0.1
    case.cache[int(case.table[0, 0]), 1:3, 7] = -math.inf    # the new tokens of sequence 0
    case.cache[int(case.table[0, 0]), 0, 530] = -math.inf    # the token before them, in the turned part
    case.q[0, 1, :, 530] = 1.0
    out, lse = case.run()
    assert (out[0, 1] == 0).all() and (lse[0, 1] == -math.inf).all()
    assert out[1].isfinite().all()
