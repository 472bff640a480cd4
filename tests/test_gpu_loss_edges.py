"""bof4_cross_entropy where losses are small, in the form for few tokens and in the one for many: against the formula in 64 bits."""
import math

import pytest
import torch

from test_gpu_cross_entropy import TOL, bof4, ramp  # noqa: F401

pytestmark = pytest.mark.gpu


def plain(z, targets):
    """Loss, log-sum and the logarithm of the others' share over the target's, in 64 bits."""
    n, keep = torch.arange(len(z), device="cuda"), targets >= 0
    at = torch.where(keep, targets, 0)
    rest = z - z[n, at][:, None]
    rest[n, at] = -math.inf
    rest = torch.logsumexp(rest, 1)
    return torch.where(keep, torch.logaddexp(rest, torch.zeros_like(rest)), 0.0), torch.logsumexp(z, 1), rest


@pytest.mark.parametrize("tokens", [1, 20, 600])
@pytest.mark.parametrize("rows", [300, 40000])
@pytest.mark.parametrize("others,own", [(-23.0, -8.25), (-23.75, -4.0), (-20.0, 0.0), (-12.0, -2.0), (-23.5, -16.0), (-23.5, -22.0), (-3.0, 4.0), (0.5, 20.0)])
def test_losses_near_zero(bof4, tokens, rows, others, own):  # noqa: F811
    """All logits within 24 of zero and a target that stands out: log(1 + e^rest) as in the tests of references, without a term that does not scale with the loss
    (logits are exact, rest is above -40, no exponential is below 2^-126)."""
    v = others - 0.125 * (torch.arange(rows) % 3)
    top = rows * 2 // 3 + 1
    v[top] = own
    v = v.bfloat16().float()
    lv, codes, scales = ramp(rows, v)
    x = torch.zeros(tokens, 64, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = 1.0
    x[1::4, 0] = 0.5
    targets = torch.full((tokens,), top, device="cuda")
    targets[3::5] = 7
    targets[4::11] = -1
    loss, lse, rest = plain(x[:, :1].double() * v.double().cuda()[None, :], targets)
    for grad in (True, False):
        got, got_lse, _, status = bof4.bof4_cross_entropy(codes, scales, rows, 64, 64, lv, x, targets, want_dx=grad)
        assert int(status.item()) == 0 and bool((got >= 0).all())
        assert bool(((got_lse.double() - lse).abs() <= TOL * (1 + lse.abs())).all())
        off = (got.double() - loss).abs() / ((TOL + 2.0 ** -22 * rest.abs()) * torch.clamp(loss, max=1) + TOL * loss).clamp(min=1e-300)
        assert bool((off <= 1).all()), (float(off.max()), float(got[off.argmax()]), float(loss[off.argmax()]))
