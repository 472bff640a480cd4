"""bof4_cross_entropy where losses are small and where logits are infinite, in the form for few tokens and in the one for many: against the formula in 64 bits."""
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


def with_infinite_weight(bof4, tokens, rows, row, kind):  # noqa: F811
    """Logits are v * x0 but for row `row`, whose weight for x0 is infinite: an outlier, or (kind "constant") a row of level one with that constant.
    A third of the tokens have x0 = 1 (logit inf), a third x0 = -1 (-inf), a third 0 (NaN).  -> arguments, keywords, logits in 64 bits"""
    v = ((torch.arange(rows) % 13) - 6.0).bfloat16().float()
    x = torch.zeros(tokens, 64, dtype=torch.bfloat16, device="cuda")
    sign = torch.tensor([1.0, -1.0, 0.0], device="cuda").repeat(tokens)[:tokens]
    z = sign.double()[:, None] * v.double().cuda()[None, :]
    if kind == "outlier":
        lv, codes, scales = ramp(rows, v)
        x[:, 0] = sign.bfloat16()
        lst = (torch.tensor([row * 64], dtype=torch.int32, device="cuda"), torch.tensor([math.inf], dtype=torch.bfloat16, device="cuda"), torch.tensor([1], device="cuda"))
    else:
        v[row] = math.inf
        lv, codes, scales = ramp(rows, v)
        codes = codes.clone().view(rows, 32)
        codes[row] = 0xff
        codes = codes.view(-1)
        x[:] = sign.bfloat16()[:, None]
        lst = None
    z[:, row] = sign.double() * math.inf
    return (codes, scales, rows, 64, 64, lv, x), dict(outliers=lst), z


@pytest.mark.parametrize("tokens,rows", [(5, 300), (40, 300), (7, 20000), (40, 20000), (600, 300), (600, 40000)])
@pytest.mark.parametrize("kind", ["outlier", "constant"])
def test_infinite_logits(bof4, tokens, rows, kind):  # noqa: F811
    """A logit of +inf or NaN leaves nothing of its token finite, the target's own as little as another's; one of -inf has no part in the sums."""
    row = rows - 9
    args, kw, z = with_infinite_weight(bof4, tokens, rows, row, kind)
    for target in (row, 4):
        targets = torch.full((tokens,), target, device="cuda")
        loss, lse, _ = plain(z, targets)
        for grad in (True, False):
            got, got_lse, dx, status = bof4.bof4_cross_entropy(*args, targets, want_dx=grad, **kw)
            assert int(status.item()) == 0
            assert not bool(got[0::3].isfinite().any()) and not bool(got[2::3].isfinite().any())
            assert not bool(got_lse[0::3].isfinite().any()) and not bool(got_lse[2::3].isfinite().any())
            assert bool(((got_lse[1::3].double() - lse[1::3]).abs() <= TOL * (1 + lse[1::3].abs())).all())
            if target == row:
                assert bool((got[1::3] == math.inf).all())
            else:
                assert bool(((got[1::3].double() - loss[1::3]).abs() <= 2 * TOL * (1 + loss[1::3])).all())
            if grad:
                assert not bool(dx[0::3].isfinite().any()) and not bool(dx[2::3].isfinite().any())
                if kind == "outlier":  # (other columns have no weights but zeros)
                    assert not bool(dx[1::3, 0].isfinite().any()) and not bool(dx[1::3, 1:].any())


@pytest.mark.parametrize("tokens,rows", [(5, 300), (40, 300), (130, 300), (7, 20000), (40, 20000), (600, 300), (600, 40000)])
@pytest.mark.parametrize("kind", ["outlier", "constant", "nan"])
def test_ignored_tokens_beside_weights_that_are_not_finite(bof4, tokens, rows, kind):  # noqa: F811
    """Loss 0 and dx 0 whatever the weights are."""
    args, kw, _ = with_infinite_weight(bof4, tokens, rows, rows // 2, "outlier" if kind == "outlier" else "constant")
    if kind == "nan":
        args[1][5] = float("nan")
    targets = torch.arange(tokens, device="cuda") % 200
    targets[::2], targets[-1] = -100, rows
    ignored = (targets < 0) | (targets >= rows)
    for dloss in (None, torch.linspace(-2, 3, tokens, device="cuda")):
        loss, _, dx, status = bof4.bof4_cross_entropy(*args, targets, dloss=dloss, want_dx=True, **kw)
        assert int(status.item()) == 2
        assert not bool(loss[ignored].any()) and not bool(dx[ignored].any())


@pytest.mark.parametrize("tokens", [20, 130, 190])
def test_ignored_tokens_in_cut_tiles(bof4, tokens):  # noqa: F811
    """The same where the second product's tiles are cut along K (the vocabulary)."""
    args, kw, _ = with_infinite_weight(bof4, tokens, 30000, 29000, "constant")
    targets = torch.full((tokens,), -1, device="cuda")
    targets[5::7] = 3
    loss, _, dx, status = bof4.bof4_cross_entropy(*args, targets, want_dx=True, **kw)
    assert int(status.item()) == 0 and not bool(loss[targets < 0].any()) and not bool(dx[targets < 0].any())
