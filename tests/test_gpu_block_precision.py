"""What the gated block and the vocabulary loss promise about precision: activations on values that are exact, and how much of a long sum in fp32 is lost at every
number of tokens.  A tensor core cuts a sum off at each step of 16 of K, a quarter of a unit of the running sum on average and always towards zero, so that n steps in one
accumulator cost about 2^-24 n / 4 of it: 3.8e-6 for K = 4096.  No accumulator of results in fp32 takes more than 64 steps (1024 of K): 0.95e-6; SUM has a third more, for the
roundings of their sums."""
import pytest
import torch

from test_gpu_cross_entropy import plain, targets_of
from test_gpu_gated import act64, act_code, bof4, decode, real_case  # noqa: F401

pytestmark = pytest.mark.gpu

TOKENS = [1, 12, 40, 64, 100, 128, 129, 200, 256, 257, 384, 600, 767, 768, 900]
SUM = 1.3e-6


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("tokens,cols", [(3, 64), (12, 256), (40, 256), (200, 4096), (900, 64)])
def test_activations_at_every_value(bof4, act, tokens, cols):  # noqa: F811
    """Tokens of zeros, a bias of every finite bf16 value for the gate and of one for the other half: h is the activation, within 2^-20 of max(|z|, 1).

    SILU: exp(-z) is off by (2 + 1.173 |z|) units of 2^-23, which moves z s(z) by |z| s (1 - s) of that, at most (0.5 + 0.33) |z| 2^-23; the quotient (2 units), the sum and two
    products another 3.5 |z| s 2^-23: below 2^-20.7 |z|.  The tanh form's argument has four roundings more, of half a unit each and of |v| s (1 - s) <= 0.28: 0.6 |z| 2^-23 more,
    2^-20.5 |z|.  The quotient is zero where its divisor is above 2^126 (v below -87): the result is below 2^-115 there."""
    bits = torch.arange(1 << 16, dtype=torch.int32)
    z = bits[(bits & 0x7F80) != 0x7F80].to(torch.int16).view(torch.bfloat16).float().cuda()
    ffn = z.numel()
    lv, codes, scales = real_case(2 * ffn, cols, 64, 1)
    x = torch.zeros(tokens, cols, dtype=torch.bfloat16, device="cuda")
    h, status = bof4.bof4_gated(codes, scales, ffn, cols, 64, lv, x, bias=torch.cat((z, torch.ones_like(z))), activation=act_code(bof4, act), out_dtype=bof4.F32)
    assert int(status.item()) == 0 and torch.equal(h[0].expand(tokens, ffn), h)
    want = act64(z.double(), act)[0]
    off = (h[0].double() - want).abs() / z.double().abs().clamp(min=1)
    assert bool((off <= 2.0 ** -20).all()), (float(off.max()), float(z[off.argmax()]))


@pytest.mark.parametrize("cols", [4096, 8192])
@pytest.mark.parametrize("tokens", TOKENS)
def test_long_sums_of_a_gated_block(bof4, tokens, cols):  # noqa: F811
    """h = g u in fp32: off by what both are."""
    ffn = 10240   # more tiles than SMs: most have their whole K in one part
    lv, codes, scales = real_case(2 * ffn, cols, 64, tokens)
    x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(tokens)).bfloat16().cuda()
    z = x.double() @ decode(codes, scales, 64, lv, 2 * ffn, cols).T
    want = z[:, :ffn] * z[:, ffn:]
    h, status = bof4.bof4_gated(codes, scales, ffn, cols, 64, lv, x, activation=bof4.ACT_NONE, out_dtype=bof4.F32)
    err = float((h.double() - want).norm() / want.norm())
    print("h by %d tokens, K = %d: %.2g" % (tokens, cols, err))
    assert int(status.item()) == 0 and err <= 2 * SUM


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("cols", [4096, 8192])
@pytest.mark.parametrize("tokens", TOKENS)
def test_long_sums_of_a_loss(bof4, tokens, cols, grad):  # noqa: F811
    """lse is off by the mean error of the logits, weighted by the probabilities, and the loss by the target's besides.  Each exponential is off by 2^-22 (1 + 0.6 d), d its argument
    (6 on such a mean), sums and logarithm by less: 2^-19 of one altogether."""
    rows = 20480
    case = real_case(rows, cols, 64, tokens)
    x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(tokens)).bfloat16().cuda()
    w = decode(case[1], case[2], 64, case[0], rows, cols)
    targets = targets_of(tokens, rows, tokens, 0.0)
    loss, lse, _, _, _ = plain(x, w, targets, torch.ones(tokens, device="cuda"))
    z = x.double() @ w.T
    mean = (torch.exp(z - lse[:, None]) * z.abs()).sum(1)
    got = bof4.bof4_cross_entropy(case[1], case[2], rows, cols, 64, case[0], x, targets, want_dx=grad)
    own, one = z[torch.arange(tokens, device="cuda"), targets].norm(), 2.0 ** -19 * tokens ** 0.5
    off = float((got[0].double() - loss).norm()), float((got[1].double() - lse).norm())
    print("loss by %d tokens, K = %d: %.2g, lse %.2g" % (tokens, cols, off[0] / float(loss.norm()), off[1] / float(lse.norm())))
    assert int(got[3].item()) == 0
    assert off[0] <= SUM * float(mean.norm() + own) + one and off[1] <= SUM * float(mean.norm()) + one
