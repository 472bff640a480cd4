"""What the layers over 4-bit matrices promise about precision, each promise by itself: activations and slopes on values before them that are
exact, the two halves of an expert layer's h, and how much of a long sum in fp32 is lost."""
import math

import pytest
import torch

from test_gpu_linear import ACTS, act64, act_code, bof4, decode, real_case  # noqa: F401
from test_gpu_moe import ONE, PICK, ZERO, packed

pytestmark = pytest.mark.gpu

ROWS = 4096


def sweep():
    """Values before an activation: -8 ... 8 closely, and far out."""
    far = torch.tensor([0.0, 9.5, 12.0, 20.0, 60.0, 87.0, 89.0, 100.0, 1e4, 1e13, 1e30])
    z = torch.linspace(-8, 8, ROWS)
    z[:22] = torch.cat((far, -far))
    return z.cuda()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("tokens,cols,block", [(3, 512, 64), (12, 512, 64), (3, 8192, 4096), (12, 8192, 64), (40, 128, 64), (300, 128, 32), (40, 4096, 64), (300, 4096, 64)])
def test_activations_of_the_linear_layer(bof4, act, tokens, cols, block):  # noqa: F811
    """Tokens of zeros, so that the bias is the value before the activation: in the forms for few and for many tokens, with rows (few) and tiles
    (many) that one CTA has whole and that are cut.  An activation is within 2^-20 of max(|z|, 1), as everywhere in these tests; the two forms of
    GELU are 2^-11 apart."""
    _, codes, scales = real_case(ROWS, cols, block, 1)
    x = torch.zeros(tokens, cols, dtype=torch.bfloat16, device="cuda")
    bias = sweep()
    ref = act64(bias.double(), act)[0]
    tol = 2.0 ** -20 * bias.double().abs().clamp(min=1)
    lv = torch.from_numpy(real_case(1, 32, 32, 1)[0]).cuda()
    pre = torch.empty(tokens, ROWS, dtype=torch.bfloat16, device="cuda")
    y, s = bof4.bof4_linear(codes, scales, ROWS, cols, block, lv, x, bias=bias, activation=act_code(bof4, act), out_dtype=bof4.F32, pre=pre)
    assert int(s.item()) == 0 and torch.equal(pre, bias.bfloat16().expand(tokens, ROWS))
    assert bool(((y.double() - ref).abs() <= tol).all()), float(((y.double() - ref).abs() / tol).max())
    res = torch.zeros(tokens, ROWS + 1, dtype=torch.bfloat16, device="cuda")
    for r in (None, res[:, :ROWS].contiguous(), res[:, :ROWS]):    # (rows an odd number of values apart are not written in pairs)
        y, s = bof4.bof4_linear(codes, scales, ROWS, cols, block, lv, x, bias=bias, residual=r, activation=act_code(bof4, act))
        assert int(s.item()) == 0 and bool(((y.double() - ref).abs() <= tol * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()).all())


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_slopes(bof4, act):  # noqa: F811
    """The derivative at every finite bf16 value, through the bias gradient of one token with dy = 1, which is not rounded.

    With u = 2^-24 and t = exp(-|v|) off by (4 + 2.4 |v|) u (the fast form's 2 + 1.173 |v| units; for the tanh form another 3 |v| u, the rounding
    of its argument v) and a quotient by 4 u (2 units) and the rounding of its divisor: the logistic part s is off by less than 6.1 u, the part
    q s (1 - s) by less than 5.5 u (SILU, q = z) and 8.1 u (tanh form), maxima over v of the first-order terms with four roundings; with the
    last sum's rounding 12 u and 15.3 u.  GELU: half of erfc, 4 units of a value of up to 2, and of its argument's rounding 5 u, z phi(z) 2 u, the sum 1 u.
    All are below 16 u = 2^-20."""
    bits = torch.arange(1 << 16, dtype=torch.int32)
    pre = bits[(bits & 0x7F80) != 0x7F80].to(torch.int16).view(torch.bfloat16).view(1, -1).cuda()
    rows = pre.shape[1]
    assert rows == 65280
    _, codes, scales = real_case(rows, 32, 32, 1)
    _, db, s = bof4.bof4_linear_backward(codes, scales, rows, 32, 32, PICK, torch.ones(1, rows, device="cuda"), pre=pre, activation=act_code(bof4, act), want_dx=False,
                                         want_dbias=True)
    z = pre[0].double()
    ref = act64(z.clamp(-1000, 1000), act)[1]
    err = (db.double() - ref).abs()
    at = int(err.argmax())
    print("%s: %.3g = 2^%.2f at z = %g" % (act, float(err[at]), math.log2(float(err[at])), float(z[at])))
    assert int(s.item()) == 0 and bool((err <= 2.0 ** -20).all()), (float(err[at]), float(z[at]))


def picked(tokens, hidden, ffn, terms, seed, power):
    """One expert whose gate's rows have `terms` columns (odd multiples of 1/16 from column 1 on), whose up rows take column 0 alone and whose
    down matrix is the identity, with tokens of x0 = 1 and x_k = `power`^(k - 1): g is exact, h = act(g), y = h.  -> x, matrices, g"""
    g = torch.Generator().manual_seed(seed)
    up = torch.full((2 * ffn, hidden), ZERO)
    up[:ffn, 1:1 + terms] = torch.randint(0, 14, (ffn, terms), generator=g)
    up[ffn:, 0] = ONE
    down = torch.full((hidden, ffn), ZERO)
    down[torch.arange(ffn), torch.arange(ffn)] = ONE
    x = torch.zeros(tokens, hidden)
    x[:, 0] = 1
    x[:, 1:1 + terms] = torch.tensor([float(power) ** k for k in range(terms)])
    x[:, 1:1 + terms] *= torch.randint(0, 2, (tokens, terms), generator=g) * 2 - 1
    z = x.double() @ torch.from_numpy(PICK).double()[up[:ffn]].T
    return x.bfloat16().cuda(), packed(up, 1.0), packed(down, 1.0), z.cuda()


def one_expert(bof4, x, gate_up, down, ffn, act):  # noqa: F811
    y, _, w, s = bof4.bof4_moe(x, torch.zeros(1, x.shape[1], device="cuda"), gate_up, down, ffn, 64, PICK, 1, activation=act_code(bof4, act), out_dtype=bof4.F32)
    assert int(s.item()) == 0 and bool((w == 1).all())
    return y[:, :ffn].double()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("tokens,hidden,ffn", [(1, 64, 64), (11, 256, 256), (5, 4608, 192)])
def test_activations_of_the_expert_layer(bof4, act, tokens, hidden, ffn):  # noqa: F811
    """h = act(g), g an exact sum of 9 values of up to 15/16: 2^-20 of max(|g|, 1) and 2^-17 of h."""
    x, gate_up, down, z = picked(tokens, hidden, ffn, 9, 3, 1)
    h = act64(z, act)[0]
    tol = 2.0 ** -20 * z.abs().clamp(min=1) + 2.0 ** -17 * h.abs()
    y = one_expert(bof4, x, gate_up, down, ffn, act)
    assert bool(((y - h).abs() <= tol).all()), float(((y - h).abs() / tol).max())


@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("tokens", [1, 4, 9])
def test_both_halves_of_h(bof4, act, tokens):  # noqa: F811
    """h of up to 12 bits arrives whole, h of 20 bits within 2^-17 (one bf16 value alone would be 2^-9 off)."""
    for terms, whole in ((2, True), (3, False)):
        x, gate_up, down, z = picked(tokens, 128, 128, terms, terms, 256)
        h = act64(z, act)[0]
        y = one_expert(bof4, x, gate_up, down, 128, act)
        if whole:
            assert torch.equal(y, h)
        assert bool(((y - h).abs() <= 2.0 ** -17 * h.abs()).all())
        assert not torch.equal(h.bfloat16().double(), h)


@pytest.mark.parametrize("tokens,cols,bound", [(12, 8192, 2.5e-6), (24, 8192, 2.5e-6), (64, 8192, 2.5e-6), (100, 8192, 5e-6), (300, 8192, 5e-6), (300, 4096, 5e-6)])
def test_long_sums_in_fp32(bof4, tokens, cols, bound):  # noqa: F811
    """2-norm of the error beside that of the result.  A tensor core cuts a sum off at each step of 16 of K, a quarter of a unit of the running sum
    on average and always towards zero, so that n steps in one accumulator cost about 2^-24 n / 4: 7e-6 at K = 8192.  Results in fp32 have two
    accumulators there up to 128 tokens of a tile and four up to 64: a half and a quarter of that, and room for the roundings of the sums of cut tiles."""
    rows, block = 20480, 64   # more tiles than SMs: most have their whole K in one part
    lv, codes, scales = real_case(rows, cols, block, tokens, torch.float32)
    x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(cols)).bfloat16().cuda()
    ref = x.double() @ decode(codes, scales, block, lv, rows, cols).T
    y, s = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32)
    err = float((y.double() - ref).norm() / ref.norm())
    print("%d tokens, K = %d: %.2g" % (tokens, cols, err))
    assert int(s.item()) == 0 and err < bound
