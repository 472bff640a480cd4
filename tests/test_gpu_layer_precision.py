"""What the layers over 4-bit matrices promise about precision, each promise by itself: activations and slopes on values before them that are
exact, the two halves of an expert layer's h, and how much of a long sum in fp32 is lost."""
import math

import pytest
import torch

from test_gpu_linear import act64, act_code, bof4, real_case  # noqa: F401
from test_gpu_moe import PICK

pytestmark = pytest.mark.gpu

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
