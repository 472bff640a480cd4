"""bof4_linear and bof4_linear_backward against a plain implementation in 64 bits (written out here, without the library).

Integer-valued cases (every partial sum is representable in fp32) must agree bit for bit: they pin operand layouts, the
nibble order, block constants, outliers, cut tiles, strides and what lies beside the outputs.  Generic cases: a sum of
products differs from the exact one by at most 2^-14 * sum |w x| (K / 16 accumulation steps of at most 2^-23 each, K <= 8192,
one K of partial sums in fp32 more); the activations have slopes of at most 1.13 in magnitude and are evaluated within 2^-20
of max(|z|, 1); a result in bf16 is rounded once (2^-8 relative)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LV = np.array([-0.8568463921546936, -0.6692874431610107, -0.5235266089439392, -0.4004882574081421, -0.2910638153553009,
               -0.1900092959403992, -0.0938529595732689, 0.0, 0.0887671709060669, 0.1794802695512772, 0.2743096053600311,
               0.3760197460651398, 0.4886530041694641, 0.6188603639602661, 0.7791395783424377, 1.0], np.float32)
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def bof4():
    import __graft_entry__ as entry
    entry.build()
    import paper_2505_06653_b200 as m
    assert torch.cuda.is_available()
    return m


def act_code(bof4, name):
    return {"none": bof4.ACT_NONE, "relu": bof4.ACT_RELU, "gelu": bof4.ACT_GELU, "gelu_tanh": bof4.ACT_GELU_TANH, "silu": bof4.ACT_SILU}[name]


def act64(z, name):
    """Activation and derivative in 64 bits."""
    if name == "relu":
        return torch.clamp(z, min=0), (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if name == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        u = torch.tanh(c * (z + 0.044715 * z ** 3))
        return z * (1 + u) / 2, (1 + u) / 2 + z / 2 * (1 - u * u) * c * (1 + 3 * 0.044715 * z * z)
    return z, torch.ones_like(z)


def decode(codes, scales, block, levels, rows, cols, outliers=None):
    """bf16(constant * level) as a [rows, cols] double matrix."""
    c = torch.stack((codes >> 4, codes & 15), -1).reshape(-1).long()
    w = (torch.as_tensor(levels, device=codes.device)[c] * scales.float().repeat_interleave(block)).bfloat16().double()
    if outliers is not None:
        k = int(outliers[2].item())
        w[outliers[0][:k].long()] = outliers[1][:k].double()
    return w.view(rows, cols)


def integer_case(rows, cols, block, seed, scale_dtype=torch.bfloat16):
    """Levels multiples of 1/16, constants powers of two: products with small integers are multiples of 2^-8 below 4, so sums of
    up to 2^14 of them are exact in fp32 in whatever order."""
    g = torch.Generator().manual_seed(seed)
    lv = ((np.arange(16) - 7.5) / 8.0).astype(np.float32)
    codes = torch.randint(0, 256, (rows * cols // 2,), generator=g, dtype=torch.uint8)
    n = rows * cols // block
    scales = (2.0 ** torch.randint(-4, 2, (n,), generator=g)) * (torch.randint(0, 2, (n,), generator=g) * 2 - 1)
    return lv, codes.cuda(), scales.to(scale_dtype).cuda()


def real_case(rows, cols, block, seed, scale_dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (rows * cols // 2,), generator=g, dtype=torch.uint8)
    n = rows * cols // block
    scales = (0.04 + 0.02 * torch.rand(n, generator=g)) * (torch.randint(0, 2, (n,), generator=g) * 2 - 1)
    return LV, codes.cuda(), scales.to(scale_dtype).cuda()


def outlier_list(n, count, seed, integers=False, spare=0):
    g = torch.Generator().manual_seed(seed)
    idx = torch.randperm(n, generator=g)[:count].sort().values.int()
    val = torch.randint(-3, 4, (count,), generator=g).float() if integers else torch.randn(count, generator=g)
    pad = torch.zeros(spare, dtype=torch.int32)
    return (torch.cat((idx, pad)).cuda(), torch.cat((val, torch.zeros(spare))).bfloat16().cuda(), torch.tensor([count]).cuda())


def ints(g, *shape, lo=-2, hi=2, dtype=torch.bfloat16):
    return torch.randint(lo, hi + 1, shape, generator=g).to(dtype).cuda()


SHAPES = [(1, 64, 64, 64), (1, 32, 32, 32), (3, 8, 96, 32), (2, 130, 256, 64), (7, 200, 4096, 128), (8, 128, 1024, 1024), (9, 1, 512, 64),
          (16, 384, 2048, 64), (17, 129, 320, 64), (33, 257, 4096, 4096), (64, 1000, 1024, 64), (100, 333, 4032, 32), (129, 128, 192, 64),
          (256, 640, 1536, 64), (257, 96, 8192, 64), (300, 2050, 512, 256), (600, 384, 64, 64), (1, 5000, 8192, 64), (5, 4096, 14336, 64)]


@pytest.mark.parametrize("tokens,rows,cols,block", SHAPES)
@pytest.mark.parametrize("scale_dtype", [torch.bfloat16, torch.float32])
def test_integer_products_are_exact(bof4, tokens, rows, cols, block, scale_dtype):
    lv, codes, scales = integer_case(rows, cols, block, rows + cols, scale_dtype)
    g = torch.Generator().manual_seed(tokens)
    x, bias, res = ints(g, tokens, cols), ints(g, rows, dtype=torch.float32), ints(g, tokens, rows, dtype=torch.float32)
    w = decode(codes, scales, block, lv, rows, cols)
    z = x.double() @ w.T
    y, status = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32)
    assert int(status.item()) == 0 and y.dtype == torch.float32 and y.shape == (tokens, rows)
    assert torch.equal(y.double(), z)
    pre = torch.full((tokens, rows), 9.0, dtype=torch.bfloat16, device="cuda")
    y, status = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, bias=bias, residual=res, activation=bof4.ACT_RELU, out_dtype=bof4.F32, pre=pre)
    assert int(status.item()) == 0
    assert torch.equal(y.double(), torch.clamp(z + bias.double(), min=0) + res.double())
    assert torch.equal(pre, (z + bias.double()).bfloat16())
    y, status = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, bias=bias.bfloat16(), residual=res.bfloat16())
    assert int(status.item()) == 0 and torch.equal(y, (z + bias.double() + res.double()).bfloat16())


@pytest.mark.parametrize("tokens,rows,cols,block", SHAPES)
@pytest.mark.parametrize("scale_dtype", [torch.bfloat16, torch.float32])
def test_integer_gradients_are_exact(bof4, tokens, rows, cols, block, scale_dtype):
    lv, codes, scales = integer_case(rows, cols, block, rows + cols, scale_dtype)
    g = torch.Generator().manual_seed(tokens)
    dy = ints(g, tokens, rows)
    w = decode(codes, scales, block, lv, rows, cols)
    for t in (dy, dy.float()):
        dx, db, status = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, t, want_dbias=True)
        assert int(status.item()) == 0 and dx.dtype == torch.bfloat16 and db.dtype == torch.float32
        assert torch.equal(dx, (dy.double() @ w).bfloat16())
        assert torch.equal(db.double(), dy.double().sum(0))
    pre = ints(g, tokens, rows)
    dz = dy.double() * (pre > 0)
    dx, db, status = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, dy, pre=pre, activation=bof4.ACT_RELU)
    assert db is None and int(status.item()) == 0 and torch.equal(dx, (dz @ w).bfloat16())
    dx, db, status = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, dy, pre=pre, activation=bof4.ACT_RELU, want_dx=False, want_dbias=True)
    assert dx is None and int(status.item()) == 0 and torch.equal(db.double(), dz.sum(0))


@pytest.mark.parametrize("tokens,rows,cols,block,count", [(1, 64, 64, 64, 1), (4, 130, 512, 64, 700), (15, 128, 256, 32, 20000), (40, 300, 1024, 128, 300),
                                                          (16, 16, 64, 64, 1024), (200, 257, 2048, 64, 5000), (300, 512, 96, 32, 49152)])
def test_outliers_replace_their_weights(bof4, tokens, rows, cols, block, count):
    """From one outlier to every weight one."""
    lv, codes, scales = integer_case(rows, cols, block, 5)
    g = torch.Generator().manual_seed(count)
    out = outlier_list(rows * cols, count, count, integers=True, spare=37)
    w = decode(codes, scales, block, lv, rows, cols, out)
    x, dy = ints(g, tokens, cols), ints(g, tokens, rows)
    y, status = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32, outliers=out)
    assert int(status.item()) == 0 and torch.equal(y.double(), x.double() @ w.T)
    dx, _, status = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, dy, outliers=out)
    assert int(status.item()) == 0 and torch.equal(dx, (dy.double() @ w).bfloat16())
    # a count beyond the arrays: the entries that are there; an empty list; a list without room
    over = (out[0][:count], out[1][:count], torch.tensor([count + 5]).cuda())
    assert torch.equal(y, bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32, outliers=over)[0])
    none = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32)[0]
    zero = (out[0], out[1], torch.tensor([0]).cuda())
    assert torch.equal(none, bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32, outliers=zero)[0])
    assert torch.equal(none, bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32, outliers=(out[0][:0], out[1][:0], zero[2]))[0])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("tokens,rows,cols,block,count", [(1, 200, 1024, 64, 0), (6, 1030, 4096, 64, 99), (12, 512, 8192, 128, 0), (90, 384, 2048, 32, 500), (300, 256, 4096, 64, 0)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_generic_products(bof4, act, tokens, rows, cols, block, count, out):
    lv, codes, scales = real_case(rows, cols, block, tokens, torch.float32)
    g = torch.Generator().manual_seed(rows)
    dt = torch.float32 if out == "f32" else torch.bfloat16
    x = torch.randn(tokens, cols, generator=g).bfloat16().cuda()
    bias, res = torch.randn(rows, generator=g).to(dt).cuda(), torch.randn(tokens, rows, generator=g).to(dt).cuda()
    lst = outlier_list(rows * cols, count, 3) if count else None
    w = decode(codes, scales, block, lv, rows, cols, lst)
    z = x.double() @ w.T + bias.double()
    mag = x.double().abs() @ w.abs().T + bias.double().abs()
    pre = torch.empty(tokens, rows, dtype=torch.bfloat16, device="cuda")
    y, status = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, bias=bias, residual=res, activation=act_code(bof4, act),
                                 out_dtype=bof4.F32 if out == "f32" else bof4.BF16, pre=pre, outliers=lst)
    assert int(status.item()) == 0
    ref = act64(z, act)[0] + res.double()
    tol = 1.13 * 2.0 ** -14 * mag + 2.0 ** -20 * torch.clamp(z.abs(), min=1) + 2.0 ** -23 * ref.abs()
    assert bool(((pre.double() - z).abs() <= 2.0 ** -14 * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * z.abs()).all())
    if out == "bf16":
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()
    assert bool(((y.double() - ref).abs() <= tol).all()), float(((y.double() - ref).abs() / tol).max())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("tokens,rows,cols,block,count", [(1, 200, 1024, 64, 0), (6, 1030, 512, 64, 99), (70, 513, 320, 64, 0), (90, 2048, 384, 32, 500), (300, 4096, 256, 64, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_generic_gradients(bof4, act, tokens, rows, cols, block, count, dtype):
    """dz is within 2^-19 of |dy| * 1.13 before its rounding to bf16 (2^-8); sums over tokens as in the module's text."""
    lv, codes, scales = real_case(rows, cols, block, tokens)
    g = torch.Generator().manual_seed(rows)
    dy = torch.randn(tokens, rows, generator=g).to(dtype).cuda()
    pre = (3 * torch.randn(tokens, rows, generator=g)).bfloat16().cuda()
    lst = outlier_list(rows * cols, count, 3) if count else None
    w = decode(codes, scales, block, lv, rows, cols, lst)
    dz = dy.double() * act64(pre.double(), act)[1]
    dx, db, status = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, dy, pre=pre, activation=act_code(bof4, act), want_dbias=True, outliers=lst)
    assert int(status.item()) == 0
    e_dz = 2.0 ** -19 * dy.double().abs() * 1.13
    tol = (2.0 ** -8 * (dz.abs() + e_dz) + e_dz + 2.0 ** -14 * dz.abs()) @ w.abs()
    ref = dz @ w
    tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()
    assert bool(((dx.double() - ref).abs() <= tol).all()), float(((dx.double() - ref).abs() / tol).max())
    tb = e_dz.sum(0) + (tokens + 16) * 2.0 ** -24 * dz.abs().sum(0)
    assert bool(((db.double() - dz.sum(0)).abs() <= tb + 1e-30).all())


@pytest.mark.parametrize("act", ACTS)
def test_gradient_agrees_with_differences(bof4, act):
    """A directional difference of the forward pass (fp32 results) against the backward pass's gradients of input and bias."""
    tokens, rows, cols, block = 24, 96, 256, 64
    lv, codes, scales = real_case(rows, cols, block, 8, torch.float32)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(tokens, cols, generator=g).bfloat16().cuda()
    bias = torch.randn(rows, generator=g).cuda()
    c = torch.randn(tokens, rows, generator=g).cuda()     # the loss is sum c * y
    a = act_code(bof4, act)
    pre = torch.empty(tokens, rows, dtype=torch.bfloat16, device="cuda")
    bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, bias=bias, activation=a, out_dtype=bof4.F32, pre=pre)
    dx, db, _ = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, c, pre=pre, activation=a, want_dbias=True)
    loss = lambda xx, bb: float((c.double() * bof4.bof4_linear(codes, scales, rows, cols, block, lv, xx, bias=bb, activation=a, out_dtype=bof4.F32)[0].double()).sum())  # noqa: E731
    # a step of exactly representable size in a few inputs of each token; relu and the curvature of the others leave 4 %
    step = torch.zeros_like(x)
    step[:, ::7] = (torch.randint(0, 2, (tokens, len(range(0, cols, 7))), generator=g) * 2 - 1).bfloat16().cuda() * 2.0 ** -6
    xp, xm = (x.float() + step.float()).bfloat16(), (x.float() - step.float()).bfloat16()
    got, want = loss(xp, bias) - loss(xm, bias), float(((xp.double() - xm.double()) * dx.double()).sum())
    scale = float(((xp.double() - xm.double()) * dx.double()).norm()) * 4
    assert abs(got - want) <= 0.04 * max(scale, abs(want)), (got, want, scale)
    h = torch.full_like(bias, 2.0 ** -8)
    got, want = loss(x, bias + h) - loss(x, bias - h), float((2 * h * db).sum())
    scale = float((2 * h * db).norm()) * 4
    assert abs(got - want) <= 0.04 * max(scale, abs(want)), (got, want, scale)


def test_strides_and_what_lies_beside(bof4):
    """Rows apart from one another in every tensor; values between the rows stay as they were; the residual may be the result."""
    for tokens, rows, cols in ((1, 70, 128), (5, 131, 512), (40, 258, 256), (270, 100, 64)):
        lv, codes, scales = integer_case(rows, cols, 32, 1)
        g = torch.Generator().manual_seed(rows)
        w = decode(codes, scales, 32, lv, rows, cols)
        xs = ints(g, tokens, cols + 24)
        ys, ps, rs = (torch.full((tokens, rows + k), 77.0, dtype=torch.bfloat16, device="cuda") for k in (3, 5, 6))
        rs[:, :rows] = ints(g, tokens, rows)
        z = xs[:, :cols].double() @ w.T
        out, status = bof4.bof4_linear(codes, scales, rows, cols, 32, lv, xs[:, :cols], residual=rs[:, :rows], pre=ps[:, :rows], out=ys[:, :rows])
        assert int(status.item()) == 0 and out.data_ptr() == ys.data_ptr()
        assert torch.equal(ys[:, :rows], (z + rs[:, :rows].double()).bfloat16()) and torch.equal(ps[:, :rows], z.bfloat16())
        assert bool((ys[:, rows:] == 77).all()) and bool((ps[:, rows:] == 77).all())
        want = (z + rs[:, :rows].double()).bfloat16()
        bof4.bof4_linear(codes, scales, rows, cols, 32, lv, xs[:, :cols], residual=rs[:, :rows], out=rs[:, :rows])
        assert torch.equal(rs[:, :rows], want) and bool((rs[:, rows:] == 77).all())
        for dt in (torch.bfloat16, torch.float32):
            for k in (0, 1, 8):  # aligned and not: by TMA, by vectors, one by one
                dys = ints(g, tokens, rows + k, dtype=dt)
                pr = ints(g, tokens, rows + 3)
                dxs = torch.full((tokens, cols + 2), 77.0, dtype=torch.bfloat16, device="cuda")
                dx, db, status = bof4.bof4_linear_backward(codes, scales, rows, cols, 32, lv, dys[:, :rows], want_dbias=True, out=dxs[:, :cols])
                assert int(status.item()) == 0 and torch.equal(dx, (dys[:, :rows].double() @ w).bfloat16()) and bool((dxs[:, cols:] == 77).all())
                assert torch.equal(db.double(), dys[:, :rows].double().sum(0))
                dx, db, status = bof4.bof4_linear_backward(codes, scales, rows, cols, 32, lv, dys[:, :rows], pre=pr[:, :rows], activation=bof4.ACT_RELU, want_dbias=True)
                dz = dys[:, :rows].double() * (pr[:, :rows] > 0)
                assert torch.equal(dx, (dz @ w).bfloat16()) and torch.equal(db.double(), dz.sum(0))


def test_empty_shapes(bof4):
    lv = LV
    e8, eb = torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(0, dtype=torch.bfloat16, device="cuda")
    bias, res = torch.randn(6).cuda(), torch.randn(3, 6).cuda()
    y, s = bof4.bof4_linear(e8, eb, 6, 0, 64, lv, torch.empty(3, 0, dtype=torch.bfloat16, device="cuda"), bias=bias, residual=res, activation=bof4.ACT_RELU, out_dtype=bof4.F32)
    assert int(s.item()) == 0 and torch.equal(y, torch.clamp(bias, min=0) + res)
    y, s = bof4.bof4_linear(e8, eb, 0, 64, 64, lv, torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda"))
    assert y.shape == (3, 0) and int(s.item()) == 0
    lv, codes, scales = integer_case(6, 64, 64, 1)
    y, s = bof4.bof4_linear(codes, scales, 6, 64, 64, lv, torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"))
    assert y.shape == (0, 6) and int(s.item()) == 0
    dx, db, s = bof4.bof4_linear_backward(codes, scales, 6, 64, 64, lv, torch.zeros(0, 6, dtype=torch.bfloat16, device="cuda"), want_dbias=True)
    assert dx.shape == (0, 64) and bool((db == 0).all()) and int(s.item()) == 0
    dx, db, s = bof4.bof4_linear_backward(e8, eb, 0, 64, 64, lv, torch.zeros(2, 0, dtype=torch.bfloat16, device="cuda"))
    assert bool((dx == 0).all()) and dx.shape == (2, 64)
    dx, db, s = bof4.bof4_linear_backward(e8, eb, 6, 0, 64, lv, torch.ones(2, 6, dtype=torch.bfloat16, device="cuda"), want_dbias=True)
    assert dx.shape == (2, 0) and bool((db == 2).all())


def test_non_finite_tokens_stay_by_themselves(bof4):
    """An infinity or a NaN in one token makes that token's results non-finite and no other's."""
    rows, cols = 200, 512
    lv, codes, scales = integer_case(rows, cols, 64, 4)
    w = decode(codes, scales, 64, lv, rows, cols)
    for tokens in (3, 20, 300):
        x = ints(torch.Generator().manual_seed(tokens), tokens, cols)
        x[1, 5], x[tokens - 1, 7] = float("inf"), float("nan")
        y, status = bof4.bof4_linear(codes, scales, rows, cols, 64, lv, x, out_dtype=bof4.F32)
        keep = [t for t in range(tokens) if t not in (1, tokens - 1)]
        assert int(status.item()) == 0 and torch.equal(y[keep].double(), x[keep].double() @ w.T)
        assert not bool(torch.isfinite(y[1]).any()) and bool(torch.isnan(y[tokens - 1]).all())


@pytest.mark.parametrize("tokens", [1, 12, 20, 300])
@pytest.mark.parametrize("rows,cols,block", [(200, 96, 32), (131, 320, 64), (64, 64, 64), (300, 4096, 4096), (77, 8256, 64)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_non_finite_weights_stay_in_their_rows_and_columns(bof4, tokens, rows, cols, block, bad):
    """Blocks whose constant is not finite reach the results of their own row (forward) and columns (backward), and no others:
    what pads a matrix to whole tiles is zero."""
    lv, codes, scales = integer_case(rows, cols, block, 6)
    per_row, row = cols // block, rows // 2
    scales[row * per_row] = scales[-1] = bad        # the first block of a row, and the last one of the matrix
    w = decode(codes, scales, block, lv, rows, cols)
    g = torch.Generator().manual_seed(tokens)
    x, dy = ints(g, tokens, cols, lo=1, hi=2), ints(g, tokens, rows, lo=1, hi=2)
    y, status = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32)
    keep = [r for r in range(rows) if r not in (row, rows - 1)]
    assert int(status.item()) == 0 and torch.equal(y[:, keep].double(), x.double() @ w[keep].T)
    assert not bool(torch.isfinite(y[:, [row, rows - 1]]).any())
    dx, _, status = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, dy)
    hit = torch.zeros(cols, dtype=torch.bool, device="cuda")
    hit[:block] = hit[-block:] = True
    assert int(status.item()) == 0 and torch.equal(dx[:, ~hit], (dy.double() @ w[:, ~hit]).bfloat16())
    assert not bool(torch.isfinite(dx[:, hit]).any())


def test_the_operand_is_what_dequantise_writes(bof4):
    """A run of the calls as they are used: quantise with outliers, one token and many through the layer, its gradient."""
    rows, cols, block = 256, 1024, 64
    w = (torch.randn(rows * cols, generator=torch.Generator().manual_seed(1)) * 0.02).bfloat16()
    w[::997] = 0.5
    tau = float(np.float32(bof4.bof4_opq_threshold(0.95, block)))
    codes, scales, idx, val, cnt = bof4.bof4_quantize_opq(w.cuda(), block, bof4.NORM_SIGNED, LV, tau, 4096)
    out = (idx, val, cnt)
    wd = bof4.bof4_dequantize(codes, scales, block, LV, bof4.BF16, out).view(rows, cols)
    assert torch.equal(wd.double(), decode(codes, scales, block, LV, rows, cols, out))
    for tokens in (1, 8, 40, 300):
        x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(tokens)).bfloat16().cuda()
        res = torch.randn(tokens, rows).bfloat16().cuda()
        pre = torch.empty(tokens, rows, dtype=torch.bfloat16, device="cuda")
        y, s = bof4.bof4_linear(codes, scales, rows, cols, block, LV, x, residual=res, activation=bof4.ACT_SILU, outliers=out, pre=pre)
        z, mag = x.double() @ wd.double().T, x.double().abs() @ wd.double().abs().T
        ref = act64(z, "silu")[0] + res.double()
        assert bool(((y.double() - ref).abs() <= 2.0 ** -13 * mag + 2.0 ** -19 * (1 + z.abs()) + 2.0 ** -8 * ref.abs()).all())
        dx, db, s = bof4.bof4_linear_backward(codes, scales, rows, cols, block, LV, y, pre=pre, activation=bof4.ACT_SILU, want_dbias=True, outliers=out)
        dz = y.double() * act64(pre.double(), "silu")[1]
        ref = dz @ wd.double()
        assert bool(((dx.double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -12) * (dz.abs() @ wd.double().abs()) + 2.0 ** -8 * ref.abs()).all())


def test_same_bits_again_on_other_streams_and_in_graphs(bof4):
    """Repeated, on a side stream, captured and replayed, two graphs sharing one workspace: the same bits."""
    for tokens, rows, cols in ((4, 1000, 2048), (50, 700, 4096), (300, 300, 1024)):
        lv, codes, scales = real_case(rows, cols, 64, 3)
        lst = outlier_list(rows * cols, 100, 2)
        x = torch.randn(tokens, cols).bfloat16().cuda()
        dy = torch.randn(tokens, rows).bfloat16().cuda()
        cb = torch.from_numpy(lv).cuda()
        fwd = lambda ws=None, out=None: bof4.bof4_linear(codes, scales, rows, cols, 64, cb, x, outliers=lst, out=out, workspace=ws)[0]  # noqa: E731
        bwd = lambda ws=None, out=None: bof4.bof4_linear_backward(codes, scales, rows, cols, 64, cb, dy, outliers=lst, out=out, workspace=ws)[0]  # noqa: E731
        y, dx = fwd().clone(), bwd().clone()
        assert torch.equal(y, fwd()) and torch.equal(dx, bwd())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            a, b = fwd(), bwd()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(a, y) and torch.equal(b, dx)
        n = max(bof4.bof4_linear_workspace_bytes(rows, cols, tokens, k, 100) for k in (False, True))
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        oy, odx = torch.empty_like(y), torch.empty_like(dx)
        graphs = []
        for f, o in ((fwd, oy), (bwd, odx)):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                f(ws, o)
            graphs.append(g)
        for _ in range(3):
            oy.zero_(), odx.zero_()
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            assert torch.equal(oy, y) and torch.equal(odx, dx)


@pytest.mark.parametrize("tokens,rows,cols", [(3, 5000, 8192), (14, 2560, 4096), (40, 5000, 8192), (100, 5120, 8192), (250, 2560, 4096)])
def test_cold_memory(bof4, tokens, rows, cols):
    """Inputs that have left L2 arrive late and in another order: the same results, with any contents of the workspace."""
    lv, codes, scales = integer_case(rows, cols, 64, rows + cols)
    g = torch.Generator().manual_seed(tokens)
    dy, x = ints(g, tokens, rows), ints(g, tokens, cols)
    w = decode(codes, scales, 64, lv, rows, cols)
    rb, rf = (dy.double() @ w).bfloat16(), (x.double() @ w.T).float()
    big = torch.empty(300 << 20, dtype=torch.uint8, device="cuda")
    n = max(bof4.bof4_linear_workspace_bytes(rows, cols, tokens, k) for k in (False, True))
    for trial in range(12):
        ws = torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda")
        big.fill_(trial)
        dx, _, s = bof4.bof4_linear_backward(codes, scales, rows, cols, 64, lv, dy, workspace=ws)
        assert int(s.item()) == 0 and torch.equal(dx, rb)
        big.fill_(trial)
        y, s = bof4.bof4_linear(codes, scales, rows, cols, 64, lv, x, out_dtype=bof4.F32, workspace=ws)
        assert int(s.item()) == 0 and torch.equal(y, rf)


def test_random_shapes_are_exact(bof4):
    rng = np.random.default_rng(11)
    for trial in range(60):
        block = int(rng.choice([32, 64, 128, 256, 1024]))
        cols = block * int(rng.integers(1, 1 + 8192 // block))
        rows, tokens = int(rng.integers(1, 1500)), int(np.exp(rng.uniform(0, np.log(700))))
        lv, codes, scales = integer_case(rows, cols, block, trial, torch.float32 if trial % 2 else torch.bfloat16)
        g = torch.Generator().manual_seed(trial)
        lst = outlier_list(rows * cols, min(rows * cols, int(rng.integers(1, 2000))), trial, integers=True) if trial % 3 == 0 else None
        w = decode(codes, scales, block, lv, rows, cols, lst)
        x, dy = ints(g, tokens, cols), ints(g, tokens, rows)
        y, s = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32, outliers=lst)
        assert int(s.item()) == 0 and torch.equal(y.double(), x.double() @ w.T), (tokens, rows, cols, block)
        dx, _, s = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, dy, outliers=lst)
        assert int(s.item()) == 0 and torch.equal(dx, (dy.double() @ w).bfloat16()), (tokens, rows, cols, block)


def test_offsets_beyond_32_bits(bof4):
    """A matrix of more than 2^32 weights, results of more than 2^31 values: rows, tokens and columns at the far ends."""
    rows, cols, block = 132000, 32768, 4096
    g = torch.Generator(device="cuda").manual_seed(1)
    lv = integer_case(1, 64, 64, 1)[0]
    codes = torch.randint(0, 256, (rows * cols // 2,), generator=g, dtype=torch.uint8, device="cuda")
    scales = 2.0 ** torch.randint(-4, 2, (rows * cols // block,), generator=g, device="cuda").bfloat16()
    some = [0, 65535, 65536, 131071, 131072, rows - 1]
    w = torch.cat([decode(codes[r * cols // 2:(r + 1) * cols // 2], scales[r * cols // block:(r + 1) * cols // block], block, lv, 1, cols) for r in some])
    for tokens in (1, 9, 20):
        x = torch.randint(-1, 2, (tokens, cols), generator=g, device="cuda").bfloat16()
        x[:, :28672] = 0  # (the sums stay exact)
        y, status = bof4.bof4_linear(codes, scales, rows, cols, block, lv, x, out_dtype=bof4.F32)
        assert int(status.item()) == 0 and torch.equal(y[:, some].double(), x.double() @ w.T)
    dy = torch.zeros(20, rows, dtype=torch.bfloat16, device="cuda")
    dy[:, some] = torch.randint(-2, 3, (20, len(some)), generator=g, device="cuda").bfloat16()
    dx, db, status = bof4.bof4_linear_backward(codes, scales, rows, cols, block, lv, dy, want_dbias=True)
    assert int(status.item()) == 0 and torch.equal(dx, (dy[:, some].double() @ w).bfloat16()) and torch.equal(db, dy.float().sum(0))
    del codes, scales, w, dy
    tokens, rows, cols = 67000, 32768, 64
    lv, codes, scales = integer_case(rows, cols, 64, 2)
    w = decode(codes, scales, 64, lv, rows, cols)
    x = torch.randint(-2, 3, (tokens, cols), generator=g, device="cuda").bfloat16()
    y, status = bof4.bof4_linear(codes, scales, rows, cols, 64, lv, x)
    some = [0, 65535, 65536, tokens - 1]
    assert int(status.item()) == 0 and torch.equal(y[some], (x[some].double() @ w.T).bfloat16())
    y.zero_()
    y[some] = torch.randint(-1, 2, (len(some), rows), generator=g, device="cuda").bfloat16()
    y[:, 4096:] = 0
    dx, db, status = bof4.bof4_linear_backward(codes, scales, rows, cols, 64, lv, y.relu(), pre=y, activation=bof4.ACT_RELU, want_dbias=True)
    assert int(status.item()) == 0 and torch.equal(dx[some], (y[some].relu().double() @ w).bfloat16()) and torch.equal(db, y[some].relu().float().sum(0))
    assert int(torch.count_nonzero(dx)) == int(torch.count_nonzero(dx[some]))


def test_refusals(bof4):
    rows, cols = 8, 128
    lv, codes, scales = integer_case(rows, cols, 64, 1)
    x = torch.zeros(2, cols, dtype=torch.bfloat16, device="cuda")
    ok = dict(codes=codes, scales=scales, rows=rows, cols=cols, block_size=64, levels=lv, x=x)
    bof4.bof4_linear(**ok)
    bad = lambda err, **kw: pytest.raises(err, bof4.bof4_linear, **{**ok, **kw})  # noqa: E731
    bad(ValueError, x=x.cpu())
    bad(TypeError, x=x.float())
    bad(ValueError, x=x[:, :64])
    bad(ValueError, x=x.T.contiguous().T)
    bad(ValueError, codes=codes[:-32])
    bad(ValueError, scales=scales[:-1])
    bad(ValueError, bias=torch.zeros(7, device="cuda"))
    bad(TypeError, bias=torch.zeros(8, device="cuda", dtype=torch.float16))
    bad(TypeError, residual=torch.zeros(2, 8, device="cuda"))
    bad(ValueError, residual=torch.zeros(3, 8, device="cuda", dtype=torch.bfloat16))
    bad(ValueError, out=torch.zeros(2, 9, device="cuda", dtype=torch.bfloat16))
    bad(ValueError, out=torch.zeros(1, 8, device="cuda", dtype=torch.bfloat16).expand(2, 8))
    bad(bof4.Bof4Error, activation=5)
    bad(bof4.Bof4Error, activation=-1)
    bad(ValueError, out_dtype=7)
    need = bof4.bof4_linear_workspace_bytes(rows, cols, 2)
    bad(bof4.Bof4Error, workspace=torch.zeros(need - 1, dtype=torch.uint8, device="cuda"))
    bad(ValueError, workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    wide = torch.zeros(2, cols + 4, dtype=torch.bfloat16, device="cuda")
    bad(bof4.Bof4Error, x=wide[:, :cols])            # rows 264 bytes apart: not a multiple of 16
    bad(bof4.Bof4Error, x=torch.zeros(2 * cols + 8, dtype=torch.bfloat16, device="cuda")[4:4 + 2 * cols].view(2, cols))
    bad(ValueError, outliers=(torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")))
    dy = torch.zeros(2, rows, dtype=torch.bfloat16, device="cuda")
    okb = dict(codes=codes, scales=scales, rows=rows, cols=cols, block_size=64, levels=lv, dy=dy)
    bof4.bof4_linear_backward(**okb)
    badb = lambda err, **kw: pytest.raises(err, bof4.bof4_linear_backward, **{**okb, **kw})  # noqa: E731
    badb(bof4.Bof4Error, activation=bof4.ACT_SILU)   # without the values before it
    badb(ValueError, dy=dy[:, :4])
    badb(TypeError, dy=dy.half())
    badb(TypeError, pre=dy.float(), activation=bof4.ACT_SILU)
    badb(bof4.Bof4Error, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
