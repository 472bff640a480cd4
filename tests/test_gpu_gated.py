"""bof4_gated and bof4_gated_backward against a plain implementation in 64 bits (written out here, without the library).

Integer-valued cases (every partial sum of a projection is representable in fp32) must agree bit for bit: a product of two exact fp32 values
is rounded once, and once more to bf16.  Generic cases: a projection differs from the exact one by at most d = 2^-14 * sum |w x| (K / 16
accumulation steps of at most 2^-23 each, K <= 8192, one K of partial sums in fp32 more); the activations have slopes of at most
1.13 in magnitude and are evaluated within 2^-20 of max(|z|, 1); so h is off by (1.13 d_g + 2^-20 max(|g|, 1)) (|u| + d_u) + |act(g)| d_u, and by half
a step of its type.  A gradient's operand is rounded to bf16 (2^-8 of each term), its sum is off like a projection's, and dx is rounded once."""

import pytest
import torch

from test_gpu_linear import LV, act64, act_code, decode, integer_case, ints, outlier_list, real_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bof4():
    import __graft_entry__ as entry
    entry.build()
    import paper_2505_06653_b200 as m
    assert torch.cuda.is_available()
    return m


# tokens on both sides of 6, 8, 16, 64, 128, 256 and of the form for many tokens; ffn that are no multiple of 8, 32, 64 or 128; K of one block and of
# part of a line; several slices of columns for few tokens
SHAPES = [(1, 32, 64, 64), (1, 5, 32, 32), (2, 65, 256, 64), (5, 200, 4096, 128), (8, 96, 1024, 1024), (9, 7, 512, 64), (16, 130, 10240, 64), (17, 129, 320, 64),
          (33, 64, 4096, 4096), (64, 1000, 512, 64), (130, 100, 4032, 32), (256, 333, 1536, 64), (300, 1025, 512, 256), (767, 192, 96, 32), (768, 127, 64, 64),
          (1000, 200, 4128, 32), (1300, 1111, 2080, 32), (2049, 64, 512, 64), (769, 4736, 256, 64),
          # tiles of the form for many tokens that are cut along K: into three, two goes of all clusters (forward; backward)
          (1000, 1500, 4096, 64), (1000, 2100, 2944, 64),
          # a large matrix by more than twelve tokens
          (14, 8200, 4096, 64),
          # several tiles of tokens of the form that decodes as it multiplies
          (200, 300, 1280, 64), (300, 2100, 4096, 64), (600, 4200, 4096, 64)]


@pytest.mark.parametrize("tokens,ffn,cols,block", SHAPES)
@pytest.mark.parametrize("scale_dtype", [torch.bfloat16, torch.float32])
def test_integer_blocks_are_exact(bof4, tokens, ffn, cols, block, scale_dtype):
    lv, codes, scales = integer_case(2 * ffn, cols, block, ffn + cols, scale_dtype)
    g = torch.Generator().manual_seed(tokens)
    x, bias = ints(g, tokens, cols), ints(g, 2 * ffn, dtype=torch.float32)
    z = x.double() @ decode(codes, scales, block, lv, 2 * ffn, cols).T
    h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, activation=bof4.ACT_NONE, out_dtype=bof4.F32)
    assert int(status.item()) == 0 and h.dtype == torch.float32 and h.shape == (tokens, ffn)
    assert torch.equal(h, (z[:, :ffn] * z[:, ffn:]).float())
    z = z + bias.double()
    want = (torch.clamp(z[:, :ffn], min=0) * z[:, ffn:]).float()
    pre = torch.full((tokens, 2 * ffn), 9.0, dtype=torch.bfloat16, device="cuda")
    h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, bias=bias, activation=bof4.ACT_RELU, out_dtype=bof4.F32, pre=pre)
    assert int(status.item()) == 0 and torch.equal(h, want) and torch.equal(pre, z.bfloat16())
    h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, bias=bias.bfloat16(), activation=bof4.ACT_RELU)
    assert int(status.item()) == 0 and torch.equal(h, want.bfloat16())


@pytest.mark.parametrize("tokens,ffn,cols,block", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_integer_gradients_are_exact(bof4, tokens, ffn, cols, block, dtype):
    lv, codes, scales = integer_case(2 * ffn, cols, block, ffn + cols)
    g = torch.Generator().manual_seed(tokens)
    dh, pre = ints(g, tokens, ffn, dtype=dtype), ints(g, tokens, 2 * ffn)
    w = decode(codes, scales, block, lv, 2 * ffn, cols)
    gate, up, d = pre[:, :ffn].double(), pre[:, ffn:].double(), dh.double()
    for act, a, slope in ((bof4.ACT_NONE, gate, torch.ones_like(gate)), (bof4.ACT_RELU, torch.clamp(gate, min=0), (gate > 0).double())):
        dz = torch.cat((d * up * slope, d * a), dim=1)
        dx, db, status = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre, activation=act, want_dbias=True)
        assert int(status.item()) == 0 and dx.dtype == torch.bfloat16 and db.shape == (2 * ffn,)
        assert torch.equal(dx, (dz @ w).float().bfloat16())
        assert torch.equal(db.double(), dz.sum(0))
    dx, db, status = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre, activation=act, want_dx=False, want_dbias=True)
    assert dx is None and int(status.item()) == 0 and torch.equal(db.double(), dz.sum(0))


def bounds(z, mag, ffn, act):
    d = 2.0 ** -14 * mag
    a, _ = act64(z[:, :ffn], act)
    gate = 1.13 * d[:, :ffn] + 2.0 ** -20 * torch.clamp(z[:, :ffn].abs(), min=1)
    return a * z[:, ffn:], gate * (z[:, ffn:].abs() + d[:, ffn:]) + a.abs() * d[:, ffn:]


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("tokens", [1, 12, 40, 200, 900])
def test_activations(bof4, act, tokens):
    ffn, cols, block = 520, 1024, 64
    lv, codes, scales = real_case(2 * ffn, cols, block, 3)
    g = torch.Generator().manual_seed(tokens)
    x, bias = torch.randn(tokens, cols, generator=g).bfloat16().cuda(), torch.randn(2 * ffn, generator=g).cuda()
    w = decode(codes, scales, block, lv, 2 * ffn, cols)
    z, mag = x.double() @ w.T + bias.double(), x.double().abs() @ w.abs().T + bias.double().abs()
    want, tol = bounds(z, mag, ffn, act)
    for out_dtype, half in ((bof4.F32, 2.0 ** -24), (bof4.BF16, 2.0 ** -8)):
        pre = torch.empty(tokens, 2 * ffn, dtype=torch.bfloat16, device="cuda")
        h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, bias=bias, activation=act_code(bof4, act), out_dtype=out_dtype, pre=pre)
        assert int(status.item()) == 0
        assert bool(((h.double() - want).abs() <= tol + half * (want.abs() + tol)).all())
        assert bool(((pre.double() - z).abs() <= 2.0 ** -14 * mag + 2.0 ** -8 * z.abs() + 2.0 ** -20).all())
    dh = torch.randn(tokens, ffn, generator=g).cuda()
    a, slope = act64(pre[:, :ffn].double(), act)
    dz = torch.cat((dh.double() * pre[:, ffn:].double() * slope, dh.double() * a), dim=1)
    dx, db, status = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre, activation=act_code(bof4, act), want_dbias=True)
    assert int(status.item()) == 0
    # terms: rounding of dz, the activation within 2^-20 of max(|z|, 1) and its slope within 2^-20
    off = torch.cat((dh.double() * pre[:, ffn:].double(), dh.double() * torch.clamp(pre[:, :ffn].double().abs(), min=1)), dim=1).abs() * 2.0 ** -19
    tol = (dz.abs() * (2.0 ** -8 + 2.0 ** -13) + off) @ w.abs()
    assert bool(((dx.double() - dz @ w).abs() <= tol + 2.0 ** -8 * ((dz @ w).abs() + tol)).all())
    assert bool(((db.double() - dz.sum(0)).abs() <= off.sum(0) + 2.0 ** -20 * dz.abs().sum(0)).all())


@pytest.mark.parametrize("tokens,ffn,cols,block,count", [(1, 64, 64, 64, 1), (4, 65, 512, 64, 700), (15, 128, 256, 32, 20000), (40, 150, 1024, 128, 300),
                                                          (200, 257, 2048, 64, 5000), (800, 100, 96, 32, 9000)])
def test_outliers_replace_their_weights(bof4, tokens, ffn, cols, block, count):
    rows = 2 * ffn
    lv, codes, scales = integer_case(rows, cols, block, 5)
    lst = outlier_list(rows * cols, count, 7, integers=True, spare=9)
    g = torch.Generator().manual_seed(tokens)
    x, dh, pre = ints(g, tokens, cols), ints(g, tokens, ffn), ints(g, tokens, rows)
    w = decode(codes, scales, block, lv, rows, cols, lst)
    z = x.double() @ w.T
    h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, activation=bof4.ACT_RELU, out_dtype=bof4.F32, outliers=lst)
    assert int(status.item()) == 0 and torch.equal(h, (torch.clamp(z[:, :ffn], min=0) * z[:, ffn:]).float())
    dx, _, status = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre, activation=bof4.ACT_NONE, outliers=lst)
    dz = torch.cat((dh.double() * pre[:, ffn:].double(), dh.double() * pre[:, :ffn].double()), dim=1)
    assert int(status.item()) == 0 and torch.equal(dx, (dz @ w).float().bfloat16())


@pytest.mark.parametrize("tokens", [1, 6, 16, 50, 300, 800])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_strides_and_what_lies_beside(bof4, tokens, offset):
    """Rows apart from one another, outputs that begin anywhere: what is not the output's stays as it was."""
    ffn, cols, block = 75, 320, 64
    lv, codes, scales = integer_case(2 * ffn, cols, block, 11)
    g = torch.Generator().manual_seed(tokens)
    x = torch.zeros(tokens, cols + 24, dtype=torch.bfloat16, device="cuda")
    x[:, 8:8 + cols] = ints(g, tokens, cols)
    x = x[:, 8:8 + cols]
    z = x.double() @ decode(codes, scales, block, lv, 2 * ffn, cols).T
    want = (z[:, :ffn] * z[:, ffn:]).float()
    for dtype, out_dtype in ((torch.bfloat16, bof4.BF16), (torch.float32, bof4.F32)):
        wide = torch.full((tokens, ffn + 13), 5.0, dtype=dtype, device="cuda")
        kept = torch.full((tokens, 2 * ffn + 11), 7.0, dtype=torch.bfloat16, device="cuda")
        out, pre = wide[:, offset:offset + ffn], kept[:, offset:offset + 2 * ffn]
        h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, activation=bof4.ACT_NONE, out_dtype=out_dtype, pre=pre, out=out)
        assert h is out and int(status.item()) == 0 and torch.equal(out, want.to(dtype)) and torch.equal(pre, z.bfloat16())
        assert bool((wide[:, :offset] == 5).all()) and bool((wide[:, offset + ffn:] == 5).all())
        assert bool((kept[:, :offset] == 7).all()) and bool((kept[:, offset + 2 * ffn:] == 7).all())
    dh = torch.zeros(tokens, ffn + 9, device="cuda")[:, offset:offset + ffn]
    dh.copy_(ints(g, tokens, ffn, dtype=torch.float32))
    pre.copy_(ints(g, tokens, 2 * ffn))
    wide = torch.full((tokens, cols + 13), 5.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, offset:offset + cols]
    dz = torch.cat((dh.double() * pre[:, ffn:].double(), dh.double() * pre[:, :ffn].double()), dim=1)
    dx, _, status = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre, activation=bof4.ACT_NONE, out=out)
    assert dx is out and int(status.item()) == 0
    assert torch.equal(out, (dz @ decode(codes, scales, block, lv, 2 * ffn, cols)).float().bfloat16())
    assert bool((wide[:, :offset] == 5).all()) and bool((wide[:, offset + cols:] == 5).all())


@pytest.mark.parametrize("tokens", [1, 5, 100, 900])
def test_nothing_to_do(bof4, tokens):
    lv, codes, scales = integer_case(2 * 64, 64, 64, 1)
    empty = codes[:0], scales[:0]
    bf = lambda *s: torch.ones(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    h, status = bof4.bof4_gated(codes, scales, 64, 64, 64, lv, bf(0, 64))
    assert h.shape == (0, 64) and int(status.item()) == 0
    h, status = bof4.bof4_gated(*empty, 0, 64, 64, lv, bf(tokens, 64))
    assert h.shape == (tokens, 0) and int(status.item()) == 0
    bias = torch.arange(8.0, device="cuda") - 3
    h, status = bof4.bof4_gated(*empty, 4, 0, 64, lv, bf(tokens, 0), bias=bias, activation=bof4.ACT_RELU, out_dtype=bof4.F32)
    assert int(status.item()) == 0 and torch.equal(h, (torch.clamp(bias[:4], min=0) * bias[4:]).expand(tokens, 4))
    dx, db, status = bof4.bof4_gated_backward(codes, scales, 64, 64, 64, lv, bf(0, 64), bf(0, 128), want_dbias=True)
    assert dx.shape == (0, 64) and int(status.item()) == 0 and not bool(db.any())
    dx, db, status = bof4.bof4_gated_backward(*empty, 0, 64, 64, lv, bf(tokens, 0), bf(tokens, 0))
    assert dx.shape == (tokens, 64) and not bool(dx.any()) and int(status.item()) == 0


@pytest.mark.parametrize("tokens", [1, 9, 40, 300, 900])
def test_what_is_not_finite_stays_where_it_is(bof4, tokens):
    """A token with NaN and one with infinity, a gate row and an up row with such constants: no other token's or column's results change."""
    ffn, cols, block = 100, 128, 64
    lv, codes, scales = integer_case(2 * ffn, cols, block, 2, torch.float32)
    g = torch.Generator().manual_seed(tokens)
    x = ints(g, tokens, cols)
    plain, _ = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, activation=bof4.ACT_SILU, out_dtype=bof4.F32)
    s = scales.clone().view(2 * ffn, 2)
    s[17, 1], s[ffn + 40, 0] = float("nan"), float("inf")
    y = x.clone()
    if tokens > 1:
        y[tokens - 1, 5] = float("nan")
    h, status = bof4.bof4_gated(codes, s.view(-1), ffn, cols, block, lv, y, activation=bof4.ACT_SILU, out_dtype=bof4.F32)
    assert int(status.item()) == 0
    columns = [f for f in range(ffn) if f not in (17, 40)]
    rows = max(1, tokens - 1)
    assert torch.equal(h[:rows, columns], plain[:rows, columns])
    assert bool(h[:, 17].isnan().all()) and (tokens == 1 or bool(h[-1].isnan().all()))
    pre, dh = ints(g, tokens, 2 * ffn), ints(g, tokens, ffn)
    clean, _, _ = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre)
    if tokens > 1:
        dh[tokens - 1, 3] = float("nan")
        dx, db, status = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre, want_dbias=True)
        assert int(status.item()) == 0 and torch.equal(dx[:-1], clean[:-1]) and bool(dx[-1].isnan().all())
        assert sorted(torch.nonzero(db.isnan())[:, 0].tolist()) == [3, ffn + 3]


@pytest.mark.parametrize("tokens", [3, 40, 900])
def test_streams_graphs_and_workspaces(bof4, tokens):
    """On another stream, twice the same bits, captured and replayed with other inputs, two graphs of one workspace in turn, a workspace of any contents."""
    ffn, cols, block = 300, 512, 64
    lv, codes, scales = real_case(2 * ffn, cols, block, 9)
    g = torch.Generator().manual_seed(1)
    xs = [torch.randn(tokens, cols, generator=g).bfloat16().cuda() for _ in range(3)]
    pres = [torch.randn(tokens, 2 * ffn, generator=g).bfloat16().cuda() for _ in range(3)]
    dhs = [torch.randn(tokens, ffn, generator=g).cuda() for _ in range(3)]
    levels = torch.from_numpy(LV).cuda()
    fw = torch.full((bof4.bof4_gated_workspace_bytes(ffn, cols, tokens),), 255, dtype=torch.uint8, device="cuda")
    bw = torch.full((bof4.bof4_gated_workspace_bytes(ffn, cols, tokens, True),), 255, dtype=torch.uint8, device="cuda")
    forward = lambda x, **kw: bof4.bof4_gated(codes, scales, ffn, cols, block, levels, x, **kw)  # noqa: E731
    backward = lambda dh, pre, **kw: bof4.bof4_gated_backward(codes, scales, ffn, cols, block, levels, dh, pre, want_dbias=True, **kw)  # noqa: E731
    want = [(forward(x)[0], *backward(dh, pre)[:2]) for x, dh, pre in zip(xs, dhs, pres)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [(forward(x, workspace=fw)[0], *backward(dh, pre, workspace=bw)[:2]) for x, dh, pre in zip(xs, dhs, pres)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for u, v in zip(want, again) for a, b in zip(u, v))
    x, dh, pre = xs[0].clone(), dhs[0].clone(), pres[0].clone()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            h, s1 = forward(x, workspace=fw)
            dx, db, s2 = backward(dh, pre, workspace=bw)
        graphs.append(graph)
        outs.append((h, dx, db, s1, s2))
    for k in (1, 2, 0, 1):
        x.copy_(xs[k]), dh.copy_(dhs[k]), pre.copy_(pres[k])
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out[:3], want[k])) and int(out[3].item()) == 0 and int(out[4].item()) == 0


@pytest.mark.parametrize("tokens", [2, 60, 1000])
def test_two_calls_at_once(bof4, tokens):
    """On two streams, with workspaces of their own, in turn: what one computes is none of the other's."""
    ffn, cols, block = 1200, 1024, 64
    lv, codes, scales = real_case(2 * ffn, cols, block, 4)
    levels = torch.from_numpy(lv).cuda()
    g = torch.Generator().manual_seed(3)
    xs = [torch.randn(tokens, cols, generator=g).bfloat16().cuda() for _ in range(2)]
    dhs = [torch.randn(tokens, ffn, generator=g).bfloat16().cuda() for _ in range(2)]

    def call(k):
        pre = torch.empty(tokens, 2 * ffn, dtype=torch.bfloat16, device="cuda")
        h, s1 = bof4.bof4_gated(codes, scales, ffn, cols, block, levels, xs[k], pre=pre)
        dx, db, s2 = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, levels, dhs[k], pre, want_dbias=True)
        return h, pre, dx, db, s1, s2

    want = [call(0), call(1)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(10):
        for k, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got.append((k, call(k)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k, out in got for a, b in zip(out, want[k]))


def test_gradient_against_differences(bof4):
    """dx against central differences of the block itself in fp32, summed with weights: a step e leaves e^2 / 6 times the third derivative and
    the roundings 2^-14 mag / e; values are chosen so that both stay below 2^-7 of the gradient's norm."""
    tokens, ffn, cols, block = 40, 64, 64, 64
    lv, codes, scales = real_case(2 * ffn, cols, block, 21)
    g = torch.Generator().manual_seed(5)
    x, c = torch.randn(tokens, cols, generator=g).bfloat16().cuda(), torch.randn(tokens, ffn, generator=g).cuda()
    pre = torch.empty(tokens, 2 * ffn, dtype=torch.bfloat16, device="cuda")
    bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, pre=pre)
    dx, _, _ = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, c, pre)
    diff = torch.empty(tokens, cols, device="cuda", dtype=torch.float64)
    for k in range(cols):
        step = torch.zeros_like(x)
        step[:, k] = 2.0 ** -4
        up, down = (x + step).bfloat16(), (x - step).bfloat16()  # rounded: the step is what the two differ by
        f = [(bof4.bof4_gated(codes, scales, ffn, cols, block, lv, v, out_dtype=bof4.F32)[0].double() * c.double()).sum(1) for v in (up, down)]
        diff[:, k] = (f[0] - f[1]) / (up[:, k].double() - down[:, k].double())
    assert float((dx.double() - diff).norm() / diff.norm()) <= 2.0 ** -6


def test_refusals(bof4):
    lv, codes, scales = integer_case(2 * 64, 128, 64, 1)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    good = dict(codes=codes, scales=scales, ffn=64, cols=128, block_size=64, levels=lv, x=bf(4, 128))
    bof4.bof4_gated(**good)
    for kw in (dict(ffn=63), dict(ffn=-64), dict(ffn=1 << 40), dict(x=bf(4, 64)), dict(x=bf(128)), dict(bias=torch.zeros(64, device="cuda")), dict(pre=bf(4, 64)),
               dict(out=bf(4, 128)), dict(out_dtype=7), dict(x=bf(4, 256)[:, ::2]), dict(workspace=torch.zeros(4096, device="cuda")), dict(x=torch.zeros(4, 128, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            bof4.bof4_gated(**{**good, **kw})
    for kw in (dict(x=bf(4, 128).float()), dict(pre=torch.zeros(4, 128, device="cuda")), dict(scales=scales.half())):
        with pytest.raises(TypeError):
            bof4.bof4_gated(**{**good, **kw})
    for kw in (dict(activation=9), dict(block_size=16, scales=scales.repeat(4)), dict(x=bf(4 * 132 + 1)[:4 * 132].view(4, 132)[:, :128]),
               dict(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(bof4.Bof4Error):
            bof4.bof4_gated(**{**good, **kw})
    good = dict(codes=codes, scales=scales, ffn=64, cols=128, block_size=64, levels=lv, dh=bf(4, 64), pre=bf(4, 128))
    bof4.bof4_gated_backward(**good)
    for kw in (dict(dh=bf(4, 128)), dict(pre=bf(4, 64)), dict(pre=bf(5, 128)), dict(out=bf(4, 64))):
        with pytest.raises(ValueError):
            bof4.bof4_gated_backward(**{**good, **kw})
    with pytest.raises(TypeError):
        bof4.bof4_gated_backward(**{**good, "pre": torch.zeros(4, 128, device="cuda")})
    with pytest.raises(bof4.Bof4Error):
        bof4.bof4_gated_backward(**{**good, "activation": -1})


@pytest.mark.parametrize("tokens", [3, 40, 800])
def test_offsets_beyond_32_bits(bof4, tokens):
    """More than 2^32 weights: codes, constants, the decoded matrix and z.  x and dh have a few values that are not zero, so that the reference needs a few columns
    and rows of the matrix only."""
    ffn, cols, block = 68000, 32768, 1024
    g = torch.Generator(device="cuda").manual_seed(tokens)
    lv = ((torch.arange(16) - 7.5) / 8).tolist()
    codes = torch.randint(0, 256, (ffn * cols,), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(0, 3, (2 * ffn * cols // block,), generator=g, device="cuda").bfloat16() - 1
    level = torch.tensor(lv, device="cuda", dtype=torch.float64)

    def part(rows, columns):
        byte = codes.view(2 * ffn, cols // 2)[rows][:, columns // 2]
        code = torch.where(columns % 2 == 0, byte >> 4, byte & 15)
        return level[code.long()] * scales.view(2 * ffn, cols // block)[rows][:, columns // block].double()

    columns = torch.tensor([0, 1, 777, 16385, 32767], device="cuda")
    x = torch.zeros(tokens, cols, dtype=torch.bfloat16, device="cuda")
    x[:, columns] = torch.randint(-2, 3, (tokens, 5), generator=g, device="cuda").bfloat16()
    z = x[:, columns].double() @ part(torch.arange(2 * ffn, device="cuda"), columns).T
    pre = torch.empty(tokens, 2 * ffn, dtype=torch.bfloat16, device="cuda")
    h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, activation=bof4.ACT_NONE, out_dtype=bof4.F32, pre=pre)
    assert int(status.item()) == 0 and torch.equal(h, (z[:, :ffn] * z[:, ffn:]).float()) and torch.equal(pre, z.bfloat16())
    del h, z, pre
    rows = torch.tensor([0, 5, 33333, 67999], device="cuda")
    dh, pre = torch.zeros(tokens, ffn, device="cuda"), torch.zeros(tokens, 2 * ffn, dtype=torch.bfloat16, device="cuda")
    dh[:, rows] = torch.randint(-2, 3, (tokens, 4), generator=g, device="cuda").float()
    both = torch.cat((rows, rows + ffn))
    pre[:, both] = torch.randint(-2, 3, (tokens, 8), generator=g, device="cuda").bfloat16()
    dz = dh[:, rows].double().repeat(1, 2) * pre[:, both].double().roll(4, 1)
    dx, _, status = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre, activation=bof4.ACT_NONE)
    assert int(status.item()) == 0 and torch.equal(dx, (dz @ part(both, torch.arange(cols, device="cuda"))).bfloat16())
