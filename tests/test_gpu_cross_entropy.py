"""bof4_cross_entropy against a plain implementation in 64 bits (written out here, without the library).

Logits are exact where inputs are small integers and constants powers of two.  Then what is left are the exponentials (relative 2^-22 for each unit
of their argument, 2^-21 more; weighted by the probabilities an argument is below 16 on the mean: 2^-18), sums of fp32 values (2^-18 is more
than all of their roundings) and the logarithm: lse is off by TOL * (1 + |lse|), TOL = 2^-17.  A loss is log(1 + e^b), b = log-sum of the others less the
target's logit: e^b is off by TOL + 2^-22 |b| of itself (the rounding of b, of the sum's reference and exp), the logarithm by TOL of itself.  A probability is off by 2^-17 of itself and is
rounded to bf16 (2^-8), sums of the second product by 2^-14 of the sum of magnitudes, dx is rounded once:
  |dx - exact| <= g (sum_v p_v |W_v| + (1 - p_y) |W_y|) (2^-8 + 2^-13) + 2^-8 |dx|.
Generic inputs: a logit is off by at most d = 2^-14 * sum |w x|, so lse by d, the loss by 2 d and a probability by 2 d of itself."""
import math

import numpy as np
import pytest
import torch

from test_gpu_linear import LV, decode, integer_case, ints, outlier_list, real_case

pytestmark = pytest.mark.gpu
TOL = 2.0 ** -17


@pytest.fixture(scope="module")
def bof4():
    import __graft_entry__ as entry
    entry.build()
    import paper_2505_06653_b200 as m
    assert torch.cuda.is_available()
    return m


def plain(x, w, targets, dloss):
    """loss, lse, dx and the magnitudes that bound dx, in 64 bits.  The target against the others: nothing cancels."""
    x, n, rows = x.double(), torch.arange(len(x), device="cuda"), w.shape[0]
    keep = (targets >= 0) & (targets < rows)
    at = torch.where(keep, targets, 0)
    z = x @ w.T
    lse = torch.logsumexp(z, 1)
    d = z - z[n, at][:, None]
    d[n, at] = -math.inf
    odds = torch.exp(torch.logsumexp(d, 1))
    loss = torch.where(keep, torch.log1p(odds), 0.0)
    most = (TOL + 2.0 ** -22 * torch.log(odds).abs().nan_to_num(0, 0, 0)) * torch.clamp(loss, max=1) + TOL * loss
    p = torch.exp(z - lse[:, None])
    p[n, at] = torch.where(odds.isinf(), -1.0, -odds / (1 + odds))
    p = p * (dloss.double() * keep)[:, None]
    return loss, lse, p @ w, p.abs() @ w.abs(), most


def check(bof4, case, rows, cols, block, x, targets, dloss=None, outliers=None, d=0.0):
    """Both calls, with and without the gradient; d: how far logits may be off, per token."""
    lv, codes, scales = case
    tokens = x.shape[0]
    w = decode(codes, scales, block, lv, rows, cols, outliers)
    loss, lse, dx, mag, most = plain(x, w, targets, torch.ones(tokens, device="cuda") if dloss is None else dloss)
    args = (codes, scales, rows, cols, block, lv, x, targets)
    got = bof4.bof4_cross_entropy(*args, dloss=dloss, want_dx=True, outliers=outliers)
    only = bof4.bof4_cross_entropy(*args, outliers=outliers)
    assert only[2] is None and got[2].shape == (tokens, cols) and got[2].dtype == torch.bfloat16
    status = 2 if bool((targets >= rows).any()) else 0
    for out in (got, only):
        assert int(out[3].item()) == status
        assert out[0].shape == out[1].shape == (tokens,) and out[0].dtype == out[1].dtype == torch.float32
        assert bool(((out[0].double() - loss).abs() <= 2 * d + most).all())
        assert bool(((out[1].double() - lse).abs() <= d + TOL * (1 + lse.abs())).all())
    keep = (targets >= 0) & (targets < rows)
    assert not bool(got[0][~keep].any()) and not bool(got[2][~keep].any())
    far = torch.as_tensor(2 * d).expand(tokens).to("cuda")[:, None]
    assert bool(((got[2].double() - dx).abs() <= mag * (2.0 ** -8 + 2.0 ** -13 + 2 * far) + 2.0 ** -8 * dx.abs()).all())
    return got


def targets_of(tokens, rows, seed, ignored=0.2):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, rows, (tokens,), generator=g)
    t[torch.rand(tokens, generator=g) < ignored] = -100
    if tokens > 3:
        t[0], t[1] = 0, rows - 1
    return t.cuda()


# tokens on both sides of 6, 8, 16, 64, 128, 256 and of the form for many tokens; vocabularies of one row, one chunk, one piece and a little more, tiles cut along K
SHAPES = [(1, 1, 32, 32), (1, 1000, 64, 64), (2, 2049, 256, 64), (7, 333, 4096, 128), (13, 5000, 1024, 1024), (17, 127, 320, 64), (40, 2048, 64, 32), (130, 16385, 96, 32),
          (300, 700, 512, 256), (511, 999, 64, 64), (512, 1000, 96, 32), (513, 16385, 128, 64), (700, 1, 64, 64), (1000, 300, 2080, 32), (1537, 33000, 64, 64),
          (600, 63, 256, 64), (2049, 1025, 512, 64), (1000, 3000, 4096, 64),
          (14, 16400, 4096, 64),
          # more than 64 tokens of the form that decodes as it multiplies
          (130, 600, 2080, 32), (250, 300, 2304, 64)]


@pytest.mark.parametrize("tokens,rows,cols,block", SHAPES)
@pytest.mark.parametrize("scale_dtype", [torch.bfloat16, torch.float32])
def test_exact_logits(bof4, tokens, rows, cols, block, scale_dtype):
    """Few columns have an input, so that logits stay within some tens."""
    case = integer_case(rows, cols, block, rows + cols, scale_dtype)
    g = torch.Generator().manual_seed(tokens)
    x = ints(g, tokens, cols) * (torch.arange(cols, device="cuda") % max(1, cols // 16) == 0)
    check(bof4, case, rows, cols, block, x.bfloat16(), targets_of(tokens, rows, tokens), torch.rand(tokens, generator=g).cuda())


@pytest.mark.parametrize("tokens", [1, 5, 60, 300, 800])
def test_generic_logits(bof4, tokens):
    rows, cols, block = 3000, 4096, 64
    case = real_case(rows, cols, block, 3)
    g = torch.Generator().manual_seed(tokens)
    x = (0.25 * torch.randn(tokens, cols, generator=g)).bfloat16().cuda()
    w = decode(case[1], case[2], block, case[0], rows, cols)
    d = 2.0 ** -14 * (x.double().abs() @ w.abs().T).max(dim=1).values
    got = check(bof4, case, rows, cols, block, x, targets_of(tokens, rows, 2, 0.0), d=d)
    # and the sizes of errors that do occur: logits within 2^-17 of their norm, probabilities rounded to bf16 at random
    loss, lse, dx, _, _ = plain(x, w, targets_of(tokens, rows, 2, 0.0), torch.ones(tokens, device="cuda"))
    for a, b, most in ((got[0], loss, 2.0 ** -16), (got[1], lse, 2.0 ** -16), (got[2], dx, 2.0 ** -8)):
        assert float((a.double() - b).norm()) <= most * float(b.norm())


def ramp(rows, values):
    """A vocabulary whose logits are the given values where x is one in its first column: code 15 (level one) there and code 7 (level zero)
    elsewhere, a constant per row."""
    codes = torch.full((rows, 32), 0x77, dtype=torch.uint8)
    codes[:, 0] = 0xf7
    lv = np.array(LV)
    return lv, codes.view(-1).cuda(), torch.as_tensor(values, dtype=torch.float32).cuda()


@pytest.mark.parametrize("tokens", [1, 20, 600])
@pytest.mark.parametrize("kind", ["rising", "falling", "high", "low", "one high", "one low", "alternating", "steps"])
def test_references(bof4, tokens, kind):
    """Logits from -300 to 300 in every order over three pieces: exponentials against a reference neither overflow nor vanish."""
    rows = 40000
    k = torch.arange(rows)
    v = {"rising": k * (600.0 / rows) - 300, "falling": 300 - k * (600.0 / rows), "high": torch.full((rows,), 280.0) + k % 7, "low": torch.full((rows,), -280.0) + k % 7,
         "one high": torch.where(k == 30000, 250.0, -20.0), "one low": torch.where(k == 5, -250.0, 3.0), "alternating": torch.where(k // 64 % 2 == 0, 120.0, -120.0) + k % 3,
         "steps": (k // 4000) * 23.0 - 100}[kind].bfloat16().float()
    lv, codes, scales = ramp(rows, v)
    x = torch.zeros(tokens, 64, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = 1.0
    x[::3, 0] = -1.0
    x[1::5, 0] = 0.5
    g = torch.Generator().manual_seed(3)
    targets = torch.randint(0, rows, (tokens,), generator=g)
    targets[0] = 39001
    if tokens > 2:
        targets[1], targets[2] = 30000 if kind == "one high" else 39500, -1
    targets = targets.cuda()
    z = x[:, :1].double() * v.double().cuda()[None, :]
    n, keep = torch.arange(tokens, device="cuda"), targets >= 0
    at = torch.where(keep, targets, 0)
    lse = torch.logsumexp(z, 1)
    rest = z - z[n, at][:, None]
    rest[n, at] = -math.inf
    rest = torch.logsumexp(rest, 1)
    loss = torch.where(keep, torch.logaddexp(rest, torch.zeros_like(rest)), 0.0)
    got, got_lse, got_dx, status = bof4.bof4_cross_entropy(codes, scales, rows, 64, 64, lv, x, targets, want_dx=True)
    assert int(status.item()) == 0
    assert bool(((got_lse.double() - lse).abs() <= TOL * (1 + lse.abs())).all())
    assert bool(((got.double() - loss).abs() <= (TOL + 2.0 ** -22 * rest.abs()) * torch.clamp(loss, max=1) + TOL * loss + 2.0 ** -100).all())
    # dx has its first column only, the rest of the row being zero levels.  What lies below 2^-126 has no fp32 value: 40000 probabilities that are each
    # off by that, times rows of at most 300, are off by less than 2^-100.
    p = torch.exp(z - lse[:, None])
    p[n, at] = -torch.exp(rest - torch.logaddexp(rest, torch.zeros_like(rest)))
    p = p * keep[:, None]
    w = v.double().cuda()
    exact, mag = p @ w, p.abs() @ w.abs()
    assert bool(((got_dx[:, 0].double() - exact).abs() <= mag * (2.0 ** -8 + 2.0 ** -13) + 2.0 ** -8 * exact.abs() + 2.0 ** -100).all())
    assert not bool(got_dx[:, 1:].any())


@pytest.mark.parametrize("tokens,rows,cols,block,count", [(1, 64, 64, 64, 1), (4, 130, 512, 64, 700), (15, 128, 256, 32, 20000), (200, 257, 2048, 64, 5000),
                                                          (600, 17000, 64, 32, 9000), (900, 512, 96, 32, 49152)])
def test_outliers_replace_their_weights(bof4, tokens, rows, cols, block, count):
    case = integer_case(rows, cols, block, 5)
    lst = outlier_list(rows * cols, count, 7, integers=True, spare=9)
    g = torch.Generator().manual_seed(tokens)
    x = ints(g, tokens, cols) * (torch.arange(cols, device="cuda") % max(1, cols // 16) == 0)
    check(bof4, case, rows, cols, block, x.bfloat16(), targets_of(tokens, rows, 5), outliers=lst)


@pytest.mark.parametrize("tokens", [1, 4, 50, 700])
def test_targets(bof4, tokens):
    """All ignored, the same target everywhere, targets beyond the vocabulary."""
    rows, cols, block = 777, 64, 64
    case = integer_case(rows, cols, block, 1)
    x = ints(torch.Generator().manual_seed(tokens), tokens, cols)
    x[:, 8:] = 0
    for value in (-1, -100, -(1 << 62), 5, rows - 1, rows, 1 << 40, (1 << 32) + 5):
        check(bof4, case, rows, cols, block, x, torch.full((tokens,), value, device="cuda"))
    mixed = torch.full((tokens,), 3, device="cuda")
    mixed[-1] = rows + 9
    check(bof4, case, rows, cols, block, x, mixed, torch.linspace(-2, 2, tokens).cuda())


@pytest.mark.parametrize("tokens", [2, 30, 700])
def test_what_is_not_finite_stays_where_it_is(bof4, tokens):
    rows, cols, block = 300, 64, 64
    lv, codes, scales = integer_case(rows, cols, block, 1)
    x = ints(torch.Generator().manual_seed(tokens), tokens, cols)
    x[:, 8:] = 0
    targets = targets_of(tokens, rows, 1, 0.0)
    plain_out = bof4.bof4_cross_entropy(codes, scales, rows, cols, block, lv, x, targets, want_dx=True)
    y = x.clone()
    y[1, 2] = float("nan")
    got = bof4.bof4_cross_entropy(codes, scales, rows, cols, block, lv, y, targets, want_dx=True)
    rows_left = [t for t in range(tokens) if t != 1]
    assert int(got[3].item()) == 0
    for a, b in zip(got[:3], plain_out[:3]):
        assert torch.equal(a[rows_left], b[rows_left]) and bool(a[1].isnan().all())


@pytest.mark.parametrize("tokens", [1, 12, 100, 600])
@pytest.mark.parametrize("offset", [0, 1])
def test_strides_and_what_lies_beside(bof4, tokens, offset):
    rows, cols, block = 555, 128, 64
    lv, codes, scales = integer_case(rows, cols, block, 4)
    g = torch.Generator().manual_seed(tokens)
    x = torch.zeros(tokens, cols + 24, dtype=torch.bfloat16, device="cuda")
    x[:, 8:16] = ints(g, tokens, 8)
    x = x[:, 8:8 + cols]
    targets, dloss = targets_of(tokens, rows, 1), torch.rand(tokens, generator=g).cuda()
    want = bof4.bof4_cross_entropy(codes, scales, rows, cols, block, lv, x.contiguous(), targets, dloss=dloss, want_dx=True)
    wide = torch.full((tokens, cols + 13), 5.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, offset:offset + cols]
    got = bof4.bof4_cross_entropy(codes, scales, rows, cols, block, lv, x, targets, dloss=dloss, want_dx=True, out=out)
    assert got[2] is out and all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool((wide[:, :offset] == 5).all()) and bool((wide[:, offset + cols:] == 5).all())


@pytest.mark.parametrize("tokens", [1, 40, 700])
def test_streams_graphs_and_workspaces(bof4, tokens):
    rows, cols, block = 18000, 128, 64
    lv, codes, scales = real_case(rows, cols, block, 9)
    g = torch.Generator().manual_seed(1)
    xs = [torch.randn(tokens, cols, generator=g).bfloat16().cuda() for _ in range(3)]
    ys = [targets_of(tokens, rows, k) for k in range(3)]
    levels = torch.from_numpy(LV).cuda()
    ws = torch.full((bof4.bof4_cross_entropy_workspace_bytes(rows, cols, tokens, True),), 255, dtype=torch.uint8, device="cuda")
    call = lambda x, y, **kw: bof4.bof4_cross_entropy(codes, scales, rows, cols, block, levels, x, y, want_dx=True, **kw)  # noqa: E731
    want = [call(x, y) for x, y in zip(xs, ys)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [call(x, y, workspace=ws) for x, y in zip(xs, ys)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for u, v in zip(want, again) for a, b in zip(u, v))
    x, y = xs[0].clone(), ys[0].clone()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call(x, y, workspace=ws)
        graphs.append(graph)
        outs.append(out)
    for k in (1, 2, 0, 1):
        x.copy_(xs[k]), y.copy_(ys[k])
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want[k]))


@pytest.mark.parametrize("tokens", [2, 60, 700])
def test_two_calls_at_once(bof4, tokens):
    """On two streams, with workspaces of their own, in turn."""
    rows, cols, block = 40000, 256, 64
    lv, codes, scales = real_case(rows, cols, block, 4)
    levels = torch.from_numpy(LV).cuda()
    g = torch.Generator().manual_seed(3)
    xs = [torch.randn(tokens, cols, generator=g).bfloat16().cuda() for _ in range(2)]
    ys = [targets_of(tokens, rows, k) for k in range(2)]
    call = lambda k: bof4.bof4_cross_entropy(codes, scales, rows, cols, block, levels, xs[k], ys[k], want_dx=True)  # noqa: E731
    want = [call(0), call(1)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(10):
        for k, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got.append((k, call(k)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k, out in got for a, b in zip(out, want[k]))


def test_nothing_to_do(bof4):
    lv, codes, scales = integer_case(64, 64, 64, 1)
    x = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda")
    loss, lse, dx, status = bof4.bof4_cross_entropy(codes, scales, 64, 64, 64, lv, x, torch.zeros(0, dtype=torch.int64, device="cuda"), want_dx=True)
    assert loss.shape == lse.shape == (0,) and dx.shape == (0, 64) and int(status.item()) == 0


def test_gradient_against_differences(bof4):
    """dx against central differences of the loss along random directions: the loss is smooth, steps of 2^-4 leave less than 2^-6 of the slope."""
    tokens, rows, cols, block = 64, 500, 256, 64
    lv, codes, scales = real_case(rows, cols, block, 6)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(tokens, cols, generator=g).bfloat16().cuda()
    targets = targets_of(tokens, rows, 4, 0.0)
    dx = bof4.bof4_cross_entropy(codes, scales, rows, cols, block, lv, x, targets, want_dx=True)[2].double()
    slopes, diffs = [], []
    for _ in range(8):
        step = (torch.randint(0, 2, (tokens, cols), generator=g).cuda() * 2 - 1) * 2.0 ** -4
        up, down = (x + step).bfloat16(), (x - step).bfloat16()
        f = [bof4.bof4_cross_entropy(codes, scales, rows, cols, block, lv, v, targets)[0].double() for v in (up, down)]
        slopes.append((dx * (up.double() - down.double())).sum(1))
        diffs.append(f[0] - f[1])
    a, b = torch.cat(slopes), torch.cat(diffs)
    assert float((a - b).norm() / b.norm()) <= 2.0 ** -6


def test_refusals(bof4):
    lv, codes, scales = integer_case(64, 128, 64, 1)
    x, y = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    good = dict(codes=codes, scales=scales, rows=64, cols=128, block_size=64, levels=lv, x=x, targets=y)
    bof4.bof4_cross_entropy(**good)
    for kw in (dict(rows=63), dict(rows=-64), dict(targets=y.int()), dict(targets=y[:3]), dict(targets=y.cpu()), dict(targets=y.view(2, 2)), dict(dloss=y), dict(dloss=torch.ones(3, device="cuda")),
               dict(out=x.clone()), dict(out=x[:, :64].clone(), want_dx=True), dict(x=x[:, ::2]), dict(workspace=torch.zeros(4096, device="cuda"))):
        with pytest.raises(ValueError):
            bof4.bof4_cross_entropy(**{**good, **kw})
    with pytest.raises(TypeError):
        bof4.bof4_cross_entropy(**{**good, "x": x.float()})
    for kw in (dict(block_size=16, scales=scales.repeat(4)), dict(rows=0, codes=codes[:0], scales=scales[:0]), dict(cols=0, codes=codes[:0], scales=scales[:0], x=x[:, :0]),
               dict(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(bof4.Bof4Error):
            bof4.bof4_cross_entropy(**{**good, **kw})


@pytest.mark.parametrize("tokens", [3, 40, 500])
def test_offsets_beyond_32_bits(bof4, tokens):
    """More than 2^32 weights.  x has a few values that are not zero, so that the reference needs a few columns for the logits; dx is compared in some."""
    rows, cols, block = 135000, 32768, 1024
    g = torch.Generator(device="cuda").manual_seed(tokens)
    lv = ((torch.arange(16) - 7.5) / 8).tolist()
    codes = torch.randint(0, 256, (rows * cols // 2,), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(0, 3, (rows * cols // block,), generator=g, device="cuda").bfloat16() - 1
    level = torch.tensor(lv, device="cuda", dtype=torch.float64)

    def part(columns):
        byte = codes.view(rows, cols // 2)[:, columns // 2]
        return level[torch.where(columns % 2 == 0, byte >> 4, byte & 15).long()] * scales.view(rows, cols // block)[:, columns // block].double()

    columns = torch.tensor([0, 1, 777, 16385, 32767], device="cuda")
    x = torch.zeros(tokens, cols, dtype=torch.bfloat16, device="cuda")
    x[:, columns] = torch.randint(-2, 3, (tokens, 5), generator=g, device="cuda").bfloat16()
    targets = targets_of(tokens, rows, 3, 0.1)
    targets[0] = rows - 3
    some = torch.cat((columns, torch.arange(9000, 9100, device="cuda"), torch.arange(32700, 32767, device="cuda")))
    w = part(some)
    small = torch.zeros(tokens, len(some), device="cuda")
    small[:, :5] = x[:, columns].float()
    loss, lse, dx, mag, most = plain(small, w, targets, torch.ones(tokens, device="cuda"))
    got = bof4.bof4_cross_entropy(codes, scales, rows, cols, block, lv, x, targets, want_dx=True)
    assert int(got[3].item()) == 0
    assert bool(((got[0].double() - loss).abs() <= most).all()) and bool(((got[1].double() - lse).abs() <= TOL * (1 + lse.abs())).all())
    assert bool(((got[2][:, some].double() - dx).abs() <= mag * (2.0 ** -8 + 2.0 ** -13) + 2.0 ** -8 * dx.abs()).all())


def test_many_tokens(bof4):
    """More than 2^31 exponentials in a piece; three blocks of tokens are compared."""
    tokens, rows, cols, block = 70000, 33000, 32, 32
    case = integer_case(rows, cols, block, 8)
    g = torch.Generator().manual_seed(1)
    x, targets = ints(g, tokens, cols), targets_of(tokens, rows, 6)
    got = bof4.bof4_cross_entropy(case[1], case[2], rows, cols, block, case[0], x, targets, want_dx=True)
    w = decode(case[1], case[2], block, case[0], rows, cols)
    assert int(got[3].item()) == 0
    for at in (0, 40000, 69000):
        t = slice(at, at + 1000)
        loss, lse, dx, mag, most = plain(x[t], w, targets[t], torch.ones(1000, device="cuda"))
        assert bool(((got[0][t].double() - loss).abs() <= most).all()) and bool(((got[1][t].double() - lse).abs() <= TOL * (1 + lse.abs())).all())
        assert bool(((got[2][t].double() - dx).abs() <= mag * (2.0 ** -8 + 2.0 ** -13) + 2.0 ** -8 * dx.abs()).all())
