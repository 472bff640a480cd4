"""Results in fp32 whose accumulators take a segment of K at a time: tiles that one CTA has whole and tiles that several share, one, two and four accumulators, sums that
are exact whatever their order."""
import pytest
import torch

from test_gpu_cross_entropy import check, targets_of
from test_gpu_gated import LV, bof4, decode, integer_case, ints, outlier_list, real_case  # noqa: F401

pytestmark = pytest.mark.gpu

# more tiles of 128 rows than SMs, and fewer; K a little above a segment, two and several of them
SHAPES = [(200, 10240, 2080, 32), (131, 9473, 1088, 64), (257, 9600, 4160, 64), (384, 10240, 4096, 64), (100, 9600, 4160, 64), (40, 9600, 8256, 64), (24, 9999, 12352, 64),
          (200, 700, 8192, 64), (100, 333, 8192, 64), (300, 2100, 4096, 128), (129, 64, 12352, 64), (64, 1500, 12288, 1024)]


@pytest.mark.parametrize("tokens,ffn,cols,block", SHAPES)
@pytest.mark.parametrize("listed", [False, True])
def test_gated_blocks_are_exact(bof4, tokens, ffn, cols, block, listed):  # noqa: F811
    lv, codes, scales = integer_case(2 * ffn, cols, block, ffn, torch.float32 if listed else torch.bfloat16)
    g = torch.Generator().manual_seed(tokens)
    x, bias = ints(g, tokens, cols), ints(g, 2 * ffn, dtype=torch.float32)
    lst = outlier_list(2 * ffn * cols, 5000, 7, integers=True) if listed else None
    z = x.double() @ decode(codes, scales, block, lv, 2 * ffn, cols, lst).T + bias.double()
    want = (torch.clamp(z[:, :ffn], min=0) * z[:, ffn:]).float()
    wide = torch.full((tokens, ffn + 5), 5.0, device="cuda")
    for out, kept in ((None, False), (wide[:, 3:3 + ffn], True)):
        pre = torch.full((tokens, 2 * ffn), 9.0, dtype=torch.bfloat16, device="cuda") if kept else None
        h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, bias=bias, activation=bof4.ACT_RELU, out_dtype=bof4.F32, pre=pre, outliers=lst, out=out)
        assert int(status.item()) == 0 and torch.equal(h, want) and (not kept or torch.equal(pre, z.bfloat16()))
    assert bool((wide[:, :3] == 5).all()) and bool((wide[:, 3 + ffn:] == 5).all())


@pytest.mark.parametrize("tokens,rows,cols,block", [(200, 20480, 4160, 64), (100, 30001, 4160, 64), (40, 20000, 8256, 64), (300, 19999, 4096, 64), (130, 1000, 8192, 64), (384, 3333, 12288, 64)])
def test_losses(bof4, tokens, rows, cols, block):  # noqa: F811
    """(With the gradient from 257 tokens on in another form.)"""
    case = integer_case(rows, cols, block, rows)
    g = torch.Generator().manual_seed(tokens)
    x = ints(g, tokens, cols) * (torch.arange(cols, device="cuda") % (cols // 16) == 0)
    check(bof4, case, rows, cols, block, x, targets_of(tokens, rows, tokens), torch.rand(tokens, generator=g).cuda())


@pytest.mark.parametrize("tokens,ffn,cols", [(200, 10240, 2304), (150, 400, 8192)])
def test_the_same_bits_again(bof4, tokens, ffn, cols):  # noqa: F811
    """On two streams at once, and captured with a workspace that another graph shares."""
    lv, codes, scales = real_case(2 * ffn, cols, 64, 9)
    levels = torch.from_numpy(LV).cuda()
    g = torch.Generator().manual_seed(1)
    xs = [torch.randn(tokens, cols, generator=g).bfloat16().cuda() for _ in range(2)]
    call = lambda x, ws=None: bof4.bof4_gated(codes, scales, ffn, cols, 64, levels, x, out_dtype=bof4.F32, workspace=ws)[0]  # noqa: E731
    want = [call(x) for x in xs]
    assert not torch.equal(want[0], want[1])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(5):
        for k, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got.append((k, call(xs[k])))
    torch.cuda.synchronize()
    assert all(torch.equal(h, want[k]) for k, h in got)
    ws = torch.full((bof4.bof4_gated_workspace_bytes(ffn, cols, tokens),), 255, dtype=torch.uint8, device="cuda")
    x, graphs, outs = xs[0].clone(), [], []
    torch.cuda.synchronize()
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(x, ws))
        graphs.append(graph)
    for k in (1, 0, 1):
        x.copy_(xs[k])
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[k])
