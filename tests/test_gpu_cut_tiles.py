"""Products with a decoded matrix whose last tiles are cut along K: the gated block (rows that begin at multiples of 32 bytes and others), its gradient and the
logits of the loss.  Whether tiles are cut is read off the size of the workspace, so that a case cannot come to test something else."""
import pytest
import torch

from test_gpu_cross_entropy import check, targets_of
from test_gpu_gated import LV, bof4, decode, integer_case, ints, outlier_list, real_case  # noqa: F401

pytestmark = pytest.mark.gpu


def cut(bof4, ffn, cols, tokens, backward=False):  # noqa: F811
    """Bytes of the workspace that are neither the decoded matrix nor dz: a product without cut tiles has next to none."""
    up256 = lambda v: (v + 255) // 256 * 256  # noqa: E731
    rest = bof4.bof4_gated_workspace_bytes(ffn, cols, tokens, backward) - up256(4 * ffn * cols)
    if backward:
        rest -= up256(2 * tokens * ((2 * ffn + 7) // 8 * 8)) + up256((tokens + 7) // 8 * 8 * ffn)  # (at most: sums of dz of eight tokens)
    assert rest > -(1 << 22)
    return rest > 1 << 18


# forward: left-over tiles of 256 tokens by 256 rows (gate and up) on 74 pairs of SMs, K of at least 96 blocks of 64
SHAPES = [(800, 300, 8192, 64), (800, 301, 8192, 64), (768, 128, 6144, 64), (1025, 2400, 8192, 64), (769, 1111, 10240, 1024), (2049, 1072, 6176, 32)]


@pytest.mark.parametrize("tokens,ffn,cols,block", SHAPES)
def test_gated_blocks_are_exact(bof4, tokens, ffn, cols, block):  # noqa: F811
    assert cut(bof4, ffn, cols, tokens)
    lv, codes, scales = integer_case(2 * ffn, cols, block, ffn)
    g = torch.Generator().manual_seed(tokens)
    x, bias = ints(g, tokens, cols), ints(g, 2 * ffn, dtype=torch.float32)
    lst = outlier_list(2 * ffn * cols, 5000, 7, integers=True)
    z = x.double() @ decode(codes, scales, block, lv, 2 * ffn, cols, lst).T + bias.double()
    want = (torch.clamp(z[:, :ffn], min=0) * z[:, ffn:]).float()
    for out_dtype, kept in ((bof4.F32, False), (bof4.F32, True), (bof4.BF16, True)):
        pre = torch.full((tokens, 2 * ffn), 9.0, dtype=torch.bfloat16, device="cuda") if kept else None
        h, status = bof4.bof4_gated(codes, scales, ffn, cols, block, lv, x, bias=bias, activation=bof4.ACT_RELU, out_dtype=out_dtype, pre=pre, outliers=lst)
        assert int(status.item()) == 0 and torch.equal(h, want.to(h.dtype)) and (not kept or torch.equal(pre, z.bfloat16()))


@pytest.mark.parametrize("tokens,ffn,cols,block", [(1000, 4000, 96, 32), (900, 3333, 512, 64), (1200, 3100, 1088, 64)])
def test_gradients_are_exact(bof4, tokens, ffn, cols, block):  # noqa: F811
    assert cut(bof4, ffn, cols, tokens, True)
    lv, codes, scales = integer_case(2 * ffn, cols, block, ffn)
    g = torch.Generator().manual_seed(tokens)
    dh, pre = ints(g, tokens, ffn), ints(g, tokens, 2 * ffn)
    w = decode(codes, scales, block, lv, 2 * ffn, cols)
    dz = torch.cat((dh.double() * pre[:, ffn:].double(), dh.double() * pre[:, :ffn].double()), dim=1)
    dx, _, status = bof4.bof4_gated_backward(codes, scales, ffn, cols, block, lv, dh, pre, activation=bof4.ACT_NONE)
    assert int(status.item()) == 0 and torch.equal(dx, (dz @ w).float().bfloat16())


@pytest.mark.parametrize("tokens,rows,cols,block", [(800, 700, 8192, 64), (769, 1300, 6144, 64), (1000, 33000, 8192, 128), (1000, 4700, 10240, 1024)])
def test_losses(bof4, tokens, rows, cols, block):  # noqa: F811
    """A piece's logits are the product of a gated block of as many rows (33000 rows are two pieces, of which the second has cut tiles)."""
    pieces = -(-rows // 32768)
    piece = (-(-rows // pieces) + 255) // 256 * 256
    assert any(cut(bof4, (min(piece, rows - k * piece) + 255) // 256 * 128, cols, tokens) for k in range(pieces))
    case = integer_case(rows, cols, block, rows)
    g = torch.Generator().manual_seed(tokens)
    x = ints(g, tokens, cols) * (torch.arange(cols, device="cuda") % (cols // 16) == 0)
    check(bof4, case, rows, cols, block, x, targets_of(tokens, rows, tokens), torch.rand(tokens, generator=g).cuda())


@pytest.mark.parametrize("tokens,ffn,cols", [(800, 300, 8192), (800, 301, 8192)])
def test_graphs_and_other_streams(bof4, tokens, ffn, cols):  # noqa: F811
    """Captured and replayed, two graphs of one workspace in turn, the same bits on every way."""
    lv, codes, scales = real_case(2 * ffn, cols, 64, 9)
    levels = torch.from_numpy(LV).cuda()
    g = torch.Generator().manual_seed(1)
    xs = [torch.randn(tokens, cols, generator=g).bfloat16().cuda() for _ in range(2)]
    ys = [targets_of(tokens, 2 * ffn, k) for k in range(2)]
    ws = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (bof4.bof4_gated_workspace_bytes(ffn, cols, tokens),
                                                                           bof4.bof4_cross_entropy_workspace_bytes(2 * ffn, cols, tokens, True))]

    def call(x, y, spaces=(None, None)):
        h, s1 = bof4.bof4_gated(codes, scales, ffn, cols, 64, levels, x, workspace=spaces[0])
        return (h, s1, *bof4.bof4_cross_entropy(codes, scales, 2 * ffn, cols, 64, levels, x, y, want_dx=True, workspace=spaces[1]))

    want = [call(x, y) for x, y in zip(xs, ys)]
    x, y, graphs, outs = xs[0].clone(), ys[0].clone(), [], []
    torch.cuda.synchronize()
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(x, y, ws))
        graphs.append(graph)
    for k in (1, 0, 1):
        x.copy_(xs[k]), y.copy_(ys[k])
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want[k]))
