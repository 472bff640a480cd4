"""bof4_gated_backward where the gradient of x is not wanted: the same sums, out of a workspace without the decoded matrix and dz."""
import pytest
import torch

from test_gpu_gated import bof4, real_case  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,ffn,cols", [(1, 40, 64), (7, 333, 128), (500, 1200, 512), (1000, 4096, 1024)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_bias_gradient_alone(bof4, tokens, ffn, cols, dtype):  # noqa: F811
    lv, codes, scales = real_case(2 * ffn, cols, 64, 3)
    g = torch.Generator().manual_seed(tokens)
    dh, pre = torch.randn(tokens, ffn, generator=g).to(dtype).cuda(), torch.randn(tokens, 2 * ffn, generator=g).bfloat16().cuda()
    args = (codes, scales, ffn, cols, 64, lv, dh, pre)
    _, both, _ = bof4.bof4_gated_backward(*args, want_dbias=True)
    small = bof4.bof4_gated_workspace_bytes(ffn, 0, tokens, True)
    parts = (tokens + 7) // 8   # at most: sums of eight tokens each
    assert small <= 256 + 256 + parts * 2 * ffn * 4
    ws = torch.full((small + 4096,), 0x55, dtype=torch.uint8, device="cuda")
    for space in (None, ws[:small]):
        dx, alone, status = bof4.bof4_gated_backward(*args, want_dx=False, want_dbias=True, workspace=space)
        assert dx is None and int(status.item()) == 0 and torch.equal(alone, both)
    assert bool((ws[small:] == 0x55).all())
    with pytest.raises(bof4.Bof4Error):
        bof4.bof4_gated_backward(*args, want_dx=False, want_dbias=True, workspace=ws[:small - 256])
    with pytest.raises(bof4.Bof4Error):
        bof4.bof4_gated_backward(*args, want_dbias=True, workspace=ws[:small])
