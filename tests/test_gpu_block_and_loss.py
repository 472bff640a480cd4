"""The operators of a model's last layers as they are used together: gated block, down projection with the residual, vocabulary loss, and back, through
torch.autograd.Function, against the same layers in 64 bits on the dequantised weights."""
import numpy as np
import pytest
import torch

from test_gpu_linear import LV, act64, act_code, decode

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bof4():
    import __graft_entry__ as entry
    entry.build()
    import paper_2505_06653_b200 as m
    return m


def quantised(bof4, rows, cols, block, seed, opq):
    """A matrix as a user has it: quantised by the library, with its outliers kept or without."""
    w = (torch.randn(rows * cols, generator=torch.Generator().manual_seed(seed)) * cols ** -0.5).bfloat16().cuda()
    if not opq:
        codes, scales = bof4.bof4_quantize(w, block, bof4.NORM_SIGNED, LV)
        return codes, scales, None
    tau = float(np.float32(bof4.bof4_opq_threshold(0.95, block)))
    codes, scales, *lst = bof4.bof4_quantize_opq(w, block, bof4.NORM_SIGNED, LV, tau, rows * cols // 8)
    return codes, scales, tuple(lst)


@pytest.mark.parametrize("tokens", [1, 7, 40, 300, 1000])
@pytest.mark.parametrize("act,opq", [("silu", False), ("gelu", True)])
def test_a_step_of_training(bof4, tokens, act, opq):
    """x -> x + down(gated(x)) -> mean loss, with the gradient of x.  Roundings to bf16, as 2-norms of what they change: h, y (2^-9 each on the mean, 2^-8 at most), the
    probabilities, dy, dh, dz and dx; eight of them in a row, each passed on by matrices of norm near one, stay below 8 * 2^-8 of the gradient's norm, and the losses, whose
    logits are off by two roundings of y along rows of norm near one (logits of size 1 to 3), below 2^-7 each."""
    hidden, ffn, vocab, block = 256, 640, 1900, 64
    up, down, head = (quantised(bof4, r, c, block, k, opq) for k, (r, c) in enumerate(((2 * ffn, hidden), (hidden, ffn), (vocab, hidden))))
    levels, code = torch.from_numpy(LV).cuda(), act_code(bof4, act)
    g = torch.Generator().manual_seed(tokens)
    targets = torch.randint(0, vocab, (tokens,), generator=g)
    targets[torch.rand(tokens, generator=g) < 0.2] = -100
    targets[0] = 3
    targets = targets.cuda()
    counted = (targets >= 0).sum()

    class Layers(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            pre = torch.empty(tokens, 2 * ffn, dtype=torch.bfloat16, device="cuda")
            h, s1 = bof4.bof4_gated(*up[:2], ffn, hidden, block, levels, x, activation=code, pre=pre, outliers=up[2])
            y, s2 = bof4.bof4_linear(*down[:2], hidden, ffn, block, levels, h, residual=x, outliers=down[2])
            loss, lse, dy, s3 = bof4.bof4_cross_entropy(*head[:2], vocab, hidden, block, levels, y, targets, dloss=(1.0 / counted.float()).expand(tokens).contiguous(),
                                                        want_dx=True, outliers=head[2])
            ctx.save_for_backward(pre, dy)
            assert not any(int(s.item()) for s in (s1, s2, s3))
            return loss.sum() / counted, loss

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, d, _):
            pre, dy = ctx.saved_tensors
            dy = (dy * d).bfloat16()
            dh, _, s1 = bof4.bof4_linear_backward(*down[:2], hidden, ffn, block, levels, dy, outliers=down[2])
            dx, _, s2 = bof4.bof4_gated_backward(*up[:2], ffn, hidden, block, levels, dh, pre, activation=code, outliers=up[2])
            assert int(s1.item()) == 0 and int(s2.item()) == 0
            return dx + dy

    x = torch.randn(tokens, hidden, generator=g).bfloat16().cuda().requires_grad_()
    mean, loss = Layers.apply(x)
    mean.backward()
    a = x.detach().double().requires_grad_()
    wu, wd, wh = (decode(m[0], m[1], block, LV, r, c, m[2]) for m, (r, c) in zip((up, down, head), ((2 * ffn, hidden), (hidden, ffn), (vocab, hidden))))
    z = a @ wu.T
    gate = torch.nn.functional.silu(z[:, :ffn]) if act == "silu" else torch.nn.functional.gelu(z[:, :ffn])
    assert torch.allclose(gate, act64(z[:, :ffn], act)[0])
    y = a + (gate * z[:, ffn:]) @ wd.T
    want = torch.nn.functional.cross_entropy(y @ wh.T, targets, ignore_index=-100, reduction="none")
    (want.sum() / counted).backward()
    assert bool(((loss.detach().double() - want.detach()).abs() <= 2.0 ** -7 * (1 + want.detach().abs())).all())
    assert float((x.grad.double() - a.grad).norm() / a.grad.norm()) <= 8 * 2.0 ** -8
