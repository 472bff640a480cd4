"""bof4_linear, bof4_linear_backward and bof4_moe as torch sees them.  They record no autograd graph: a tensor that requires a gradient is
refused while gradients are on, and taken where they are off (inference, or inside a torch.autograd.Function)."""
import numpy as np
import pytest
import torch

LV = (np.arange(16, dtype=np.float32) - 7.5) / 8


@pytest.fixture(scope="module")
def bof4():
    import __graft_entry__ as entry
    entry.build()
    import paper_2505_06653_b200 as m
    return m


def arguments(bof4, device):
    """The three calls with every tensor argument that can require a gradient."""
    g = torch.Generator().manual_seed(1)
    codes = lambda n: torch.randint(0, 256, (n // 2,), generator=g, dtype=torch.uint8).to(device)  # noqa: E731
    scales = lambda n: torch.ones(n // 32, device=device)  # noqa: E731
    rows, cols, tokens = 32, 64, 3
    bf = lambda *s: torch.randn(*s, generator=g).bfloat16().to(device)  # noqa: E731
    lst = (torch.tensor([5], dtype=torch.int32, device=device), bf(1), torch.tensor([1], device=device))
    common = dict(codes=codes(rows * cols), scales=scales(rows * cols), rows=rows, cols=cols, block_size=32, levels=torch.from_numpy(LV).to(device), outliers=lst)
    linear = dict(common, x=bf(tokens, cols), bias=bf(rows), residual=bf(tokens, rows), pre=bf(tokens, rows), out=bf(tokens, rows))
    backward = dict(common, dy=bf(tokens, rows), pre=bf(tokens, rows), activation=bof4.ACT_SILU, out=bf(tokens, cols))
    moe = dict(x=bf(tokens, cols), router=bf(4, cols), gate_up=(codes(4 * 64 * cols), scales(4 * 64 * cols)), down=(codes(4 * 32 * cols), scales(4 * 32 * cols)),
               ffn=32, block_size=32, levels=common["levels"], top_k=2, out=bf(tokens, cols))
    return [(bof4.bof4_linear, linear), (bof4.bof4_linear_backward, backward), (bof4.bof4_moe, moe)]


def wanting(value):
    """The argument with a tensor that requires a gradient in it, or None where none of its tensors can."""
    if isinstance(value, tuple):
        parts = [wanting(v) for v in value]
        return tuple(v if w is None else w for v, w in zip(value, parts)) if any(w is not None for w in parts) else None
    return value.detach().requires_grad_() if torch.is_tensor(value) and value.is_floating_point() else None


def each(bof4, device):
    for fn, kw in arguments(bof4, device):
        n = 0
        for name, value in kw.items():
            w = wanting(value)
            if w is not None:
                n += 1
                yield fn, name, {**kw, name: w}
        assert n >= 6


def test_refused_while_gradients_are_on(bof4):
    """Before anything else is looked at: without a device too."""
    for fn, name, kw in each(bof4, "cpu"):
        with pytest.raises(ValueError, match="records no autograd graph and %s requires a gradient" % name):
            fn(**kw)
        with torch.no_grad(), pytest.raises(ValueError, match="must be a CUDA tensor"):
            fn(**kw)
        with torch.inference_mode(), pytest.raises(ValueError, match="must be a CUDA tensor"):
            fn(**kw)


@pytest.mark.gpu
def test_taken_where_they_are_off(bof4):
    plain = {fn: [t.clone() for t in fn(**kw) if torch.is_tensor(t)] for fn, kw in arguments(bof4, "cuda")}
    for fn, name, kw in each(bof4, "cuda"):
        with pytest.raises(ValueError, match="requires a gradient"):
            fn(**kw)
        with torch.no_grad():
            got = [t for t in fn(**kw) if torch.is_tensor(t)]
        assert len(got) == len(plain[fn]) and all(torch.equal(a, b) for a, b in zip(got, plain[fn])), (fn.__name__, name)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [3, 40])
def test_a_layer_that_is_trained_through(bof4, tokens):
    """The pair inside a torch.autograd.Function: gradients of input, bias and residual, against the same layer in 64 bits.  Values are
    small multiples of powers of two and the activation is relu: everything but the rounding of dx (2^-8) is exact."""
    rows, cols, block = 96, 128, 64
    g = torch.Generator().manual_seed(tokens)
    codes = torch.randint(0, 256, (rows * cols // 2,), generator=g, dtype=torch.uint8).cuda()
    scales = torch.ones(rows * cols // block, device="cuda")
    w = torch.from_numpy(LV)[torch.stack((codes.cpu() >> 4, codes.cpu() & 15), -1).long()].view(rows, cols).double().cuda()

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, bias, residual):
            pre = torch.empty(x.shape[0], rows, dtype=torch.bfloat16, device=x.device)
            y, status = bof4.bof4_linear(codes, scales, rows, cols, block, LV, x, bias=bias, residual=residual, activation=bof4.ACT_RELU, pre=pre)
            ctx.save_for_backward(pre, status)
            return y

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            pre, _ = ctx.saved_tensors
            dx, db, _ = bof4.bof4_linear_backward(codes, scales, rows, cols, block, LV, dy.contiguous(), pre=pre, activation=bof4.ACT_RELU, want_dbias=True)
            return dx, db, dy

    ints = lambda *s: torch.randint(-2, 3, s, generator=g).float().cuda()  # noqa: E731
    x, bias, residual, c = ints(tokens, cols), ints(rows), ints(tokens, rows), ints(tokens, rows)
    a = [x.bfloat16().requires_grad_(), bias.requires_grad_(), residual.bfloat16().requires_grad_()]
    (Layer.apply(*a) * c.bfloat16()).sum().backward()
    b = [t.detach().double().requires_grad_() for t in (x, bias, residual)]
    ((torch.relu(b[0] @ w.T + b[1]) + b[2]) * c.double()).sum().backward()
    assert torch.equal(a[0].grad, b[0].grad.bfloat16())
    assert torch.equal(a[1].grad.double(), b[1].grad) and torch.equal(a[2].grad.double(), b[2].grad)


@pytest.mark.gpu
def test_numbers_are_not_cut_off(bof4):
    """A code beyond 32 bits is refused, not taken for its lower half; a flag that has no truth value raises its own error."""
    (linear, kl), (backward, kb), (moe, km) = arguments(bof4, "cuda")
    for fn, kw, names in ((linear, kl, ("activation", "out_dtype", "block_size")), (backward, kb, ("activation", "block_size")),
                          (moe, km, ("activation", "score", "out_dtype", "block_size", "top_k"))):
        for name in names:
            for value in (1 << 32, (1 << 32) + 1, -(1 << 32), (1 << 32) + 32):
                with pytest.raises(ValueError):
                    fn(**{**kw, name: value})
    neither = torch.ones(2)
    for fn, kw, name in ((backward, kb, "want_dx"), (backward, kb, "want_dbias"), (moe, km, "renormalize")):
        with pytest.raises(RuntimeError, match="ambiguous"):
            fn(**{**kw, name: neither})
