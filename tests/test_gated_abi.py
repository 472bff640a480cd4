"""CPU-only checks of bof4_gated, bof4_gated_backward and bof4_cross_entropy: every refusal that needs no device comes back as its error code at the C
ABI before anything is launched (the pointers are addresses that are never read), the workspace functions answer without one, and a tensor that requires a
gradient is refused while gradients are on."""
import numpy as np
import pytest
import torch

import __graft_entry__ as entry

P = 1 << 20  # an aligned address
F32, BF16 = 0, 1
GATED = ("codes scales scale_dtype ffn cols block_size codebook x ldx n_tokens bias bias_dtype activation out_idx out_val n_out capacity h h_dtype ldh pre ld_pre "
         "status ws ws_bytes stream").split()
BACKWARD = ("codes scales scale_dtype ffn cols block_size codebook dh dh_dtype ld_dh n_tokens pre ld_pre activation out_idx out_val n_out capacity dx ld_dx dbias "
            "status ws ws_bytes stream").split()
LOSS = ("codes scales scale_dtype rows cols block_size codebook x ldx n_tokens targets dloss out_idx out_val n_out capacity loss lse dx ld_dx status ws "
        "ws_bytes stream").split()


@pytest.fixture(scope="module")
def L():
    entry.build()
    from paper_2505_06653_b200 import binding
    return binding.lib()


def caller(fn, names, base):
    def call(**kw):
        values = {**base, **kw}
        assert set(values) == set(names)
        return fn(*[values[n] for n in names])
    return call


MATRIX = dict(codes=P, scales=P, scale_dtype=BF16, cols=512, block_size=64, codebook=P, out_idx=None, out_val=None, n_out=None, capacity=0, n_tokens=4, status=P, ws=P,
              ws_bytes=0, stream=None)


def calls(L):
    return {"bof4_gated": caller(L.bof4_gated, GATED, dict(MATRIX, ffn=128, x=P, ldx=512, bias=None, bias_dtype=F32, activation=4, h=P, h_dtype=BF16, ldh=128, pre=None, ld_pre=0)),
            "bof4_gated_backward": caller(L.bof4_gated_backward, BACKWARD, dict(MATRIX, ffn=128, dh=P, dh_dtype=BF16, ld_dh=128, pre=P, ld_pre=256, activation=4, dx=P, ld_dx=512, dbias=P)),
            "bof4_cross_entropy": caller(L.bof4_cross_entropy, LOSS, dict(MATRIX, rows=256, x=P, ldx=512, targets=P, dloss=None, loss=P, lse=P, dx=P, ld_dx=512))}


def refused(L, name, groups, ws=True):
    """The arguments of a group come back with the same code, those of different groups with different ones; the call as it is lacks a workspace."""
    call, codes = calls(L)[name], []
    for group in groups:
        got = {call(**kw) for kw in group}
        assert len(got) == 1 and 0 not in got, (name, group, got)
        codes.append(got.pop())
        assert name in L.bof4_last_error().decode()
    last = call()
    assert "workspace" in L.bof4_last_error().decode()
    assert len({0, last, *codes}) == len(codes) + 2
    assert call(ws=None, ws_bytes=1 << 40) == last and call(ws=P + 16, ws_bytes=1 << 40) == last


def test_gated_refuses(L):
    big = dict(ffn=1 << 19, cols=4096, ldx=4096, ldh=1 << 19, out_idx=P, out_val=P, n_out=P, capacity=1)
    refused(L, "bof4_gated", [
        [dict(ffn=-1), dict(cols=-64), dict(n_tokens=-1), dict(activation=5), dict(activation=-1), dict(status=None), dict(codes=None), dict(scales=None), dict(codebook=None), dict(x=None),
         dict(h=None), dict(codes=P + 16), dict(x=P + 8), dict(ldx=516), dict(out_idx=P, capacity=1)],
        [dict(block_size=48), dict(block_size=16), dict(block_size=8192), dict(cols=96), dict(ldx=504), dict(ldh=127), dict(pre=P, ld_pre=255), dict(ffn=1 << 30), dict(ffn=1 << 62),
         dict(n_tokens=1 << 31), big],
        [dict(scale_dtype=7), dict(h_dtype=5), dict(bias=P, bias_dtype=9)]])


def test_gated_backward_refuses(L):
    refused(L, "bof4_gated_backward", [
        [dict(ffn=-1), dict(n_tokens=-1), dict(activation=5), dict(status=None), dict(codes=None), dict(scales=None), dict(codebook=None), dict(dh=None), dict(pre=None), dict(codes=P + 16)],
        [dict(block_size=48), dict(cols=96), dict(ld_dh=127), dict(ld_pre=255), dict(ld_dx=511), dict(ffn=1 << 30), dict(n_tokens=1 << 31)],
        [dict(scale_dtype=7), dict(dh_dtype=5)]])


def test_cross_entropy_refuses(L):
    refused(L, "bof4_cross_entropy", [
        [dict(rows=-1), dict(n_tokens=-1), dict(status=None), dict(codes=None), dict(scales=None), dict(codebook=None), dict(x=None), dict(targets=None), dict(loss=None), dict(codes=P + 16),
         dict(x=P + 8), dict(ldx=516), dict(out_idx=P, out_val=P, capacity=1)],
        [dict(block_size=48), dict(cols=96), dict(rows=0), dict(cols=0), dict(ldx=504), dict(ld_dx=511), dict(rows=1 << 31), dict(n_tokens=1 << 31)],
        [dict(scale_dtype=7)]])


def test_workspaces(L):
    for fn, shape in ((L.bof4_gated_workspace_bytes, (11008, 4096)), (L.bof4_cross_entropy_workspace_bytes, (32000, 4096))):
        for flag in (0, 1):
            sizes = [fn(*shape, t, flag, 0) for t in (0, 1, 13, 100, 384, 385, 767, 768, 5000)]
            assert all(s > 0 and s % 256 == 0 for s in sizes)
            assert fn(*shape, 1000, flag, 5000) >= fn(*shape, 1000, flag, 0)
            assert not any(fn(*a) for a in ((-1, 4096, 1, flag, 0), (11008, -1, 1, flag, 0), (11008, 4096, -1, flag, 0), (11008, 4096, 1, flag, -1), (1 << 31, 4096, 1, flag, 0),
                                            (11008, 1 << 31, 1, flag, 0), (11008, 4096, 1 << 31, flag, 0)))
    # the logits of all rows are never kept for many tokens: 100,000 tokens of 152,000 rows would be 61 GB
    assert L.bof4_cross_entropy_workspace_bytes(152000, 4096, 100000, 1, 0) < 10 << 30


def arguments(bof4, device):
    g = torch.Generator().manual_seed(1)
    ffn, cols, tokens = 32, 64, 3
    bf = lambda *s: torch.randn(*s, generator=g).bfloat16().to(device)  # noqa: E731
    lst = (torch.tensor([5], dtype=torch.int32, device=device), bf(1), torch.tensor([1], device=device))
    common = dict(codes=torch.zeros(ffn * cols, dtype=torch.uint8, device=device), scales=torch.ones(2 * ffn * cols // 32, device=device), cols=cols, block_size=32,
                  levels=torch.from_numpy((np.arange(16, dtype=np.float32) - 7.5) / 8).to(device), outliers=lst)
    return [(bof4.bof4_gated, dict(common, ffn=ffn, x=bf(tokens, cols), bias=bf(2 * ffn), pre=bf(tokens, 2 * ffn), out=bf(tokens, ffn))),
            (bof4.bof4_gated_backward, dict(common, ffn=ffn, dh=bf(tokens, ffn), pre=bf(tokens, 2 * ffn), out=bf(tokens, cols))),
            (bof4.bof4_cross_entropy, dict(common, rows=2 * ffn, x=bf(tokens, cols), targets=torch.zeros(tokens, dtype=torch.int64, device=device),
                                           dloss=torch.ones(tokens, device=device), want_dx=True, out=bf(tokens, cols)))]


def test_refused_while_gradients_are_on(L):
    import paper_2505_06653_b200 as bof4
    for fn, kw in arguments(bof4, "cpu"):
        names = [k for k, v in kw.items() if (torch.is_tensor(v) and v.is_floating_point()) or k == "outliers"]
        assert len(names) >= 6
        for name in names:
            v = kw[name]
            wanting = {**kw, name: (v[0], v[1].detach().requires_grad_(), v[2]) if name == "outliers" else v.detach().requires_grad_()}
            with pytest.raises(ValueError, match="records no autograd graph and %s requires a gradient" % name):
                fn(**wanting)
            with torch.no_grad(), pytest.raises(ValueError, match="must be a CUDA tensor"):
                fn(**wanting)


@pytest.mark.gpu
def test_numbers_are_not_cut_off(L):
    """A code beyond 32 bits is refused, not taken for its lower half; a flag that has no truth value raises its own error."""
    import paper_2505_06653_b200 as bof4
    for fn, kw in arguments(bof4, "cuda"):
        fn(**kw)
        for name in ("block_size", *(n for n in ("activation", "out_dtype") if n in fn.__code__.co_varnames)):
            for value in (1 << 32, (1 << 32) + 1, -(1 << 32), (1 << 32) + 32):
                with pytest.raises(ValueError):
                    fn(**{**kw, name: value})
        for name in (n for n in ("want_dx", "want_dbias") if n in fn.__code__.co_varnames):
            with pytest.raises(RuntimeError, match="ambiguous"):
                fn(**{**kw, name: torch.ones(2)})
