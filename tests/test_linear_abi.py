"""CPU-only checks of bof4_linear, bof4_linear_backward and bof4_moe at the C ABI: every refusal that needs no device comes back
as its error code before anything is launched, and the workspace functions answer without one.  The pointers are addresses that
are never read."""
import pytest

import __graft_entry__ as entry

P = 1 << 20  # an aligned address
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def L():
    entry.build()
    from paper_2505_06653_b200 import binding
    assert (F32, BF16) == (binding.F32, binding.BF16)
    return binding.lib()


LINEAR = ("codes scales scale_dtype rows cols block_size codebook x ldx n_tokens bias bias_dtype residual ld_residual activation out_idx out_val n_out "
          "capacity y y_dtype ldy pre ld_pre status ws ws_bytes stream").split()
BACKWARD = ("codes scales scale_dtype rows cols block_size codebook dy dy_dtype ld_dy n_tokens pre ld_pre activation out_idx out_val n_out capacity dx "
            "ld_dx dbias status ws ws_bytes stream").split()
MOE = ("x ldx n_tokens hidden router router_dtype n_experts top_k score renormalize scale gate_up_codes gate_up_scales down_codes down_scales "
       "scale_dtype ffn block_size codebook activation y y_dtype ldy ids weights status ws ws_bytes stream").split()


def caller(fn, names, base):
    def call(**kw):
        values = {**base, **kw}
        assert set(values) == set(names)
        return fn(*[values[n] for n in names])
    return call


def linear(L):
    return caller(L.bof4_linear, LINEAR, dict(
        codes=P, scales=P, scale_dtype=BF16, rows=256, cols=512, block_size=64, codebook=P, x=P, ldx=512, n_tokens=4, bias=None, bias_dtype=F32,
        residual=None, ld_residual=0, activation=0, out_idx=None, out_val=None, n_out=None, capacity=0, y=P, y_dtype=BF16, ldy=256, pre=None, ld_pre=0,
        status=P, ws=P, ws_bytes=0, stream=None))


def backward(L):
    return caller(L.bof4_linear_backward, BACKWARD, dict(
        codes=P, scales=P, scale_dtype=BF16, rows=256, cols=512, block_size=64, codebook=P, dy=P, dy_dtype=BF16, ld_dy=256, n_tokens=4, pre=None, ld_pre=0,
        activation=0, out_idx=None, out_val=None, n_out=None, capacity=0, dx=P, ld_dx=512, dbias=P, status=P, ws=P, ws_bytes=0, stream=None))


def moe(L):
    return caller(L.bof4_moe, MOE, dict(
        x=P, ldx=256, n_tokens=4, hidden=256, router=P, router_dtype=BF16, n_experts=8, top_k=2, score=0, renormalize=1, scale=1.0, gate_up_codes=P,
        gate_up_scales=P, down_codes=P, down_scales=P, scale_dtype=BF16, ffn=128, block_size=64, codebook=P, activation=4, y=P, y_dtype=BF16, ldy=256,
        ids=P, weights=P, status=P, ws=P, ws_bytes=0, stream=None))


def message(L):
    return L.bof4_last_error().decode()


def test_linear_refuses(L):
    call = linear(L)
    codes = dict(rows=-1, cols=-64, n_tokens=-1, activation=5)
    first = call(rows=-1)
    assert first != 0 and "bof4_linear" in message(L)
    for name, value in codes.items():
        assert call(**{name: value}) == first, name
    for kw in (dict(activation=-1), dict(status=None), dict(codes=None), dict(scales=None), dict(codebook=None), dict(x=None), dict(y=None),
               dict(codes=P + 16), dict(x=P + 8), dict(ldx=516), dict(out_idx=P, capacity=1), dict(out_idx=P, out_val=P, capacity=1)):
        assert call(**kw) == first, kw
    shape = call(block_size=48)
    assert shape not in (0, first)
    for kw in (dict(block_size=16), dict(block_size=8192), dict(cols=96), dict(ldx=504), dict(ldy=255), dict(residual=P, ld_residual=8), dict(pre=P, ld_pre=8),
               dict(rows=1 << 31), dict(n_tokens=1 << 31), dict(rows=1 << 20, cols=4096, ldx=4096, ldy=1 << 20, out_idx=P, out_val=P, n_out=P, capacity=1)):
        assert call(**kw) == shape, kw
    dtype = call(scale_dtype=7)
    assert dtype not in (0, first, shape)
    for kw in (dict(y_dtype=5), dict(bias=P, bias_dtype=9)):
        assert call(**kw) == dtype, kw
    ws = call()
    assert ws not in (0, first, shape, dtype) and "workspace" in message(L)
    assert call(ws=None) == ws and call(ws=P + 64, ws_bytes=1 << 30) == ws
    assert call(n_tokens=100) == ws  # (the form for many tokens)
    assert call(out_idx=P, out_val=P, n_out=P, capacity=-1) not in (0, ws)


def test_backward_refuses(L):
    call = backward(L)
    first = call(rows=-1)
    for kw in (dict(cols=-64), dict(n_tokens=-1), dict(activation=9), dict(status=None), dict(dy=None), dict(codes=None), dict(scales=None),
               dict(codebook=None), dict(activation=4), dict(codes=P + 16), dict(out_idx=P, capacity=1)):
        assert call(**kw) == first != 0, kw
    shape = call(block_size=48)
    for kw in (dict(cols=96), dict(ld_dy=255), dict(ld_dx=511), dict(activation=4, pre=P, ld_pre=255), dict(cols=1 << 31, ld_dx=1 << 31)):
        assert call(**kw) == shape != first, kw
    dtype = call(dy_dtype=4)
    assert call(scale_dtype=4) == dtype not in (0, first, shape)
    ws = call()
    need = L.bof4_linear_workspace_bytes(256, 512, 4, 1, 0)
    assert ws not in (0, first, shape, dtype) and call(ws=P + 1, ws_bytes=need) == ws and call(ws_bytes=need - 1) == ws


def test_moe_refuses(L):
    call = moe(L)
    shape = call(n_tokens=65)
    assert shape != 0 and "64 tokens" in message(L)
    for kw in (dict(n_tokens=-1), dict(n_experts=0), dict(n_experts=513), dict(top_k=0), dict(top_k=17), dict(top_k=9), dict(hidden=48), dict(ffn=96),
               dict(block_size=512), dict(block_size=33), dict(hidden=1 << 21), dict(ffn=0), dict(ldx=248), dict(ldy=255)):
        assert call(**kw) == shape, kw
    dtype = call(router_dtype=3)
    for kw in (dict(scale_dtype=3), dict(y_dtype=3)):
        assert call(**kw) == dtype not in (0, shape), kw
    arg = call(score=2)
    for kw in (dict(activation=5), dict(activation=-1), dict(status=None), dict(x=None), dict(router=None), dict(gate_up_codes=None), dict(gate_up_scales=None),
               dict(down_codes=None), dict(down_scales=None), dict(codebook=None), dict(y=None), dict(ids=None), dict(weights=None),
               dict(gate_up_codes=P + 16), dict(down_codes=P + 8), dict(x=P + 2), dict(router=P + 4), dict(ldx=260)):
        assert call(**kw) == arg not in (0, shape, dtype), kw
    ws = call()
    need = L.bof4_moe_workspace_bytes(4, 256, 128, 8, 2)
    for kw in (dict(ws=None, ws_bytes=need), dict(ws=P + 128, ws_bytes=need), dict(ws_bytes=need - 1)):
        assert call(**kw) == ws not in (0, shape, dtype, arg), kw


def test_linear_workspace(L):
    f = L.bof4_linear_workspace_bytes
    for bad in ((-1, 64, 1, 0, 0), (64, -64, 1, 0, 0), (64, 64, -1, 0, 0), (64, 64, 1, 0, -1), (1 << 31, 64, 1, 0, 0), (64, 1 << 31, 1, 0, 0), (64, 64, 1 << 31, 0, 0)):
        assert f(*bad) == 0, bad
    for tokens in (0, 1, 6, 7, 16, 17, 64, 257, 5000):
        for rows, cols in ((0, 64), (1, 32), (130, 96), (4096, 14336), (28672, 8192)):
            plain, list_, back = f(rows, cols, tokens, 0, 0), f(rows, cols, tokens, 0, 1000), f(rows, cols, tokens, 1, 0)
            assert plain > 0 and list_ > 0 and back > 0, (tokens, rows, cols)
            if rows and tokens:
                assert back >= tokens * rows * 2  # dz
    assert f(64, 0, 5, 0, 0) > 0


def test_moe_workspace(L):
    f = L.bof4_moe_workspace_bytes
    for bad in ((65, 256, 128, 8, 2), (-1, 256, 128, 8, 2), (4, 250, 128, 8, 2), (4, 256, 0, 8, 2), (4, 256, 128, 0, 1), (4, 256, 128, 513, 2), (4, 256, 128, 8, 9),
                (4, 256, 128, 32, 17), (4, 1 << 21, 128, 8, 2)):
        assert f(*bad) == 0, bad
    for tokens, hidden, ffn, experts, top in ((0, 32, 32, 1, 1), (1, 2048, 1408, 64, 6), (64, 4096, 14336, 512, 16), (64, 1 << 20, 1 << 20, 512, 16)):
        # logits, two halves of h, the experts' results
        assert f(tokens, hidden, ffn, experts, top) >= tokens * (4 * experts + top * (4 * ffn + 4 * hidden))
