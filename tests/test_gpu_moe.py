"""bof4_moe against a plain implementation in 64 bits (written out here, without the library).

Tolerance: with sums of products within 2^-14 of their sum of magnitudes (mma.sync, at most 2^-23 per accumulation step of 16)
and activations within 2^-20 of max(|z|, 1) and slopes of at most 1.13, h = act(g) u is off by at most
1.13 e_g |u| + |act(g)| e_u + 2^-18 |h| + 2^-20 max(|g|, 1) |u| before and 2^-17 |h| more after its rounding to 16 bits; y by the sum of
w |D| (e_h + 2^-14 |h|) and the error of the weights, twice that of a logit (2^-20 of its sum of magnitudes) and 2^-20
relative; a result in bf16 is rounded once (2^-8)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_linear import LV, act64, act_code, bof4, decode, ints  # noqa: F401

pytestmark = pytest.mark.gpu


def layer(seed, experts, hidden, ffn, block, scale_dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)

    def matrix(n):
        codes = torch.randint(0, 256, (n // 2,), generator=g, dtype=torch.uint8)
        scales = (0.04 + 0.02 * torch.rand(n // block, generator=g)) * (torch.randint(0, 2, (n // block,), generator=g) * 2 - 1)
        return codes.cuda(), scales.to(scale_dtype).cuda()
    return matrix(experts * 2 * ffn * hidden), matrix(experts * hidden * ffn)


def reference(x, router, gate_up, down, ffn, block, top, act, score, renorm, scale, check_gap=True):
    """y, its bound, ids, weights, the weights' bound."""
    experts, hidden = router.shape
    xd = x.double()
    logits = xd @ router.double().T
    e_l = 2.0 ** -20 * (xd.abs() @ router.double().abs().T)
    order = torch.argsort(-logits, dim=1, stable=True)
    if check_gap:  # the choice must not hang on rounding
        s = torch.gather(logits, 1, order)
        b = torch.gather(e_l, 1, order)
        k = min(top + 1, experts)
        assert bool(((s[:, :k - 1] - s[:, 1:k]) > b[:, :k - 1] + b[:, 1:k]).all()), "the oracle's case is ill-conditioned"
    ids = order[:, :top]
    p = torch.softmax(logits, 1) if score == "softmax" else torch.sigmoid(logits)
    w = torch.gather(p, 1, ids)
    if renorm:
        w = w / w.sum(1, keepdim=True)
    w = w * scale
    rel = 4 * e_l.max(1, keepdim=True).values + 2.0 ** -20
    y, tol = torch.zeros_like(xd), torch.zeros_like(xd)
    per1, per2 = 2 * ffn * hidden, hidden * ffn
    for e in torch.unique(ids).tolist():
        w1 = decode(gate_up[0][e * per1 // 2:(e + 1) * per1 // 2], gate_up[1][e * per1 // block:(e + 1) * per1 // block], block, LV, 2 * ffn, hidden)
        w2 = decode(down[0][e * per2 // 2:(e + 1) * per2 // 2], down[1][e * per2 // block:(e + 1) * per2 // block], block, LV, hidden, ffn)
        t, j = torch.nonzero(ids == e, as_tuple=True)
        z, ez = xd[t] @ w1.T, 2.0 ** -14 * (xd[t].abs() @ w1.abs().T)
        g, u, eg, eu = z[:, :ffn], z[:, ffn:], ez[:, :ffn], ez[:, ffn:]
        a = act64(g, act)[0]
        h = a * u
        eh = 1.13 * eg * (u.abs() + eu) + a.abs() * eu + (2.0 ** -18 + 2.0 ** -17) * h.abs() + 2.0 ** -20 * g.abs().clamp(min=1) * u.abs()
        o = h @ w2.T
        y[t] += w[t, j][:, None] * o
        tol[t] += w[t, j].abs()[:, None] * ((eh + 2.0 ** -14 * h.abs()) @ w2.abs().T + rel[t] * o.abs())
    return y, tol + 2.0 ** -22 * y.abs(), ids.int(), w, rel * w.abs()


def check(bof4, x, router, gate_up, down, ffn, block, top, act="silu", score="softmax", renorm=True, scale=1.0, out="f32", levels=LV, **kw):
    y, ids, weights, status = bof4.bof4_moe(
        x, router, gate_up, down, ffn, block, levels, top, activation=act_code(bof4, act), score=bof4.SCORE_SOFTMAX if score == "softmax" else bof4.SCORE_SIGMOID,
        renormalize=renorm, scale=scale, out_dtype=bof4.F32 if out == "f32" else bof4.BF16, **kw)
    assert int(status.item()) == 0
    ry, tol, rids, rw, tw = reference(x, router, gate_up, down, ffn, block, top, act, score, renorm, scale)
    assert torch.equal(ids, rids)
    assert bool(((weights.double() - rw).abs() <= tw + 1e-12).all())
    if out == "bf16":
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * ry.abs()
    assert y.dtype == (torch.float32 if out == "f32" else torch.bfloat16)
    assert bool(((y.double() - ry).abs() <= tol + 1e-12).all()), float(((y.double() - ry).abs() / (tol + 1e-12)).max())
    return y, ids, weights


@pytest.mark.parametrize("tokens,hidden,ffn,experts,top,block", [
    (1, 64, 64, 1, 1, 64), (1, 32, 32, 4, 2, 32), (1, 2048, 1408, 16, 6, 64), (2, 96, 160, 8, 8, 32), (3, 512, 256, 512, 16, 128),
    (5, 1024, 96, 7, 3, 32), (8, 256, 1024, 2, 1, 256), (19, 1024, 768, 64, 8, 64), (33, 320, 576, 33, 2, 64), (64, 256, 256, 3, 2, 64),
    (64, 512, 128, 100, 16, 128), (4, 8192, 64, 4, 2, 64), (2, 64, 4544, 4, 2, 64), (9, 4352, 4160, 2, 2, 64), (7, 4096, 4096, 2, 1, 1024)])
@pytest.mark.parametrize("scale_dtype", [torch.bfloat16, torch.float32])
def test_layer(bof4, tokens, hidden, ffn, experts, top, block, scale_dtype):  # noqa: F811
    g = torch.Generator().manual_seed(tokens + hidden)
    gate_up, down = layer(hidden + ffn, experts, hidden, ffn, block, scale_dtype)
    x = torch.randn(tokens, hidden, generator=g).bfloat16().cuda()
    router = (torch.randn(experts, hidden, generator=g) * 1.5 / math.sqrt(hidden)).to(scale_dtype).cuda()
    check(bof4, x, router, gate_up, down, ffn, block, top)
    check(bof4, x, router, gate_up, down, ffn, block, top, out="bf16", score="sigmoid", renorm=False, scale=2.5)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_activations_and_scores(bof4, act, score, renorm):  # noqa: F811
    g = torch.Generator().manual_seed(4)
    gate_up, down = layer(1, 12, 256, 192, 64)
    x = torch.randn(6, 256, generator=g).bfloat16().cuda()
    router = (torch.randn(12, 256, generator=g) * 0.1).bfloat16().cuda()
    check(bof4, x, router, gate_up, down, 192, 64, 4, act, score, renorm, 0.75)


def test_ties_and_extreme_logits(bof4):  # noqa: F811
    """Equal logits (small integers, exact in fp32) go to the lowest index; infinities and NaN leave the choice in range."""
    g = torch.Generator().manual_seed(8)
    experts, hidden, ffn = 40, 64, 64
    gate_up, down = layer(2, experts, hidden, ffn, 64)
    x = ints(g, 9, hidden, lo=-1, hi=1)
    router = ints(g, experts, hidden, lo=-1, hi=1)
    router[10:20] = router[0]
    x[3] = 0                                     # all logits equal
    logits = x.double() @ router.double().T
    y, ids, w, s = bof4.bof4_moe(x, router, gate_up, down, ffn, 64, LV, 6)
    assert int(s.item()) == 0 and torch.equal(ids, torch.argsort(-logits, dim=1, stable=True)[:, :6].int())
    assert ids[3].tolist() == list(range(6)) and bool(((w[3] - 1 / 6).abs() < 1e-6).all())
    r32 = router.float() * 1e30                  # far apart: one expert takes everything, nothing overflows
    y, ids, w, s = bof4.bof4_moe(x, r32, gate_up, down, ffn, 64, LV, 2, renormalize=False)
    assert bool(torch.isfinite(w).all()) and bool(torch.isfinite(y.float()).all())
    x[1, 5], x[2, 7] = float("inf"), float("nan")
    y2, ids, w, s = bof4.bof4_moe(x, router, gate_up, down, ffn, 64, LV, 6)
    assert int(s.item()) == 0 and bool((ids >= 0).all()) and bool((ids < experts).all())
    assert all(len(set(row)) == 6 for row in ids.tolist())
    y, _, _, _ = bof4.bof4_moe(ints(torch.Generator().manual_seed(8), 9, hidden, lo=-1, hi=1), router, gate_up, down, ffn, 64, LV, 6)
    for t in (0, 4, 5, 6, 7, 8):
        assert torch.equal(y[t], y2[t])


def test_same_bits_again_and_beside(bof4):  # noqa: F811
    """Repeated, on a side stream, in two graphs that share a workspace; rows apart; what lies between the rows stays."""
    g = torch.Generator().manual_seed(6)
    tokens, experts, hidden, ffn, top = 11, 24, 640, 320, 4
    gate_up, down = layer(9, experts, hidden, ffn, 64)
    xs = torch.randn(tokens, hidden + 16, generator=g).bfloat16().cuda()
    router = (torch.randn(experts, hidden, generator=g) * 0.05).bfloat16().cuda()
    cb = torch.from_numpy(LV).cuda()
    x = xs[:, :hidden]
    y, ids, w = check(bof4, x, router, gate_up, down, ffn, 64, top, out="bf16", levels=cb)
    ys = torch.full((tokens, hidden + 3), 5.0, dtype=torch.bfloat16, device="cuda")
    bof4.bof4_moe(x, router, gate_up, down, ffn, 64, cb, top, out=ys[:, :hidden])
    assert torch.equal(ys[:, :hidden], y) and bool((ys[:, hidden:] == 5).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = bof4.bof4_moe(x, router, gate_up, down, ffn, 64, cb, top)[0]
    torch.cuda.synchronize()
    assert torch.equal(z, y)
    ws = torch.full((bof4.bof4_moe_workspace_bytes(tokens, hidden, ffn, experts, top),), 255, dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.zeros_like(y) for _ in range(2)], []
    for o in outs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            bof4.bof4_moe(x, router, gate_up, down, ffn, 64, cb, top, out=o, workspace=ws)
        graphs.append(gr)
    for _ in range(4):
        for o, gr in zip(outs, graphs):
            o.zero_()
            gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], y) and torch.equal(outs[1], y)


def test_next_to_the_dense_layers(bof4):  # noqa: F811
    """One expert, chosen by every token: the same as bof4_linear twice with the gate between."""
    g = torch.Generator().manual_seed(3)
    tokens, hidden, ffn = 6, 512, 256
    (c1, s1), (c2, s2) = layer(5, 1, hidden, ffn, 64)
    x = torch.randn(tokens, hidden, generator=g).bfloat16().cuda()
    y, ids, w, _ = bof4.bof4_moe(x, torch.zeros(1, hidden, device="cuda"), (c1, s1), (c2, s2), ffn, 64, LV, 1, out_dtype=bof4.F32)
    assert bool((ids == 0).all()) and bool((w == 1).all())
    z, _ = bof4.bof4_linear(c1, s1, 2 * ffn, hidden, 64, LV, x, out_dtype=bof4.F32)
    h = (torch.nn.functional.silu(z[:, :ffn].double()) * z[:, ffn:].double()).bfloat16()
    d, _ = bof4.bof4_linear(c2, s2, hidden, ffn, 64, LV, h, out_dtype=bof4.F32)
    mag = h.double().abs() @ decode(c2, s2, 64, LV, hidden, ffn).abs().T
    assert bool(((y.double() - d.double()).abs() <= 2.0 ** -7 * mag).all())   # h rounded to bf16 here: 2^-8, and to 16 bits there


def test_random_layers(bof4):  # noqa: F811
    rng = np.random.default_rng(3)
    done = 0
    for trial in range(40):
        block = int(rng.choice([32, 64, 128]))
        hidden, ffn = block * int(rng.integers(1, 1 + 1500 // block)), block * int(rng.integers(1, 1 + 800 // block))
        experts, tokens = int(rng.integers(1, 70)), int(rng.integers(1, 65))
        top = int(rng.integers(1, min(16, experts) + 1))
        g = torch.Generator().manual_seed(trial)
        gate_up, down = layer(trial, experts, hidden, ffn, block, torch.float32 if trial % 2 else torch.bfloat16)
        x = torch.randn(tokens, hidden, generator=g).bfloat16().cuda()
        router = (torch.randn(experts, hidden, generator=g) * 1.5 / math.sqrt(hidden)).cuda()
        logits = x.double() @ router.double().T
        s = torch.sort(logits, dim=1, descending=True).values[:, :top + 1]
        if s.shape[1] > 1 and float((s[:, :-1] - s[:, 1:]).min()) < 2e-4:
            continue      # the choice would hang on the rounding of a logit
        check(bof4, x, router, gate_up, down, ffn, block, top, out="bf16" if trial % 4 == 0 else "f32")
        done += 1
    assert done >= 10, done


def test_other_experts_do_not_matter(bof4):  # noqa: F811
    """Experts that nobody chose may hold anything, next to the chosen ones as they lie."""
    experts, hidden, ffn, block = 8, 96, 160, 32
    gate_up, down = layer(3, experts, hidden, ffn, block)
    g = torch.Generator().manual_seed(5)
    x = torch.randn(7, hidden, generator=g).bfloat16().cuda()
    router = (torch.randn(experts, hidden, generator=g) * 0.1).bfloat16().cuda()
    router[[1, 2, 4, 6, 7]] = 0
    x[:, 0], router[:, 0] = 100.0, torch.tensor([1.0, -1, -1, 1, -1, 1, -1, -1], device="cuda").bfloat16()
    y, ids, w, s = bof4.bof4_moe(x, router, gate_up, down, ffn, block, LV, 3)
    assert sorted(set(ids.flatten().tolist())) == [0, 3, 5]
    for bad in (float("inf"), float("nan")):
        for scales, per in ((gate_up[1], 2 * ffn * hidden // block), (down[1], hidden * ffn // block)):
            scales.view(experts, per)[[1, 2, 4, 6, 7]] = bad
        y2, ids2, w2, s = bof4.bof4_moe(x, router, gate_up, down, ffn, block, LV, 3)
        assert int(s.item()) == 0 and torch.equal(y, y2) and torch.equal(ids, ids2) and torch.equal(w, w2) and bool(torch.isfinite(y2.float()).all())


def test_offsets_beyond_32_bits(bof4):  # noqa: F811
    """Experts of more than 2^32 weights together; the last ones are chosen."""
    experts, hidden, ffn, block = 512, 2112, 2112, 64
    g = torch.Generator(device="cuda").manual_seed(9)

    def matrix(n):
        codes = torch.randint(0, 256, (n // 2,), generator=g, dtype=torch.uint8, device="cuda")
        return codes, (0.04 + 0.02 * torch.rand(n // block, generator=g, device="cuda")).bfloat16()
    gate_up, down = matrix(experts * 2 * ffn * hidden), matrix(experts * hidden * ffn)
    x = torch.randn(5, hidden, generator=g, device="cuda").bfloat16()
    router = (torch.randn(experts, hidden, generator=g, device="cuda") * 1.5 / math.sqrt(hidden)).bfloat16()
    x[:, 0], router[:, 0], router[[0, 300, 509, 511], 0] = 32.0, 0.0, 1.0
    y, ids, w = check(bof4, x, router, gate_up, down, ffn, block, 4)
    assert sorted(set(ids.flatten().tolist())) == [0, 300, 509, 511]


def test_two_layers_at_once(bof4):  # noqa: F811
    """Calls on two streams, with workspaces of their own, and a dense layer on a third: none waits for another in vain."""
    g = torch.Generator().manual_seed(12)
    experts, hidden, ffn = 16, 2048, 1024
    gate_up, down = layer(12, experts, hidden, ffn, 64)
    router = (torch.randn(experts, hidden, generator=g) * 0.05).bfloat16().cuda()
    xs = [torch.randn(n, hidden, generator=g).bfloat16().cuda() for n in (3, 40)]
    x = torch.randn(300, hidden, generator=g).bfloat16().cuda()
    want = [bof4.bof4_moe(t, router, gate_up, down, ffn, 64, LV, 4)[0] for t in xs]
    dense = bof4.bof4_linear(*gate_up, experts * 2 * ffn, hidden, 64, LV, x)[0]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for _ in range(10):
        for t, s in zip(xs, streams):
            with torch.cuda.stream(s):
                got.append(bof4.bof4_moe(t, router, gate_up, down, ffn, 64, LV, 4))
        with torch.cuda.stream(streams[2]):
            got.append(bof4.bof4_linear(*gate_up, experts * 2 * ffn, hidden, 64, LV, x))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert int(r[-1].item()) == 0 and torch.equal(r[0], (want + [dense])[i % 3])


def test_no_tokens(bof4):  # noqa: F811
    gate_up, down = layer(1, 4, 64, 64, 64)
    y, ids, w, s = bof4.bof4_moe(torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 64, device="cuda"), gate_up, down, 64, 64, LV, 2)
    assert y.shape == (0, 64) and ids.shape == (0, 2) and int(s.item()) == 0


def test_refusals(bof4):  # noqa: F811
    experts, hidden, ffn = 4, 128, 64
    gate_up, down = layer(1, experts, hidden, ffn, 64)
    x = torch.zeros(2, hidden, dtype=torch.bfloat16, device="cuda")
    router = torch.zeros(experts, hidden, device="cuda")
    ok = dict(x=x, router=router, gate_up=gate_up, down=down, ffn=ffn, block_size=64, levels=LV, top_k=2)
    bof4.bof4_moe(**ok)
    bad = lambda err, **kw: pytest.raises(err, bof4.bof4_moe, **{**ok, **kw})  # noqa: E731
    bad(bof4.Bof4Error, top_k=5)
    bad(ValueError, top_k=0)
    bad(ValueError, top_k=17)
    bad(bof4.Bof4Error, score=2)
    bad(bof4.Bof4Error, activation=9)
    bad(ValueError, out_dtype=3)
    bad(TypeError, x=x.float())
    bad(ValueError, x=x.cpu())
    bad(ValueError, x=x[:, :64])
    bad(bof4.Bof4Error, x=torch.zeros(65, hidden, dtype=torch.bfloat16, device="cuda"))
    bad(TypeError, router=router.half())
    bad(ValueError, router=router[:3])
    bad(ValueError, ffn=32)
    bad(ValueError, gate_up=(gate_up[0][:-32], gate_up[1]))
    bad(ValueError, down=(down[0], down[1][:-1]))
    bad(TypeError, down=(down[0], down[1].float()))
    bad(bof4.Bof4Error, block_size=128, gate_up=(gate_up[0], gate_up[1][::2].contiguous()), down=(down[0], down[1][::2].contiguous()))
    bad(ValueError, out=torch.zeros(2, hidden, device="cuda"), out_dtype=7)
    bad(TypeError, out=torch.zeros(2, hidden, device="cuda"))
    need = bof4.bof4_moe_workspace_bytes(2, hidden, ffn, experts, 2)
    bad(bof4.Bof4Error, workspace=torch.zeros(need - 1, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("tokens,hidden,ffn", [(3, 8192, 5120), (20, 4608, 8448)])
def test_cold_memory(bof4, tokens, hidden, ffn):  # noqa: F811
    """Rows of more columns than a CTA has warps for, so that a unit takes several turns of the ring of codes, from memory that has
    left L2: the same bits as the first time, whatever the workspace holds."""
    experts, top, block = 4, 2, 64
    g = torch.Generator().manual_seed(tokens)
    gate_up, down = layer(hidden, experts, hidden, ffn, block)
    x = torch.randn(tokens, hidden, generator=g).bfloat16().cuda()
    router = (torch.randn(experts, hidden, generator=g) * 1.5 / math.sqrt(hidden)).bfloat16().cuda()
    y, ids, w = check(bof4, x, router, gate_up, down, ffn, block, top)
    big = torch.empty(300 << 20, dtype=torch.uint8, device="cuda")
    n = bof4.bof4_moe_workspace_bytes(tokens, hidden, ffn, experts, top)
    for trial in range(12):
        ws = torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda")
        big.fill_(trial)
        y2, ids2, w2, s = bof4.bof4_moe(x, router, gate_up, down, ffn, block, LV, top, out_dtype=bof4.F32, workspace=ws)
        assert int(s.item()) == 0 and torch.equal(y2, y) and torch.equal(ids2, ids) and torch.equal(w2, w)


@pytest.mark.parametrize("router_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("first,step", [(-90, 1), (-88, 1), (-100, 7), (-200, 30), (-1, 30), (-600, 1), (0, 60), (3, 40), (100, 64)])
def test_logistic_scores_far_out(bof4, router_dtype, first, step):  # noqa: F811
    """Weights that are divided by their sum depend on the differences of logits where all lie far below zero.  The logits are integers
    that x picks out of the router, so a weight is off by a few units of exp, sum and quotient only: 2^-20 relative, or what fp32
    cannot hold."""
    experts, hidden, ffn, top = 9, 64, 64, 4
    gate_up, down = layer(21, experts, hidden, ffn, 64)
    g = torch.Generator().manual_seed(22)
    x = torch.randn(3, hidden, generator=g).bfloat16().cuda()
    x[:, :3] = torch.eye(3)
    order = torch.randperm(experts, generator=g).cuda()
    router = torch.zeros(experts, hidden, device="cuda")
    router[order, 0] = first - step * torch.arange(experts, device="cuda").float()
    router[:, 1], router[order, 2] = first, first - 2.0 * step * torch.arange(experts, device="cuda").float()
    router = router.to(router_dtype)
    assert torch.equal(x.double() @ router.double().T, router[:, :3].double().T.round())
    y, ids, w, s = bof4.bof4_moe(x, router, gate_up, down, ffn, 64, LV, top, score=bof4.SCORE_SIGMOID, out_dtype=bof4.F32)
    ry, tol, rids, rw, _ = reference(x, router, gate_up, down, ffn, 64, top, "silu", "sigmoid", True, 1.0, check_gap=False)
    assert int(s.item()) == 0 and torch.equal(ids, rids)
    assert bool(((w.double() - rw).abs() <= 2.0 ** -20 * rw + 1e-37).all()), (w, rw)
    assert bool(((y.double() - ry).abs() <= tol + 1e-12).all())
    _, _, one, _ = bof4.bof4_moe(x, router, gate_up, down, ffn, 64, LV, 1, score=bof4.SCORE_SIGMOID, scale=0.5)
    assert bool((one == 0.5).all())
    # an expert that is masked out has no weight beside one that is not
    masked = router.clone()
    masked[order[1:], 0] = -float("inf")
    y, ids, w, s = bof4.bof4_moe(x[:1], masked, gate_up, down, ffn, 64, LV, top, score=bof4.SCORE_SIGMOID)
    assert int(ids[0, 0]) == int(order[0]) and w[0].tolist() == [1.0, 0.0, 0.0, 0.0] and bool(torch.isfinite(y.float()).all())


# Levels among which 0 and 1 are: matrices that pick single values out of their operand, and exact sums.
PICK = np.array([-15, -13, -11, -9, -7, -5, -3, -1, 1, 3, 5, 7, 9, 11, 0, 16], np.float32) / 16
ZERO, ONE = 14, 15


def packed(codes, scale, block=64):
    """(codes, scales) of a matrix of codes, all blocks with the same constant."""
    c = codes.to(torch.uint8).reshape(-1, 2)
    return ((c[:, 0] << 4) | c[:, 1]).cuda(), torch.full((codes.numel() // block,), scale).bfloat16().cuda()


def test_h_beside_the_largest_values(bof4):  # noqa: F811
    """h above the largest bf16 value but finite in fp32: both halves stay finite, and the product with a small weight is exact."""
    hidden = ffn = 64
    up = torch.full((2 * ffn, hidden), ZERO)
    up[:ffn, :2], up[ffn:, 2] = ONE, ONE      # g = x0 + x1, u = x2
    x = torch.zeros(4, hidden, dtype=torch.bfloat16, device="cuda")
    x[:, 0], x[:, 1], x[:, 2] = 255 * 2.0 ** 57, 3 * 2.0 ** 55, 2.0 ** 63
    x[1, 2], x[2, 1], x[3, 2] = -2.0 ** 63, 0.0, float("inf")
    h = (x[:, 0].double() + x[:, 1].double()) * x[:, 2].double()
    assert h[0] > 255.5 * 2.0 ** 120 and h[0] < 2.0 ** 128 and h[2] == 255 * 2.0 ** 120
    down = torch.full((hidden, ffn), ZERO)
    down[torch.arange(hidden), torch.arange(ffn)] = ONE
    y, _, _, s = bof4.bof4_moe(x, torch.zeros(1, hidden, device="cuda"), packed(up, 1.0), packed(down, 2.0 ** -10), ffn, 64, PICK, 1, activation=bof4.ACT_NONE,
                               out_dtype=bof4.F32)
    assert int(s.item()) == 0 and torch.equal(y[:3].double(), (h[:3, None] * 2.0 ** -10).expand(3, hidden))
    assert not bool(torch.isfinite(y[3]).any())
