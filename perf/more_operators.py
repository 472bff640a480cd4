"""The gated block and the vocabulary loss over 4-bit matrices, as cases that can be prepared and run.

A case is a dict of plain values.  ``op`` says which operator it is:

    gated     bof4_gated: h = act(x G^T) * (x U^T), gate and up rows in one 4-bit matrix of 2 ``ffn`` rows
    backward  bof4_gated_backward: the gradients of x and bias of that block (the weights are frozen)
    loss      bof4_cross_entropy: softmax cross entropy of the logits x W^T over ``vocab`` rows, with the gradient of x where ``grad``

W is a 4-bit matrix: the dequantised weight of the library is bf16(constant * level), and where a list of outliers belongs
to the matrix its entries hold their stored bf16 values.  Weights are near-Gaussian, as the weights of language models are.
"""
import math

import torch

own = False

LEVELS = [-0.8568463921546936, -0.6692874431610107, -0.5235266089439392, -0.4004882574081421, -0.2910638153553009,
          -0.1900092959403992, -0.0938529595732689, 0.0, 0.0887671709060669, 0.1794802695512772, 0.2743096053600311,
          0.3760197460651398, 0.4886530041694641, 0.6188603639602661, 0.7791395783424377, 1.0]
DEVICE = "cuda"
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
ACTS = ["silu", "silu", "gelu_tanh", "gelu", "relu"]
IGNORED = -100


def _gated(name, tokens, ffn, cols, block=64, scales="bf16", act="silu", bias=False, pre=False, out="bf16", outliers=0):
    return {"name": name, "op": "gated", "tokens": tokens, "ffn": ffn, "cols": cols, "block": block, "scales": scales, "act": act,
            "bias": bias, "pre": pre, "out": out, "outliers": outliers}


def _backward(name, tokens, ffn, cols, block=64, scales="bf16", act="silu", bias=False, dh="bf16", outliers=0):
    return {"name": name, "op": "backward", "tokens": tokens, "ffn": ffn, "cols": cols, "block": block, "scales": scales, "act": act,
            "bias": bias, "dh": dh, "outliers": outliers}


def _loss(name, tokens, vocab, cols, block=64, scales="bf16", grad=False, outliers=0):
    return {"name": name, "op": "loss", "tokens": tokens, "vocab": vocab, "cols": cols, "block": block, "scales": scales, "grad": grad,
            "outliers": outliers}


def listed():
    return [
        # One token through the block of the 7B shape: a decoder's step for a single sequence.
        _gated("gated_1_11008x4096", 1, 11008, 4096),
        # Eleven sequences in flight through the 8B shape's block, larger quantisation blocks, fp32 results.
        _gated("gated_11_14336x4096", 11, 14336, 4096, block=128, scales="f32", act="gelu_tanh", out="f32"),
        # Fifty-three sequences (or a short prompt) through the 70B shape's block with its outliers preserved.
        _gated("gated_53_28672x8192_opq", 53, 28672, 8192, outliers=1 << 18),
        # A prompt, no multiple of anything, biased.
        _gated("gated_777_11008x4096", 777, 11008, 4096, block=32, act="gelu", bias=True),
        # A training batch through the 8B shape's block, its products kept for the backward pass.
        _gated("gated_4096_14336x4096_pre", 4096, 14336, 4096, pre=True),
        # Gradients of a short batch.
        _backward("backward_131_11008x4096", 131, 11008, 4096, scales="f32", bias=True),
        # Gradients of that training batch.
        _backward("backward_4096_14336x4096", 4096, 14336, 4096),
        # The score of one token under a vocabulary of 32000.
        _loss("loss_1_32000x4096", 1, 32000, 4096),
        # A few answers of one token each under a large vocabulary, with the gradient.
        _loss("loss_13_128256x4096_grad", 13, 128256, 4096, block=128, grad=True),
        # A short batch, no multiple of anything, through a head with its outliers preserved.
        _loss("loss_501_32000x4096_opq_grad", 501, 32000, 4096, scales="f32", grad=True, outliers=1 << 16),
        # Perplexity of a window of 2048 tokens.
        _loss("loss_2048_128256x4096", 2048, 128256, 4096),
        # A training batch.
        _loss("loss_4096_128256x4096_grad", 4096, 128256, 4096, grad=True),
    ]


def draw(rng):
    """One more case of the same ranges: tokens from 1 to 8192, blocks from small ones to the 70B shape's, vocabularies up to 152,000."""
    span = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))  # noqa: E731
    op = rng.choice(["gated", "gated", "backward", "loss", "loss"])
    block = rng.choice([32, 64, 64, 64, 128, 256, 1024])
    scales = rng.choice(["bf16", "bf16", "f32"])
    tokens, cols = span(1, 8192), block * span(max(1, 512 // block), max(2, 8192 // block))
    if op == "loss":
        vocab = span(1000, 152000)
        while tokens * vocab * cols > 4096 * 128256 * 4096:
            tokens = tokens * 2 // 3
        if rng.random() < 0.5:  # padded vocabularies are common, others exist
            vocab = max(64, vocab // 64 * 64)
        outliers = rng.choice([0, 0, span(1, max(1, vocab * cols // 1500))])
        return {**_loss("", tokens, vocab, cols, block, scales, rng.random() < 0.6, outliers if vocab * cols < 2 ** 31 else 0), "name": "loss drawn"}
    ffn = span(256, 28672)
    while ffn * cols > 28672 * 8192 or tokens * ffn * cols > 4096 * 14336 * 4096:
        tokens, ffn = max(1, tokens * 2 // 3), max(32, ffn * 4 // 5)
    if rng.random() < 0.7:
        ffn = max(8, ffn // 8 * 8)
    outliers = rng.choice([0, 0, span(1, max(1, ffn * cols // 750))])
    act, bias = rng.choice(ACTS), rng.random() < 0.3
    if op == "backward":
        return {**_backward("", tokens, ffn, cols, block, scales, act, bias, rng.choice(["bf16", "bf16", "f32"]), outliers), "name": "backward drawn"}
    return {**_gated("", tokens, ffn, cols, block, scales, act, bias, rng.random() < 0.5, rng.choice(["bf16", "bf16", "f32"]), outliers), "name": "gated drawn"}


# ---------------------------------------------------------------- inputs


def _quantised(n, block, scales, gen):
    """Codes of near-Gaussian normalised weights, even element in the high nibble, and signed block constants."""
    levels = torch.tensor(LEVELS, device=DEVICE)
    codes = torch.bucketize(torch.randn(n, device=DEVICE, generator=gen).mul_(0.4), (levels[1:] + levels[:-1]) / 2, out_int32=True)
    codes = codes.to(torch.uint8).view(-1, 2)
    blocks = n // block
    m = 0.05 + 0.01 * torch.rand(blocks, device=DEVICE, generator=gen)
    sign = torch.randint(0, 2, (blocks,), device=DEVICE, generator=gen) * 2 - 1
    return (codes[:, 0] << 4) | codes[:, 1], (m * sign).to(DTYPE[scales])


def _outliers(n, count, gen):
    idx = torch.unique(torch.randint(0, n, (count,), device=DEVICE, generator=gen, dtype=torch.int64)).to(torch.int32)
    val = (0.2 + 0.6 * torch.rand(idx.numel(), device=DEVICE, generator=gen)) * (torch.randint(0, 2, idx.shape, device=DEVICE, generator=gen) * 2 - 1)
    return idx, val.to(torch.bfloat16), torch.tensor([idx.numel()], device=DEVICE)


def _normal(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(*shape, device=DEVICE, generator=gen) * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = {"case": case, "levels": torch.tensor(LEVELS, device=DEVICE)}
    t, cols = case["tokens"], case["cols"]
    rows = case["vocab"] if case["op"] == "loss" else 2 * case["ffn"]
    s["codes"], s["scales"] = _quantised(rows * cols, case["block"], case["scales"], gen)
    s["outliers"] = _outliers(rows * cols, case["outliers"], gen) if case["outliers"] else None
    if case["op"] == "backward":
        s["dh"] = _normal(gen, t, case["ffn"], scale=0.01, dtype=DTYPE[case["dh"]])
        s["pre"] = _normal(gen, t, rows)
        return s
    if case["op"] == "gated":
        s["x"] = _normal(gen, t, cols)
        s["bias"] = _normal(gen, rows, dtype=DTYPE[case["out"]], scale=0.1) if case["bias"] else None
        return s
    # Hidden states of a model that has learned something: a part of each points along its target's row, so that targets have
    # probabilities from next to nothing to next to one.  Some targets are ignored (prompts, padding); the mean is what is trained on.
    targets = torch.randint(0, rows, (t,), device=DEVICE, generator=gen)
    row = _rows(s["codes"], s["scales"], case["block"], s["levels"], targets, cols)
    along = 12.0 * torch.rand(t, 1, device=DEVICE, generator=gen) / row.norm(dim=1, keepdim=True)
    s["x"] = (torch.randn(t, cols, device=DEVICE, generator=gen) + along * row).to(torch.bfloat16)
    ignored = torch.rand(t, device=DEVICE, generator=gen) < 0.1
    ignored[0] = False
    s["targets"] = targets.masked_fill(ignored, IGNORED)
    s["dloss"] = (1.0 / (~ignored).sum().float()).expand(t).contiguous()
    return s


# ---------------------------------------------------------------- plain forms


def _rows(codes, scales, block, levels, rows, cols):
    pairs = codes.view(-1, cols // 2)[rows]
    values = levels[torch.stack((pairs >> 4, pairs & 15), dim=-1).int()].view(len(rows), cols // block, block)
    return (values * scales.view(-1, cols // block)[rows].float()[:, :, None]).to(torch.bfloat16).float().view(len(rows), cols)


def _weights(codes, scales, block, levels, outliers=None):
    """The dequantised weights as fp32, flat: bf16(constant * level), outliers in their places."""
    pairs = torch.stack((codes >> 4, codes & 15), dim=-1).view(-1, block)
    w = (levels[pairs.int()] * scales.float()[:, None]).to(torch.bfloat16).float().view(-1)
    if outliers is not None:
        w[outliers[0].long()] = outliers[1].float()
    return w


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z))


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        u = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + u) + 0.5 * z * (1 - u * u) * a * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def run(state):
    s, case = state, state["case"]
    if own:
        return _own(s, case)
    rows = case["vocab"] if case["op"] == "loss" else 2 * case["ffn"]
    w = _weights(s["codes"], s["scales"], case["block"], s["levels"], s["outliers"]).view(rows, case["cols"])
    if case["op"] == "gated":
        z = s["x"].float() @ w.T
        if s["bias"] is not None:
            z = z + s["bias"].float()
        h = _act(z[:, :case["ffn"]], case["act"]) * z[:, case["ffn"]:]
        out = {"h": h.to(DTYPE[case["out"]])}
        if case["pre"]:
            out["pre"] = z.to(torch.bfloat16)
        return out
    if case["op"] == "backward":
        dh, g, u = s["dh"].float(), s["pre"][:, :case["ffn"]].float(), s["pre"][:, case["ffn"]:].float()
        dz = torch.cat((dh * u * _slope(g, case["act"]), dh * _act(g, case["act"])), dim=1)
        out = {"dx": (dz @ w).to(torch.bfloat16)}
        if case["bias"]:
            out["dbias"] = dz.sum(dim=0)
        return out
    keep = s["targets"] >= 0
    target = torch.where(keep, s["targets"], 0)[:, None]
    logits = s["x"].float() @ w.T
    top = logits.max(dim=1, keepdim=True).values
    p = torch.exp(logits - top)
    total = p.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    out = {"loss": torch.where(keep, lse - logits.gather(1, target)[:, 0], 0.0), "lse": lse}
    if case["grad"]:
        p = p / total
        p.scatter_add_(1, target, torch.full_like(top, -1.0))
        out["dx"] = ((p * (s["dloss"] * keep)[:, None]) @ w).to(torch.bfloat16)
    return out


# ---------------------------------------------------------------- the library's calls


def _own(s, case):
    import paper_2505_06653_b200 as bof4

    matrix = (s["codes"], s["scales"])
    if case["op"] == "loss":
        loss, lse, dx, _ = bof4.bof4_cross_entropy(*matrix, case["vocab"], case["cols"], case["block"], s["levels"], s["x"], s["targets"],
                                                   dloss=s["dloss"] if case["grad"] else None, want_dx=case["grad"], outliers=s["outliers"])
        return {"loss": loss, "lse": lse, "dx": dx} if case["grad"] else {"loss": loss, "lse": lse}
    act = {"relu": bof4.ACT_RELU, "gelu": bof4.ACT_GELU, "gelu_tanh": bof4.ACT_GELU_TANH, "silu": bof4.ACT_SILU}[case["act"]]
    if case["op"] == "backward":
        dx, dbias, _ = bof4.bof4_gated_backward(*matrix, case["ffn"], case["cols"], case["block"], s["levels"], s["dh"], s["pre"],
                                                activation=act, want_dbias=case["bias"], outliers=s["outliers"])
        return {"dx": dx, "dbias": dbias} if case["bias"] else {"dx": dx}
    pre = torch.empty(case["tokens"], 2 * case["ffn"], dtype=torch.bfloat16, device=DEVICE) if case["pre"] else None
    h, _ = bof4.bof4_gated(*matrix, case["ffn"], case["cols"], case["block"], s["levels"], s["x"], bias=s["bias"], activation=act,
                           out_dtype=bof4.BF16 if case["out"] == "bf16" else bof4.F32, pre=pre, outliers=s["outliers"])
    return {"h": h, "pre": pre} if case["pre"] else {"h": h}


# ---------------------------------------------------------------- floors and 64-bit values


def work(case):
    """Bytes and operations that a pass cannot do without: the weights once, inputs and outputs once, each product once."""
    t, cols, o = case["tokens"], case["cols"], case["op"]
    rows = case["vocab"] if o == "loss" else 2 * case["ffn"]
    b = rows * cols * (0.5 + BYTES[case["scales"]] / case["block"]) + 6 * case["outliers"] + 2 * t * cols
    if o == "gated":
        return {"bytes": b + BYTES[case["out"]] * (t * case["ffn"] + (rows if case["bias"] else 0)) + (2 * t * rows if case["pre"] else 0),
                "flops": 2 * t * rows * cols}
    if o == "backward":
        return {"bytes": b + BYTES[case["dh"]] * t * case["ffn"] + 2 * t * rows + (4 * rows if case["bias"] else 0), "flops": 2 * t * rows * cols}
    return {"bytes": b + 16 * t + ((2 * cols + 4) * t if case["grad"] else 0), "flops": (4 if case["grad"] else 2) * t * rows * cols}


def _act64(z, act):
    """Activation and its derivative in 64 bits."""
    if act == "relu":
        return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).to(z.dtype)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    u = torch.tanh(c * (z + 0.044715 * z ** 3))
    return z * (1 + u) / 2, (1 + u) / 2 + z / 2 * (1 - u ** 2) * c * (1 + 3 * 0.044715 * z ** 2)


def _dense64(codes, scales, block, rows, cols, outliers):
    """A 4-bit matrix in 64 bits, from the nibbles one by one."""
    level = torch.tensor(LEVELS, dtype=torch.float32, device=DEVICE)
    w = torch.empty(rows * cols, dtype=torch.float32, device=DEVICE)
    w[0::2] = level[torch.div(codes, 16, rounding_mode="floor").int()]
    w[1::2] = level[torch.remainder(codes, 16).int()]
    w = (w * torch.repeat_interleave(scales.float(), block)).bfloat16().double()   # one fp32 product, rounded to bf16
    if outliers is not None:
        w.index_copy_(0, outliers[0].long(), outliers[1].double())
    return w.view(rows, cols)


def exact(case, seed):
    s = prepare(case, seed)
    t, cols, f = case["tokens"], case["cols"], case.get("ffn")
    rows = case["vocab"] if case["op"] == "loss" else 2 * f
    w = _dense64(s["codes"], s["scales"], case["block"], rows, cols, s["outliers"])
    if case["op"] == "gated":
        z = torch.einsum("tc,rc->tr", s["x"].double(), w)
        if s["bias"] is not None:
            z = z + s["bias"].double()
        out = {"h": _act64(z[:, :f], case["act"])[0] * z[:, f:]}
        return {**out, "pre": z} if case["pre"] else out
    if case["op"] == "backward":
        dh = s["dh"].double()
        a, slope = _act64(s["pre"][:, :f].double(), case["act"])
        dz = torch.empty(t, rows, dtype=torch.float64, device=DEVICE)
        dz[:, :f] = dh * s["pre"][:, f:].double() * slope
        dz[:, f:] = dh * a
        out = {"dx": torch.einsum("tr,rc->tc", dz, w)}
        return {**out, "dbias": torch.einsum("tr->r", dz)} if case["bias"] else out
    loss, lse, dx = [], [], []
    for i in range(0, t, 512):
        x, target = s["x"][i:i + 512].double(), s["targets"][i:i + 512]
        n, keep = torch.arange(len(x), device=DEVICE), target != IGNORED
        at = torch.clamp(target, min=0)
        z = torch.einsum("tc,rc->tr", x, w)
        # the other rows against the target's own: nothing cancels where the target has next to all of the probability
        d = z - z[n, at][:, None]
        d[n, at] = -math.inf
        rest = torch.logsumexp(d, dim=1)
        lse.append(torch.logsumexp(z, dim=1))
        loss.append(torch.where(keep, torch.logaddexp(rest, torch.zeros_like(rest)), 0.0))
        if case["grad"]:
            g = torch.exp(z - lse[-1][:, None])
            g[n, at] = -torch.exp(rest - torch.logaddexp(rest, torch.zeros_like(rest)))
            dx.append(torch.einsum("tr,rc->tc", g * (s["dloss"][i:i + 512].double() * keep)[:, None], w))
    out = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    return {**out, "dx": torch.cat(dx)} if case["grad"] else out
