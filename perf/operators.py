"""Products with quantised weights as a model uses them, as cases that can be prepared and run.

A case is a dict of plain values.  ``op`` says which operator it is:

    linear    bof4_linear: y = act(x W^T + bias) + residual for ``tokens`` rows of x
    backward  bof4_linear_backward: the gradients of x and bias of that product (the weights are frozen)
    moe       bof4_moe: router, choice of ``top_k`` of ``experts``, gated expert products, weighted sum

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
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def _linear(name, tokens, rows, cols, block=64, scales="bf16", act="none", bias=False, residual=False, out="bf16", outliers=0):
    return {"name": name, "op": "linear", "tokens": tokens, "rows": rows, "cols": cols, "block": block, "scales": scales, "act": act,
            "bias": bias, "residual": residual, "out": out, "outliers": outliers}


def _backward(name, tokens, rows, cols, block=64, scales="bf16", act="none", bias=False, outliers=0):
    return {"name": name, "op": "backward", "tokens": tokens, "rows": rows, "cols": cols, "block": block, "scales": scales,
            "act": act, "bias": bias, "outliers": outliers}


def _moe(name, tokens, hidden, ffn, experts, top_k, block=64, scales="bf16", act="silu", score="softmax", renorm=True, out="bf16"):
    return {"name": name, "op": "moe", "tokens": tokens, "hidden": hidden, "ffn": ffn, "experts": experts, "top_k": top_k,
            "block": block, "scales": scales, "act": act, "score": score, "renorm": renorm, "out": out}


def listed():
    return [
        # One token through an attention projection of the 7B shape, added to the residual stream: the smallest call of a decoder.
        _linear("linear_1_4096x4096", 1, 4096, 4096, residual=True),
        # Five sequences (or five drafted tokens) through an MLP matrix of the 7B shape, biased and activated.
        _linear("linear_5_11008x4096_silu", 5, 11008, 4096, block=128, scales="f32", act="silu", bias=True),
        # Two dozen sequences in flight through the 70B shape's MLP matrix with its outliers preserved, fp32 results.
        _linear("linear_24_28672x8192_opq", 24, 28672, 8192, out="f32", outliers=1 << 17),
        # A short prompt, no multiple of anything, through an up projection of the 8B shape.
        _linear("linear_201_14336x4096_gelu", 201, 14336, 4096, act="gelu", bias=True),
        # A long prompt or a training batch through the 8B shape's down projection, added to the residual stream.
        _linear("linear_4096_4096x14336", 4096, 4096, 14336, residual=True),
        # Gradients of a short batch through an attention projection.
        _backward("backward_77_4096x4096", 77, 4096, 4096, scales="f32", bias=True),
        # Gradients of a training batch through an activated up projection of the 8B shape (adapters over frozen weights).
        _backward("backward_2048_14336x4096_silu", 2048, 14336, 4096, act="silu", bias=True),
        # One token through a layer of many small experts.
        _moe("moe_1_2048_e64", 1, 2048, 1408, 64, 6),
        # Four sequences, few large experts.
        _moe("moe_4_4096_e8", 4, 4096, 4096, 8, 2, block=128),
        # Nineteen sequences over many experts: most experts are read, each for one or two tokens; scores by the logistic function.
        _moe("moe_19_2048_e128", 19, 2048, 768, 128, 8, scales="f32", score="sigmoid", out="f32"),
    ]


def draw(rng):
    """One more case of the same ranges: tokens from 1 to 4096, matrices from a few rows to those of the 70B shape."""
    span = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))  # noqa: E731
    op = rng.choice(["linear", "linear", "linear", "backward", "backward", "moe", "moe"])
    block = rng.choice([32, 64, 64, 64, 128, 256, 1024])
    scales = rng.choice(["bf16", "bf16", "f32"])
    if op == "moe":
        block = min(block, 256)
        unit = max(block, 64)
        hidden, ffn = unit * span(max(1, 512 // unit), 4096 // unit), unit * span(max(1, 256 // unit), 4096 // unit)
        experts = span(4, 128)
        while 3 * hidden * ffn * experts > 5 * 10 ** 8:
            experts = max(4, experts // 2)
            ffn = max(unit, ffn // 2 // unit * unit) if experts == 4 else ffn
        return {**_moe("", span(1, 32), hidden, ffn, experts, min(experts, span(1, 8)), block, scales, rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]),
                       rng.choice(["softmax", "softmax", "sigmoid"]), rng.random() < 0.7, rng.choice(["bf16", "bf16", "f32"])), "name": "moe drawn"}
    tokens, rows, cols = span(1, 4096) if op == "linear" else span(8, 4096), span(64, 28672), block * span(max(1, 512 // block), max(2, 16384 // block))
    while rows * cols > 28672 * 8192 or tokens * rows * cols > 4096 * 4096 * 14336:
        rows, cols = max(32, rows * 2 // 3), max(block, cols * 2 // 3 // block * block)
    # the entry points take any number of rows; most matrices have a multiple of 8
    if rng.random() < 0.7:
        rows = max(8, rows // 8 * 8)
    outliers = rng.choice([0, 0, span(1, max(1, rows * cols // 1500))])
    act, bias = rng.choice(ACTS), rng.random() < 0.5
    if op == "backward":
        return {**_backward("", tokens, rows, cols, block, scales, act, bias, outliers), "name": "backward drawn"}
    return {**_linear("", tokens, rows, cols, block, scales, act, bias, rng.random() < 0.5, rng.choice(["bf16", "bf16", "f32"]), outliers), "name": "linear drawn"}


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
    if case["op"] == "moe":
        t, h, f, e = case["tokens"], case["hidden"], case["ffn"], case["experts"]
        s["gate_up"] = _quantised(e * 2 * f * h, case["block"], case["scales"], gen)
        s["down"] = _quantised(e * h * f, case["block"], case["scales"], gen)
        s["router"] = _normal(gen, e, h, scale=1.5 / math.sqrt(h))
        s["x"] = _normal(gen, t, h)
        return s
    t, rows, cols = case["tokens"], case["rows"], case["cols"]
    s["codes"], s["scales"] = _quantised(rows * cols, case["block"], case["scales"], gen)
    s["outliers"] = _outliers(rows * cols, case["outliers"], gen) if case["outliers"] else None
    if case["op"] == "backward":
        s["dy"] = _normal(gen, t, rows, scale=0.01)
        s["pre"] = _normal(gen, t, rows) if case["act"] != "none" else None
        return s
    out = DTYPE[case["out"]]
    s["x"] = _normal(gen, t, cols)
    s["bias"] = _normal(gen, rows, dtype=out, scale=0.1) if case["bias"] else None
    s["residual"] = _normal(gen, t, rows, dtype=out) if case["residual"] else None
    return s


# ---------------------------------------------------------------- plain forms


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
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        u = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + u) + 0.5 * z * (1 - u * u) * a * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _plain_moe(s, case):
    t, h, f, e = case["tokens"], case["hidden"], case["ffn"], case["experts"]
    x = s["x"].float()
    logits = s["x"].double() @ s["router"].double().T   # 64 bits: two experts may be close
    p = torch.softmax(logits, dim=-1) if case["score"] == "softmax" else 1 / (1 + torch.exp(-logits))
    p, ids = torch.sort(p, dim=-1, descending=True, stable=True)
    p, ids = p[:, :case["top_k"]], ids[:, :case["top_k"]]
    if case["renorm"]:
        p = p / p.sum(dim=-1, keepdim=True)
    p = p.float()
    z = x @ _weights(*s["gate_up"], case["block"], s["levels"]).view(e, 2 * f, h).transpose(1, 2)
    act = _act(z[:, :, :f], case["act"]) * z[:, :, f:]
    o = act @ _weights(*s["down"], case["block"], s["levels"]).view(e, h, f).transpose(1, 2)
    share = torch.zeros(t, e, device=DEVICE).scatter_(1, ids, p)
    y = (share.T[:, :, None] * o).sum(dim=0)
    return {"y": y.to(DTYPE[case["out"]]), "ids": ids.int(), "weights": p}


def run(state):
    s, case = state, state["case"]
    if own:
        return _own(s, case)
    if case["op"] == "moe":
        return _plain_moe(s, case)
    w = _weights(s["codes"], s["scales"], case["block"], s["levels"], s["outliers"]).view(case["rows"], case["cols"])
    if case["op"] == "backward":
        dz = s["dy"].float()
        if s["pre"] is not None:
            dz = dz * _slope(s["pre"].float(), case["act"])
        out = {"dx": (dz @ w).to(torch.bfloat16)}
        if case["bias"]:
            out["dbias"] = dz.sum(dim=0)
        return out
    z = s["x"].float() @ w.T
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(DTYPE[case["out"]])}


# ---------------------------------------------------------------- the library's calls


def _own(s, case):
    import paper_2505_06653_b200 as bof4

    act = {"none": bof4.ACT_NONE, "relu": bof4.ACT_RELU, "gelu": bof4.ACT_GELU, "gelu_tanh": bof4.ACT_GELU_TANH, "silu": bof4.ACT_SILU}[case["act"]]
    if case["op"] == "moe":
        y, ids, weights, _ = bof4.bof4_moe(
            s["x"], s["router"], s["gate_up"], s["down"], case["ffn"], case["block"], s["levels"], case["top_k"], activation=act,
            score=bof4.SCORE_SOFTMAX if case["score"] == "softmax" else bof4.SCORE_SIGMOID, renormalize=case["renorm"],
            out_dtype=bof4.BF16 if case["out"] == "bf16" else bof4.F32)
        return {"y": y, "ids": ids, "weights": weights}
    if case["op"] == "backward":
        dx, dbias, _ = bof4.bof4_linear_backward(s["codes"], s["scales"], case["rows"], case["cols"], case["block"], s["levels"], s["dy"],
                                                 pre=s["pre"], activation=act, want_dbias=case["bias"], outliers=s["outliers"])
        return {"dx": dx, "dbias": dbias} if case["bias"] else {"dx": dx}
    y, _ = bof4.bof4_linear(s["codes"], s["scales"], case["rows"], case["cols"], case["block"], s["levels"], s["x"], bias=s["bias"],
                            residual=s["residual"], activation=act, out_dtype=bof4.BF16 if case["out"] == "bf16" else bof4.F32,
                            outliers=s["outliers"])
    return {"y": y}


# ---------------------------------------------------------------- floors and 64-bit values


def work(case):
    """Bytes and operations that a pass cannot do without (a pass over experts: of those that are expected to be chosen)."""
    per_weight = 0.5 + BYTES[case["scales"]] / case["block"]
    t = case["tokens"]
    if case["op"] == "moe":
        h, f, e, k = case["hidden"], case["ffn"], case["experts"], case["top_k"]
        chosen = e * (1 - (1 - k / e) ** t)
        return {"bytes": 3 * h * f * chosen * per_weight + 2 * e * h + 2 * t * h + t * h * BYTES[case["out"]] + 8 * t * k,
                "flops": 2 * t * (k * 3 * h * f + e * h)}
    rows, cols = case["rows"], case["cols"]
    b = rows * cols * per_weight + 6 * case["outliers"]
    if case["op"] == "backward":
        b += 2 * t * rows * (2 if case["act"] != "none" else 1) + 2 * t * cols + (4 * rows if case["bias"] else 0)
    else:
        o = BYTES[case["out"]]
        b += 2 * t * cols + o * t * rows * (2 if case["residual"] else 1) + (o * rows if case["bias"] else 0)
    return {"bytes": b, "flops": 2 * t * rows * cols}


def _act64(z, act):
    """Activation and its derivative in 64 bits."""
    if act == "none":
        return z, torch.ones_like(z)
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


def _dense64(codes, scales, block, rows, cols):
    """A 4-bit matrix in 64 bits, from the nibbles one by one."""
    level = torch.tensor(LEVELS, dtype=torch.float32, device=DEVICE)
    w = torch.empty(rows * cols, dtype=torch.float32, device=DEVICE)
    w[0::2] = level[torch.div(codes, 16, rounding_mode="floor").long()]
    w[1::2] = level[torch.remainder(codes, 16).long()]
    w = w * torch.repeat_interleave(scales.float(), block)   # one fp32 product, rounded to bf16: the dequantised weight
    return w.bfloat16().double().view(rows, cols)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "moe":
        t, h, f, e, k = case["tokens"], case["hidden"], case["ffn"], case["experts"], case["top_k"]
        x = s["x"].double()
        logits = torch.einsum("th,eh->te", x, s["router"].double())
        score = torch.exp(logits - torch.logsumexp(logits, dim=1, keepdim=True)) if case["score"] == "softmax" else torch.sigmoid(logits)
        order = torch.argsort(-logits, dim=1, stable=True)[:, :k]
        weight = torch.gather(score, 1, order)
        if case["renorm"]:
            weight = weight / weight.sum(1, keepdim=True)
        y = torch.zeros(t, h, dtype=torch.float64, device=DEVICE)
        per1, per2 = 2 * f * h, h * f
        for i in torch.unique(order).tolist():
            c1, m1 = s["gate_up"][0][i * per1 // 2:(i + 1) * per1 // 2], s["gate_up"][1][i * per1 // case["block"]:(i + 1) * per1 // case["block"]]
            c2, m2 = s["down"][0][i * per2 // 2:(i + 1) * per2 // 2], s["down"][1][i * per2 // case["block"]:(i + 1) * per2 // case["block"]]
            tok, slot = torch.nonzero(order == i, as_tuple=True)
            z = x[tok] @ _dense64(c1, m1, case["block"], 2 * f, h).T
            o = (_act64(z[:, :f], case["act"])[0] * z[:, f:]) @ _dense64(c2, m2, case["block"], h, f).T
            y[tok] += weight[tok, slot][:, None] * o
        return {"y": y, "ids": order.int(), "weights": weight}
    t, rows, cols = case["tokens"], case["rows"], case["cols"]
    if 2 * t * rows * cols > 10 ** 14:
        return None
    w = _dense64(s["codes"], s["scales"], case["block"], rows, cols)
    if s["outliers"] is not None:
        w.view(-1).index_copy_(0, s["outliers"][0].long(), s["outliers"][1].double())
    if case["op"] == "backward":
        dz = s["dy"].double()
        if s["pre"] is not None:
            dz = dz * _act64(s["pre"].double(), case["act"])[1]
        out = {"dx": torch.einsum("tr,rc->tc", dz, w)}
        if case["bias"]:
            out["dbias"] = torch.einsum("tr->r", dz)
        return out
    z = torch.einsum("tc,rc->tr", s["x"].double(), w)
    if s["bias"] is not None:
        z = z + s["bias"].double()
    y = _act64(z, case["act"])[0]
    return {"y": y if s["residual"] is None else y + s["residual"].double()}
