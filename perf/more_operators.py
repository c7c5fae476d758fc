"""Cases of the feed-forward projections of a deep sliced GCN (one or two matrix products per slice with bias, activation, gate and
residual, and their gradients) and of the AdamW step over its parameters.

Sizes come from the workloads of `paper_2408_11500_b200.synth`: tiny (2,708 nodes, 1,433 columns, hidden 16, 4 slices),
citation (169,343 nodes, hidden 256, 8 slices, 40 classes), social (232,965 nodes, 602 columns) and co-purchase
(2,449,029 nodes, 100 columns, hidden 256, 8 slices, 47 classes); inner widths are two or four times the hidden width.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256                          # elements of a tensor that share a scale of their 8-bit states
MAX_FLOPS, MAX_FLOPS_FP32, MAX_BYTES = 5.4e11, 1.6e11, 3.6e9      # largest drawn projection
LEAST_NORMAL = 1.17549435e-38


def listed():
    return [
        # serving: one node that has just arrived goes through the inner projection of a block
        {"name": "gated_fwd_one", "op": "ffn_fwd", "n": 1, "p": 1, "in_s": 256, "out_s": 1024, "gated": True, "act": "silu", "dtype": "bf16", "residual": False, "scale": 1.0, "pad": 1},
        # inner projection of a block of the citation model, bf16
        {"name": "gated_fwd_citation", "op": "ffn_fwd", "n": 169_343, "p": 1, "in_s": 256, "out_s": 1024, "gated": True, "act": "silu", "dtype": "bf16", "residual": False, "scale": 1.0, "pad": 1},
        # the same per slice on the co-purchase graph: eight slices of 32 columns, each to 64
        {"name": "gated_fwd_copurchase", "op": "ffn_fwd", "n": 2_449_029, "p": 8, "in_s": 32, "out_s": 64, "gated": True, "act": "gelu", "dtype": "bf16", "residual": False, "scale": 1.0, "pad": 1},
        # gradients of the citation block's inner projection
        {"name": "gated_bwd_citation", "op": "ffn_bwd", "n": 169_343, "p": 1, "in_s": 256, "out_s": 1024, "gated": True, "act": "silu", "dtype": "bf16", "grad": "bf16", "scale": 1.0, "pad": 1},
        # fp32 storage (the framework's default) on the social graph's 602 input columns
        {"name": "gated_bwd_social", "op": "ffn_bwd", "n": 232_965, "p": 1, "in_s": 602, "out_s": 128, "gated": True, "act": "silu", "dtype": "fp32", "grad": "fp32", "scale": 1.0, "pad": 8},
        # outer projection of the citation block with the residual stream added
        {"name": "linear_fwd_citation", "op": "ffn_fwd", "n": 169_343, "p": 1, "in_s": 1024, "out_s": 256, "gated": False, "act": "none", "dtype": "bf16", "residual": True, "scale": 0.5, "pad": 1},
        # a generic wide block, where arithmetic is all there is
        {"name": "linear_fwd_wide", "op": "ffn_fwd", "n": 16_384, "p": 1, "in_s": 4096, "out_s": 4096, "gated": False, "act": "gelu", "dtype": "bf16", "residual": True, "scale": 1.0, "pad": 1},
        # gradients of the citation block's outer projection
        {"name": "linear_bwd_citation", "op": "ffn_bwd", "n": 169_343, "p": 1, "in_s": 1024, "out_s": 256, "gated": False, "act": "none", "dtype": "bf16", "grad": "bf16", "scale": 0.5, "pad": 1},
        # gradients of a first projection of the tiny graph: 1,433 fp32 columns, no width or stride a multiple of four
        {"name": "linear_bwd_tiny", "op": "ffn_bwd", "n": 2_708, "p": 1, "in_s": 1433, "out_s": 16, "gated": False, "act": "gelu", "dtype": "fp32", "grad": "fp32", "scale": 1.0, "pad": 1},
        # update of the citation model, clipped by the norm of its gradients
        {"name": "adamw_citation", "op": "adamw", "table": 0, "in_d": 128, "hidden": 256, "layers": 3, "p": 8, "classes": 40, "grad": "fp32", "states": "fp32", "copy": False, "clip": True, "decay": 0.01, "done": 999},
        # the co-purchase model with a learned vector per node
        {"name": "adamw_copurchase", "op": "adamw", "table": 2_449_029, "in_d": 100, "hidden": 256, "layers": 3, "p": 8, "classes": 47, "grad": "fp32", "states": "fp32", "copy": False, "clip": True, "decay": 0.01, "done": 99},
        # the same with states of 8 bits, bf16 gradients, and the bf16 weights that the next step reads
        {"name": "adamw_8bit_copurchase", "op": "adamw", "table": 2_449_029, "in_d": 100, "hidden": 256, "layers": 3, "p": 8, "classes": 47, "grad": "bf16", "states": "q8", "copy": True, "clip": False, "decay": 0.01, "done": 99},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["ffn_fwd", "ffn_fwd", "ffn_bwd", "ffn_bwd", "adamw"])
    if op == "adamw":
        in_d = _log_int(rng, 8, 1433)
        return {"op": op, "table": rng.choice([0, _log_int(rng, 10, min(2_449_029, 240_000_000 // in_d))]), "in_d": in_d, "hidden": _log_int(rng, 16, 1024),
                "layers": rng.randint(1, 6), "p": rng.choice([1, 2, 4, 8]), "classes": _log_int(rng, 2, 128), "grad": rng.choice(["fp32", "bf16"]),
                "states": rng.choice(["fp32", "q8"]), "copy": rng.random() < 0.4, "clip": rng.random() < 0.5, "decay": rng.choice([0.0, 0.01, 0.1]),
                "done": _log_int(rng, 1, 20_000) - 1}
    p = rng.choice([1, 1, 2, 4, 8])
    case = {"op": op, "n": 1, "p": p, "in_s": _log_int(rng, 4, 4096 // p), "out_s": _log_int(rng, 4, 4096 // p), "gated": rng.random() < 0.5,
            "act": rng.choice(["silu", "gelu", "relu", "none"]), "dtype": rng.choice(["bf16", "bf16", "fp32"]), "scale": round(rng.uniform(0.2, 1.0), 3),
            "pad": rng.choice([1, 8])}
    if op == "ffn_fwd":
        case["residual"] = rng.random() < 0.5
    else:
        case["grad"] = "fp32" if case["dtype"] == "fp32" else rng.choice(["bf16", "bf16", "fp32"])
        if case["grad"] == "fp32" and case["act"] == "relu":      # a pre-activation within fp32's rounding of zero has either of two gradients
            case["act"] = "silu"
    one, two = work(case), work(dict(case, n=2))
    most = MAX_FLOPS if "fp32" not in (case["dtype"], case.get("grad")) else MAX_FLOPS_FP32
    wide = 8.0 * case["p"] * (case["in_s"] + case["out_s"] * (1 + case["gated"]))      # memory of the plain form
    top = min(2_449_029.0, most / (two["flops"] - one["flops"]), MAX_BYTES / (two["bytes"] - one["bytes"]), 1.6e10 / wide)
    case["n"] = _log_int(rng, 1, max(1, int(top)))
    return case


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand(g, shape, dtype=torch.float32, std=1.0, pad=1):
    """Normal numbers; the leading dimension is a multiple of `pad`, as the framework lays its activations out."""
    c = shape[-1]
    t = torch.randn(shape[:-1] + (-(-c // pad) * pad,), generator=g, device="cuda", dtype=dtype)
    return t.mul_(std)[..., :c]


def _empty(n, c, dtype, pad):
    return torch.empty((n, -(-c // pad) * pad), device="cuda", dtype=dtype)[:, :c]


def _param_shapes(case):
    """Tensors of a sliced model (per-layer tensors are stacked over the slices), after the embedding table; and whether each decays."""
    p, hid, h_s, w = case["p"], case["hidden"], -(-case["hidden"] // case["p"]), -(-case["in_d"] // case["p"])
    shapes = [(case["table"] * case["in_d"], True)] if case["table"] else []
    for layer in range(case["layers"]):
        k = w if layer == 0 else h_s
        shapes += [(p * k * h_s, True), (p * k * h_s, True), (p * h_s, False)]
    return shapes + [(p * h_s * hid, True), (hid, False), (hid * case["classes"], True), (case["classes"], False)]


def _prepare_adamw(case, g, s):
    """One buffer each for parameters, gradients and states; every tensor starts at a multiple of BLOCK elements of it, the rest is zero."""
    shapes = _param_shapes(case)
    blocks = [-(-e // BLOCK) for e, _ in shapes]
    first = [sum(blocks[:i]) for i in range(len(blocks))]
    nb = sum(blocks)
    dev = {"device": "cuda"}
    counts = torch.tensor(blocks, **dev)
    place = torch.arange(nb, **dev) - torch.repeat_interleave(torch.tensor(first, **dev), counts, output_size=nb)   # of a block within its tensor
    lane = torch.arange(BLOCK, **dev)
    inside = place[:, None] * BLOCK + lane < torch.repeat_interleave(torch.tensor([e for e, _ in shapes], **dev), counts, output_size=nb)[:, None]
    s["place"], s["decayed"] = place, torch.repeat_interleave(torch.tensor([d for _, d in shapes], **dev), counts, output_size=nb)
    s["slots"] = [(f * BLOCK, e) for f, (e, _) in zip(first, shapes)]
    s["decays"] = [d for _, d in shapes]

    def flat(dtype, std):
        return torch.randn((nb, BLOCK), generator=g, dtype=dtype, **dev).mul_(std).mul_(inside)
    s["p"], s["g"] = flat(torch.float32, 0.05), flat(TYPES[case["grad"]], 1e-3)
    if case["states"] == "fp32":
        s["m"], s["v"] = flat(torch.float32, 3e-4), flat(torch.float32, 1e-3).square_()
    else:
        s["m"] = (torch.randn((nb, BLOCK), generator=g, **dev) * 40.0).round_().clamp_(-127, 127).mul_(inside).to(torch.int8)
        s["v"] = (torch.randn((nb, BLOCK), generator=g, **dev).abs_() * 85.0).ceil_().clamp_(1, 255).mul_(inside).to(torch.uint8)
        s["m_scale"] = torch.rand(nb, generator=g, **dev).add_(0.5).mul_(1e-3 / 127)
        s["v_scale"] = torch.rand(nb, generator=g, **dev).add_(0.5).mul_(3e-3 / 255)
    if case["copy"]:
        s["copy"] = torch.zeros((nb, BLOCK), dtype=torch.bfloat16, **dev)
    s["step"] = torch.tensor([case["done"], 0], dtype=torch.int64, **dev)
    if case["clip"]:      # the norm that the clipping call leaves on the device, without clipped gradients
        s["norm"] = s["g"].float().square_().sum().sqrt_().reshape(1)
        s["max_norm"] = 0.5 * 1e-3 * math.sqrt(sum(e for e, _ in shapes))
    return s


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case, "stream": torch.cuda.current_stream().cuda_stream}
    if case["op"] == "adamw":
        return _prepare_adamw(case, g, s)
    n, p, ins, outs, dt, pad = case["n"], case["p"], case["in_s"], case["out_s"], TYPES[case["dtype"]], case["pad"]
    s["x"] = _rand(g, (n, p * ins), dt, pad=pad)
    for w, b in (("W", "b"), ("W2", "b2"))[:1 + case["gated"]]:
        s[w] = _rand(g, (p, ins, outs), std=1.0 / math.sqrt(ins)).to(dt)
        s[b] = _rand(g, (p, outs), std=0.1)
    if case["op"] == "ffn_fwd":
        if case["residual"]:
            s["r"] = _rand(g, (n, p * outs), dt, pad=pad)
        s["out"] = _empty(n, p * outs, dt, pad)
    else:
        gt = TYPES[case["grad"]]
        s["dout"] = _rand(g, (n, p * outs), gt, 1e-3, pad=pad)
        s["dx"] = _empty(n, p * ins, gt, pad)
        for w, b in (("W", "b"), ("W2", "b2"))[:1 + case["gated"]]:
            s["d" + w] = torch.empty((p, ins, outs), device="cuda", dtype=gt)
            s["d" + b] = torch.empty((p, outs), device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- one pass

BETA1, BETA2, EPS, LR = 0.9, 0.999, 1e-8, 1e-3
GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


def _act(name, a):
    if name == "none":
        return a
    if name == "relu":
        return torch.clamp(a, min=0.0)
    if name == "silu":
        return a / (1.0 + torch.exp(-a))
    return 0.5 * a * (1.0 + torch.tanh(GELU_A * (a + GELU_B * a * a * a)))


def _act_back(name, a):
    """The activation's derivative."""
    if name == "none":
        return torch.ones_like(a)
    if name == "relu":
        return (a > 0).to(a.dtype)
    if name == "silu":
        q = 1.0 / (1.0 + torch.exp(-a))
        return q * (1.0 + a * (1.0 - q))
    t = torch.tanh(GELU_A * (a + GELU_B * a * a * a))
    return 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * GELU_A * (1.0 + 3.0 * GELU_B * a * a)


def _slices(t, p):
    """n x p*w -> p x n x w in fp32."""
    return t.float().reshape(t.shape[0], p, -1).transpose(0, 1)


def _joined(t):
    """p x n x w -> n x p*w."""
    return t.transpose(0, 1).reshape(t.shape[1], -1)


def _plain_ffn_fwd(s):
    c = s["case"]
    x = _slices(s["x"], c["p"])
    y = _act(c["act"], torch.matmul(x, s["W"].float()) + s["b"][:, None])
    if c["gated"]:
        y = y * (torch.matmul(x, s["W2"].float()) + s["b2"][:, None])
    y = _joined(y) * c["scale"]
    if "r" in s:
        y = y + s["r"].float()
    return {"out": y.to(s["out"].dtype)}


def _plain_ffn_bwd(s):
    c = s["case"]
    x, W, g = _slices(s["x"], c["p"]), s["W"].float(), _slices(s["dout"], c["p"]) * c["scale"]
    a = torch.matmul(x, W) + s["b"][:, None]
    da = g * _act_back(c["act"], a)
    if c["gated"]:
        W2 = s["W2"].float()
        da, dc = da * (torch.matmul(x, W2) + s["b2"][:, None]), g * _act(c["act"], a)
    xt = x.transpose(1, 2)
    dx = torch.matmul(da, W.transpose(1, 2))
    out = {"dW": torch.matmul(xt, da).to(s["dW"].dtype), "db": da.sum(1)}
    if c["gated"]:
        dx = dx + torch.matmul(dc, W2.transpose(1, 2))
        out["dW2"], out["db2"] = torch.matmul(xt, dc).to(s["dW2"].dtype), dc.sum(1)
    out["dx"] = _joined(dx).to(s["dx"].dtype)
    return out


def _thresholds(s, t):
    """Two numbers in [0, 1) for every element, from its place in its tensor and the step: where a state is rounded up."""
    low = 0xFFFFFFFF
    h = (s["place"][:, None] * BLOCK + torch.arange(BLOCK, device="cuda")) * 0x9E3779B1 + t * 0x85EBCA6B
    h = h & low
    h = ((h ^ (h >> 15)) * 0x2C1B3C6D) & low
    h = ((h ^ (h >> 13)) * 0x297A2D39) & low
    h = h ^ (h >> 16)
    return (h & 0xFFFF).float() * 2.0 ** -16, (h >> 16).float() * 2.0 ** -16


def _scale(top, codes):
    """Scale of a block whose largest magnitude is `top`, and what its elements are multiplied by."""
    scale = top / codes
    scale = torch.where(scale < LEAST_NORMAL, 0.0, scale)
    return scale, torch.where(scale > 0, 1.0 / scale, 0.0)


def _plain_adamw(s):
    c = s["case"]
    s["step"][0] += 1
    t = s["step"][0]
    corr1, corr2 = (1.0 - torch.pow(torch.full_like(t, 1, dtype=torch.float64) * b, t.double()) for b in (BETA1, BETA2))
    q8 = c["states"] == "q8"
    g = s["g"].float()
    if "norm" in s:
        norm = s["norm"].double()
        g = g * torch.where((norm > s["max_norm"]) & torch.isfinite(norm), s["max_norm"] / norm, 1.0).float()
    if q8:
        root = s["v"].float() * s["v_scale"][:, None]
        m, v = s["m"].float() * s["m_scale"][:, None], root * root
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * (1.0 - BETA2)) * g
    root = torch.sqrt(v)
    rate = LR / corr1
    shrink = torch.where(s["decayed"], 1.0 - LR * c["decay"], 1.0).to(torch.float32)[:, None]
    s["p"].copy_(s["p"] * shrink - rate.float() * (m / (root / torch.sqrt(corr2).float() + EPS)))
    if q8:
        up_m, up_v = _thresholds(s, t)
        s["m_scale"], inv = _scale(m.abs().amax(1), 127.0)
        s["m"].copy_(torch.floor(m * inv[:, None] + up_m).clamp(-127, 127))
        s["v_scale"], inv = _scale(root.amax(1), 255.0)
        s["v"].copy_(torch.where(root > 0, torch.floor(root * inv[:, None] + up_v).clamp(1, 255), 0.0))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if "copy" in s:
        s["copy"].copy_(s["p"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    """Parameters, states as the values they stand for, and the copy."""
    out = {"p": s["p"], "step": s["step"][:1]}
    if s["case"]["states"] == "q8":
        out["m"], out["root_v"] = s["m"] * s["m_scale"][:, None], s["v"] * s["v_scale"][:, None]
    else:
        out["m"], out["v"] = s["m"], s["v"]
    if "copy" in s:
        out["copy"] = s["copy"]
    return out


PLAIN = {"ffn_fwd": _plain_ffn_fwd, "ffn_bwd": _plain_ffn_bwd, "adamw": _plain_adamw}


def _describe(s):
    """What a program keeps beside its tensors: the description of the call and its scratch memory."""
    from paper_2408_11500_b200 import binding as B
    c, code = s["case"], {"fp32": B.F32, "bf16": B.BF16}
    if c["op"] == "adamw":
        views = {k: [s[k].view(-1)[at:at + e] for at, e in s["slots"]] for k in ("p", "g", "m", "v", "copy") if k in s}
        scales = {k: [s[k][at // BLOCK:at // BLOCK + -(-e // BLOCK)] for at, e in s["slots"]] for k in ("m_scale", "v_scale") if k in s}
        d = B.make_adamw_desc(views["p"], views["g"], views["m"], views["v"], scales.get("m_scale"), scales.get("v_scale"), copies=views.get("copy"),
                              lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=c["decay"], decayed=s["decays"], max_norm=s.get("max_norm", math.inf))
        return B, d, None, 0
    lds = {k + "_ld": s[k].stride(0) for k in ("x", "r", "out", "dout", "dx") if k in s}
    d = B.make_ffn_desc(c["n"], c["p"], c["in_s"], c["out_s"], s["W"], s.get("W2"), s["b"], s.get("b2"),
                        act={"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}[c["act"]], dtype=code[c["dtype"]],
                        grad_dtype=code[c.get("grad", c["dtype"])], scale=c["scale"], **lds)
    need = B.slicegcn_ffn_workspace_bytes(d, s["x"], s.get("dout"))
    return B, d, torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, need


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return PLAIN[op](s)
    if "call" not in s:
        s["call"] = _describe(s)
    B, d, ws, ws_bytes = s["call"]
    if op == "ffn_fwd":
        B.slicegcn_ffn_forward(d, s["x"], s.get("r"), s["out"], None, ws, ws_bytes, s["stream"])
        return {"out": s["out"]}
    if op == "ffn_bwd":
        B.slicegcn_ffn_backward(d, s["x"], s["dout"], s["dx"], s["dW"], s.get("dW2"), s["db"], s.get("db2"), None, ws, ws_bytes, s["stream"])
        return {k: s[k] for k in ("dx", "dW", "dW2", "db", "db2") if k in s}
    B.slicegcn_adamw_step(d, s["step"], s.get("norm"), s["stream"])
    return _adamw_outputs(s)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = {"fp32": 4, "bf16": 2}
    if case["op"] == "adamw":
        e = sum(n for n, _ in _param_shapes(case))
        states = 16 if case["states"] == "fp32" else 4 + 16.0 / BLOCK + 8      # read and written (8 bits: and read as values)
        return {"bytes": e * (8 + size[case["grad"]] + states + (2 if case["copy"] else 0)), "flops": 20 * e}
    n, ins, outs, k = case["n"], case["p"] * case["in_s"], case["p"] * case["out_s"], 1 + case["gated"]
    w, b = k * ins * case["out_s"], size[case["dtype"]]
    product = 2.0 * n * w
    if case["op"] == "ffn_fwd":
        return {"bytes": b * (n * ins + w + n * outs * (1 + case["residual"])) + 4 * k * outs, "flops": product}
    gb = size[case["grad"]]
    again = 1 if case["act"] != "none" or case["gated"] else 0       # the pre-activations
    return {"bytes": b * (n * ins + w) + gb * (n * (ins + outs) + w) + 4 * 2 * k * outs, "flops": product * (2 + again)}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits

def _act64(name, a):
    return {"none": lambda: a, "relu": lambda: a.relu(), "silu": lambda: a * a.sigmoid(), "gelu": lambda: torch.nn.functional.gelu(a, approximate="tanh")}[name]()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        t = case["done"] + 1
        g = s["g"].double()
        if "norm" in s and float(s["norm"]) > s["max_norm"]:
            g = g * (s["max_norm"] / float(s["norm"]))
        q8 = case["states"] == "q8"
        m = s["m"].double() * s["m_scale"][:, None].double() if q8 else s["m"].double()
        v = (s["v"].double() * s["v_scale"][:, None].double()) ** 2 if q8 else s["v"].double()
        m.mul_(BETA1).add_(g, alpha=1.0 - BETA1)
        v.mul_(BETA2).addcmul_(g, g, value=1.0 - BETA2)
        p = s["p"].double()
        p -= p * (LR * case["decay"]) * s["decayed"][:, None]
        p -= LR * (m / (1.0 - BETA1 ** t)) / ((v / (1.0 - BETA2 ** t)).sqrt() + EPS)
        # a code next to a border has no 64-bit value: the states of 8 bits are compared as they are
        return {"p": p, "m": None if q8 else m, **({"root_v": None} if q8 else {"v": v}), **({"copy": p} if case["copy"] else {})}
    n, p, ins, outs = case["n"], case["p"], case["in_s"], case["out_s"]
    names = ("W", "W2")[:1 + case["gated"]]
    leaves = {k: s[k].double().requires_grad_(case["op"] == "ffn_bwd") for k in names + tuple(k.replace("W", "b") for k in names)}
    rows = max(1, (1 << 26) // (p * (ins + outs * (1 + case["gated"]))))

    def block(a, b, x):
        y = _act64(case["act"], torch.einsum("nsi,sio->nso", x.view(b - a, p, ins), leaves["W"]) + leaves["b"])
        if case["gated"]:
            y = y * (torch.einsum("nsi,sio->nso", x.view(b - a, p, ins), leaves["W2"]) + leaves["b2"])
        return y.reshape(b - a, p * outs) * case["scale"]

    if case["op"] == "ffn_fwd":
        out = torch.empty((n, p * outs), device="cuda", dtype=torch.float64)
        for a in range(0, n, rows):
            b = min(n, a + rows)
            out[a:b] = block(a, b, s["x"][a:b].double().contiguous())
            if case["residual"]:
                out[a:b] += s["r"][a:b].double()
        return {"out": out}
    dx = torch.empty((n, p * ins), device="cuda", dtype=torch.float64)
    sums = {k: torch.zeros_like(t) for k, t in leaves.items()}
    for a in range(0, n, rows):          # the gradients of <dout, out> by differentiating the definition
        b = min(n, a + rows)
        x = s["x"][a:b].double().contiguous().requires_grad_(True)
        got = torch.autograd.grad(block(a, b, x), [x] + list(leaves.values()), s["dout"][a:b].double())
        dx[a:b] = got[0]
        for k, t in zip(leaves, got[1:]):
            sums[k] += t
    return {"dx": dx, **{"d" + k: t.detach() for k, t in sums.items()}}
