"""Cases of the operators around a sliced GCN trained from ids: embedding lookup and its gradient, the normalised, gated
residual step between sliced layers and its gradient, and clipping by the global gradient norm.

Sizes come from the workloads of `paper_2408_11500_b200.synth`: tiny (2,708 nodes, 1,433 columns, hidden 16, 4 slices),
citation (169,343 nodes, 128 columns, hidden 256, 8 slices, 40 classes), social (232,965 nodes, 602 columns) and co-purchase
(2,449,029 nodes, 100 columns, hidden 256, 8 slices, 47 classes).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

MAX_ELEMS = 2_449_029 * 128          # largest embedding matrix of a drawn case
MAX_NORM_BYTES = 6.0e9               # and the largest traffic of a drawn residual step
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # serving: the feature row of one node that has just arrived (bf16 model, fp32 parameters)
        {"name": "embed_fwd_one", "op": "embed_fwd", "n": 1, "vocab": 169_343, "d": 128, "ids": "zipf", "table": "fp32", "out": "bf16", "scale": 1.0},
        # a categorical field of the citation graph looked up as its 128-column input features
        {"name": "embed_fwd_citation", "op": "embed_fwd", "n": 169_343, "vocab": 40_009, "d": 128, "ids": "zipf", "table": "fp32", "out": "fp32", "scale": 11.3137085},
        # one learned vector per node of the co-purchase graph, nodes in another order than the table, stored as bf16 features
        {"name": "embed_fwd_copurchase", "op": "embed_fwd", "n": 2_449_029, "vocab": 2_449_029, "d": 100, "ids": "own", "table": "fp32", "out": "bf16", "scale": 10.0},
        # gradient for the words of the tiny graph, where latency is all there is
        {"name": "embed_bwd_tiny", "op": "embed_bwd", "n": 2_708, "vocab": 1_433, "d": 16, "ids": "zipf", "scale": 4.0},
        # gradient of the citation field above: a few ids hold thousands of rows
        {"name": "embed_bwd_citation", "op": "embed_bwd", "n": 169_343, "vocab": 40_009, "d": 128, "ids": "zipf", "scale": 11.3137085},
        # gradient of a category table of the co-purchase graph, 100 columns (no power of two)
        {"name": "embed_bwd_copurchase", "op": "embed_bwd", "n": 2_449_029, "vocab": 200_003, "d": 100, "ids": "zipf", "scale": 10.0},
        # residual step of the tiny model: four slices of four columns, layer norm, no gate
        {"name": "norm_fwd_tiny", "op": "norm_fwd", "n": 2_708, "p": 4, "h_s": 4, "kind": "layer", "gate": False, "dtype": "fp32", "pad": 1, "scale": 1.0},
        # residual step of the co-purchase model: eight slices of 32 columns in bf16, gated
        {"name": "norm_fwd_copurchase", "op": "norm_fwd", "n": 2_449_029, "p": 8, "h_s": 32, "kind": "rms", "gate": True, "dtype": "bf16", "pad": 1, "scale": 0.5},
        # its gradient on the citation model, fp32 storage, layer norm
        {"name": "norm_bwd_citation", "op": "norm_bwd", "n": 169_343, "p": 8, "h_s": 32, "kind": "layer", "gate": True, "dtype": "fp32", "pad": 1, "scale": 0.5},
        # one unsliced, odd width (602 columns kept at a leading dimension of 608) with bf16 storage
        {"name": "norm_bwd_social", "op": "norm_bwd", "n": 232_965, "p": 1, "h_s": 602, "kind": "rms", "gate": True, "dtype": "bf16", "pad": 8, "scale": 1.0},
        # all gradients of the citation model (a few hundred thousand numbers in 13 tensors)
        {"name": "clip_citation", "op": "clip", "table": 0, "in_d": 128, "hidden": 256, "layers": 3, "p": 8, "classes": 40, "dtype": "fp32", "std": 1e-2, "max_norm": 1.0},
        # the co-purchase model with a learned vector per node
        {"name": "clip_copurchase", "op": "clip", "table": 2_449_029, "in_d": 100, "hidden": 256, "layers": 3, "p": 8, "classes": 47, "dtype": "fp32", "std": 1e-4, "max_norm": 1.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "clip"])
    if op.startswith("embed"):
        d = _log_int(rng, 4, 1433)
        case = {"op": op, "n": _log_int(rng, 1, min(2_449_029, MAX_ELEMS // d)), "vocab": _log_int(rng, 7, min(2_449_029, MAX_ELEMS // d)),
                "d": d, "ids": "zipf", "scale": round(rng.uniform(0.5, 16.0), 3)}
        if rng.random() < 0.25:
            case.update(vocab=max(case["n"], 7), ids="own")
        if op == "embed_fwd":
            case["table"], case["out"] = rng.choice([("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
        return case
    if op.startswith("norm"):
        p = rng.choice([1, 1, 2, 4, 8])
        case = {"op": op, "n": 1, "p": p, "h_s": _log_int(rng, 4, 8192 // p), "kind": rng.choice(["rms", "layer"]), "gate": rng.random() < 0.7,
                "dtype": rng.choice(["fp32", "bf16"]), "pad": rng.choice([1, 8]), "scale": round(rng.uniform(0.1, 1.0), 3)}
        per_row = work(case)["bytes"]
        case["n"] = _log_int(rng, 1, max(1, min(2_449_029, int(MAX_NORM_BYTES / per_row))))
        return case
    in_d = _log_int(rng, 8, 1433)
    return {"op": "clip", "table": rng.choice([0, _log_int(rng, 10, min(2_449_029, 240_000_000 // in_d))]), "in_d": in_d,
            "hidden": _log_int(rng, 16, 1024), "layers": rng.randint(1, 6), "p": rng.choice([1, 2, 4, 8]), "classes": _log_int(rng, 2, 128),
            "dtype": rng.choice(["fp32", "fp32", "bf16"]), "std": 10.0 ** rng.uniform(-6, 0), "max_norm": round(rng.uniform(0.1, 5.0), 3)}


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand(g, shape, dtype=torch.float32, std=1.0, mean=0.0, pad=1):
    """Normal numbers; the leading dimension is a multiple of `pad`, as the framework lays its activations out."""
    n, c = shape
    ld = -(-c // pad) * pad
    t = torch.randn((n, ld), generator=g, device="cuda", dtype=dtype)
    return t.mul_(std).add_(mean)[:, :c]


def _empty(n, c, dtype, pad):
    return torch.empty((n, -(-c // pad) * pad), device="cuda", dtype=dtype)[:, :c]


def _ids(g, case):
    n, vocab = case["n"], case["vocab"]
    if case["ids"] == "own":                        # a row of its own for every position
        ids = torch.randperm(vocab, generator=g, device="cuda")[:n]
    else:                                           # rank r in proportion to log(1 + 1/r), as words and categories come; ranks shuffled over the table
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        rank = torch.exp(u * math.log(vocab + 1.0)).long().sub_(1).clamp_(0, vocab - 1)
        step = next(s for s in (1_000_003, 999_983, 1) if math.gcd(s, vocab) == 1)
        ids = (rank * step + 12_345) % vocab
        if n > 8:                                   # one in a hundred has no category
            ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.01, -1, ids)
    return ids.to(torch.int32)


def _grad_shapes(case):
    """Gradient tensors of a sliced model (per-layer tensors are stacked over the slices), after the embedding table's."""
    p, hid, h_s, w = case["p"], case["hidden"], -(-case["hidden"] // case["p"]), -(-case["in_d"] // case["p"])
    shapes = [(case["table"], case["in_d"])] if case["table"] else []
    for layer in range(case["layers"]):
        k = w if layer == 0 else h_s
        shapes += [(p * k, h_s), (p * k, h_s), (p * h_s, 1)]
    return shapes + [(p * h_s, hid), (hid, 1), (hid, case["classes"]), (case["classes"], 1)]


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    s = {"case": case, "stream": torch.cuda.current_stream().cuda_stream}
    if op == "embed_fwd":
        s["ids"] = _ids(g, case)
        s["table"] = _rand(g, (case["vocab"], case["d"]), TYPES[case["table"]], 0.05)
        s["out"] = torch.empty((case["n"], case["d"]), device="cuda", dtype=TYPES[case["out"]])
    elif op == "embed_bwd":
        s["ids"] = _ids(g, case)
        s["dout"] = _rand(g, (case["n"], case["d"]), std=1e-3)
        s["dtable"] = torch.empty((case["vocab"], case["d"]), device="cuda")
    elif op in ("norm_fwd", "norm_bwd"):
        n, cols, dt, pad = case["n"], case["p"] * case["h_s"], TYPES[case["dtype"]], case["pad"]
        layer = case["kind"] == "layer"
        for name, mean in (("w_post", 1.0), ("w_pre", 1.0)) + ((("b_post", 0.0), ("b_pre", 0.0)) if layer else ()):
            s[name] = _rand(g, (1, cols), std=0.2, mean=mean)[0]
        s["y"] = _rand(g, (n, cols), dt, 0.7, pad=pad)
        if case["gate"]:
            s["gate"] = _rand(g, (n, cols), dt, 1.5, pad=pad)
        if op == "norm_fwd":
            s["x"] = _rand(g, (n, cols), dt, 1.3, pad=pad)
            s["h"], s["u"] = _empty(n, cols, dt, pad), _empty(n, cols, dt, pad)
        else:
            s["h"] = _rand(g, (n, cols), dt, 1.5, pad=pad)
            s["dh"], s["du"] = _rand(g, (n, cols), std=1e-3, pad=pad), _rand(g, (n, cols), std=1e-3, pad=pad)
            s["dx"], s["dy"] = _empty(n, cols, torch.float32, pad), _empty(n, cols, torch.float32, pad)
            if case["gate"]:
                s["dgate"] = _empty(n, cols, torch.float32, pad)
            for name in ("w_post", "w_pre") + (("b_post", "b_pre") if layer else ()):
                s["d" + name] = torch.empty(cols, device="cuda")
    else:
        dt = TYPES[case["dtype"]]
        s["grads"] = [_rand(g, shape, dt, case["std"]) for shape in _grad_shapes(case)]
        s["clipped"] = [torch.empty_like(t) for t in s["grads"]]
        s["norm"] = torch.empty(1, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- one pass

EPS = 1e-5


def _outputs(s):
    names = {"embed_fwd": ("out",), "embed_bwd": ("dtable",), "norm_fwd": ("h", "u"), "clip": ("clipped", "norm"),
             "norm_bwd": ("dx", "dy", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")}[s["case"]["op"]]
    return {k: s[k] for k in names if k in s}


def _per_slice(t, p, h_s):
    return t.float().reshape(t.shape[0], p, h_s)


def _centred(t, kind):
    return t - t.mean(-1, keepdim=True) if kind == "layer" else t


def _normal(t, kind):
    """N(t) and 1 / its scale, over the last axis."""
    c = _centred(t, kind)
    r = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    return c * r, r


def _normal_back(that, r, g, kind):
    """J_N(t)^T g."""
    return r * (_centred(g, kind) - that * (g * that).mean(-1, keepdim=True))


def _plain_embed_fwd(s):
    ids = s["ids"].long()
    rows = s["table"][ids.clamp(min=0)].float() * s["case"]["scale"]
    return {"out": torch.where((ids >= 0)[:, None], rows, 0.0).to(s["out"].dtype)}


def _plain_embed_bwd(s):
    ids = s["ids"].long()
    rows = torch.where((ids >= 0)[:, None], s["dout"] * s["case"]["scale"], 0.0)
    return {"dtable": torch.zeros_like(s["dtable"]).index_add_(0, ids.clamp(min=0), rows)}


def _branch(s, p, h_s):
    """N(y), 1 / its scale, the branch before its gate, and the gate."""
    kind = s["case"]["kind"]
    yhat, ry = _normal(_per_slice(s["y"], p, h_s), kind)
    t = yhat * s["w_post"].view(p, h_s)
    t = t + s["b_post"].view(p, h_s) if "b_post" in s else t
    gate = 1.0 / (1.0 + torch.exp(-_per_slice(s["gate"], p, h_s))) if "gate" in s else None
    return yhat, ry, t, gate


def _plain_norm_fwd(s):
    c = s["case"]
    n, p, h_s = c["n"], c["p"], c["h_s"]
    t, gate = _branch(s, p, h_s)[2:]
    h = _per_slice(s["x"], p, h_s) + c["scale"] * (t if gate is None else gate * t)
    u = _normal(h, c["kind"])[0] * s["w_pre"].view(p, h_s)
    u = u + s["b_pre"].view(p, h_s) if "b_pre" in s else u
    return {"h": h.reshape(n, -1).to(s["h"].dtype), "u": u.reshape(n, -1).to(s["u"].dtype)}


def _plain_norm_bwd(s):
    c = s["case"]
    n, p, h_s, kind = c["n"], c["p"], c["h_s"], c["kind"]
    hhat, rh = _normal(_per_slice(s["h"], p, h_s), kind)
    du = _per_slice(s["du"], p, h_s)
    dx = _per_slice(s["dh"], p, h_s) + _normal_back(hhat, rh, du * s["w_pre"].view(p, h_s), kind)
    yhat, ry, t, gate = _branch(s, p, h_s)
    r = c["scale"] * dx
    dt = r if gate is None else r * gate
    out = {"dx": dx.reshape(n, -1), "dy": _normal_back(yhat, ry, dt * s["w_post"].view(p, h_s), kind).reshape(n, -1),
           "dw_post": (dt * yhat).sum(0).reshape(-1), "dw_pre": (du * hhat).sum(0).reshape(-1)}
    if gate is not None:
        out["dgate"] = (r * t * gate * (1.0 - gate)).reshape(n, -1)
    if kind == "layer":
        out["db_post"], out["db_pre"] = dt.sum(0).reshape(-1), du.sum(0).reshape(-1)
    return out


def _plain_clip(s):
    flat = torch.cat([t.reshape(-1).float() for t in s["grads"]])
    norm = (flat * flat).sum().sqrt()
    limit = s["case"]["max_norm"]
    flat = flat * torch.where((norm > limit) & torch.isfinite(norm), limit / norm, 1.0)
    parts = flat.split([t.numel() for t in s["grads"]])
    return {"clipped": [v.view_as(t).to(t.dtype) for v, t in zip(parts, s["grads"])], "norm": norm.reshape(1)}


PLAIN = {"embed_fwd": _plain_embed_fwd, "embed_bwd": _plain_embed_bwd, "norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "clip": _plain_clip}


def _describe(s):
    """What a program keeps beside its tensors: the description of the call and its scratch memory."""
    from paper_2408_11500_b200 import binding as B
    c, code = s["case"], {"fp32": B.F32, "bf16": B.BF16}
    need = 0
    if c["op"] == "embed_fwd":
        d = B.make_embed_desc(c["n"], c["vocab"], c["d"], scale=c["scale"], table_dtype=code[c["table"]], table_ld=s["table"].stride(0),
                              out_dtype=code[c["out"]], out_ld=s["out"].stride(0))
    elif c["op"] == "embed_bwd":
        d = B.make_embed_desc(c["n"], c["vocab"], c["d"], scale=c["scale"], dout_ld=s["dout"].stride(0), dtable_ld=s["dtable"].stride(0))
        need = B.slicegcn_embed_workspace_bytes(d)
    elif c["op"] in ("norm_fwd", "norm_bwd"):
        lds = {k + "_ld": s[k].stride(0) for k in ("x", "y", "gate", "h", "u", "dh", "du", "dx", "dy", "dgate") if k in s}
        d = B.make_residual_norm_desc(c["n"], c["p"], c["h_s"], kind=B.ROWNORM_LAYER if c["kind"] == "layer" else B.ROWNORM_RMS,
                                      dtype=code[c["dtype"]], eps=EPS, residual_scale=c["scale"], w_post=s["w_post"],
                                      b_post=s.get("b_post"), w_pre=s["w_pre"], b_pre=s.get("b_pre"), **lds)
        if c["op"] == "norm_bwd":
            need = B.slicegcn_residual_norm_workspace_bytes(d)
    else:
        d = B.make_tensor_list(s["grads"], s["clipped"])
        need = B.slicegcn_clip_workspace_bytes()
    return B, d, torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, need


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return PLAIN[op](s)
    if "call" not in s:
        s["call"] = _describe(s)
    B, d, ws, ws_bytes = s["call"]
    if op == "embed_fwd":
        B.slicegcn_embed_forward(d, s["ids"], s["table"], s["out"], None, s["stream"])
    elif op == "embed_bwd":
        B.slicegcn_embed_backward(d, s["ids"], s["dout"], s["dtable"], None, ws, ws_bytes, s["stream"])
    elif op == "norm_fwd":
        B.slicegcn_residual_norm_forward(d, s["x"], s["y"], s.get("gate"), s["h"], s["u"], s["stream"])
    elif op == "norm_bwd":
        B.slicegcn_residual_norm_backward(d, s["y"], s.get("gate"), s["h"], s["dh"], s["du"], s["dx"], s["dy"], s.get("dgate"), s["dw_post"],
                                          s.get("db_post"), s["dw_pre"], s.get("db_pre"), ws, ws_bytes, s["stream"])
    else:
        B.slicegcn_clip_grads(d, s["case"]["max_norm"], s["norm"], ws, ws_bytes, s["stream"])
    return _outputs(s)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def _distinct(case):
    """Table rows that n ids touch, on average."""
    n, vocab = case["n"], case["vocab"]
    if case["ids"] == "own":
        return float(min(n, vocab))
    r = np.arange(1, vocab + 1, dtype=np.float64)
    return float(-np.expm1(n * np.log1p(-np.log1p(1.0 / r) / math.log(vocab + 1.0))).sum())


def work(case):
    op, size = case["op"], {"fp32": 4, "bf16": 2}
    if op == "embed_fwd":
        e = case["n"] * case["d"]
        return {"bytes": 4 * case["n"] + _distinct(case) * case["d"] * size[case["table"]] + e * size[case["out"]], "flops": e}
    if op == "embed_bwd":
        e = case["n"] * case["d"]
        return {"bytes": 4 * case["n"] + 4 * e + 4 * case["vocab"] * case["d"], "flops": 2 * e}
    if op in ("norm_fwd", "norm_bwd"):
        cols = case["p"] * case["h_s"]
        e, b, gate, vectors = case["n"] * cols, size[case["dtype"]], int(case["gate"]), 4 if case["kind"] == "layer" else 2
        if op == "norm_fwd":             # x, y, gate in; h, u out
            return {"bytes": e * b * (4 + gate) + 4 * vectors * cols, "flops": e * (14 + 5 * gate)}
        # y, h, gate, dh, du in; dx, dy, dgate and the vectors' gradients out
        return {"bytes": e * (b * (2 + gate) + 4 * (4 + gate)) + 8 * vectors * cols, "flops": e * (35 + 10 * gate)}
    e = sum(a * b for a, b in _grad_shapes(case))
    return {"bytes": 2 * e * size[case["dtype"]] + 4, "flops": 3 * e}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits

def _norm64(t, layer):
    """(t - mean) / sqrt(variance + eps), or t / sqrt(mean square + eps)."""
    if layer:
        return (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, unbiased=False, keepdim=True) + EPS)
    return t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + EPS)


def _step64(case, s, a, b, x, y, gate, vec):
    """h and a function of h that gives u, for rows a..b and any 64-bit leaves."""
    p, h_s, layer = case["p"], case["h_s"], case["kind"] == "layer"
    shape = (b - a, p, h_s)
    v = _norm64(y.view(shape), layer) * vec["w_post"].view(p, h_s) + (vec["b_post"].view(p, h_s) if layer else 0.0)
    v = v * case["scale"] * (torch.sigmoid(gate.view(shape)) if gate is not None else 1.0)
    h = (x.view(shape) + v).view(b - a, p * h_s)
    return h, lambda t: (_norm64(t.view(shape), layer) * vec["w_pre"].view(p, h_s) + (vec["b_pre"].view(p, h_s) if layer else 0.0)).view(b - a, p * h_s)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "embed_fwd":
        out = torch.zeros((case["n"], case["d"]), device="cuda", dtype=torch.float64)
        at = torch.nonzero(s["ids"] >= 0)[:, 0]
        out[at] = s["table"].double().index_select(0, s["ids"][at].long()) * case["scale"]
        return {"out": out}
    if op == "embed_bwd":
        out = torch.zeros((case["vocab"], case["d"]), device="cuda", dtype=torch.float64)
        at = torch.nonzero(s["ids"] >= 0)[:, 0]
        out.index_put_((s["ids"][at].long(),), s["dout"][at].double(), accumulate=True)
        return {"dtable": out * case["scale"]}
    if op == "clip":
        square = sum(float(t.double().pow(2).sum()) for t in s["grads"])
        norm = math.sqrt(square)
        c = case["max_norm"] / norm if norm > case["max_norm"] and math.isfinite(norm) else 1.0
        return {"clipped": [t.double() * c for t in s["grads"]], "norm": torch.tensor([norm], device="cuda", dtype=torch.float64)}
    n, cols = case["n"], case["p"] * case["h_s"]
    names = [k for k in ("w_post", "b_post", "w_pre", "b_pre") if k in s]
    vec = {k: s[k].double().requires_grad_(op == "norm_bwd") for k in names}
    rows = max(1, (1 << 25) // cols)
    if op == "norm_fwd":
        h, u = (torch.empty((n, cols), device="cuda", dtype=torch.float64) for _ in range(2))
        for a in range(0, n, rows):
            b = min(n, a + rows)
            part = [s[k][a:b].double().contiguous() if k in s else None for k in ("x", "y", "gate")]
            h[a:b], pre = _step64(case, s, a, b, *part, vec)
            u[a:b] = pre(h[a:b])
        return {"h": h, "u": u}
    out = {k: torch.empty((n, cols), device="cuda", dtype=torch.float64) for k in ("dx", "dy", "dgate") if k != "dgate" or "gate" in s}
    out.update({"d" + k: torch.zeros(cols, device="cuda", dtype=torch.float64) for k in names})
    for a in range(0, n, rows):          # the gradients of <dh, h> + <du, u> by differentiating the definition
        b = min(n, a + rows)
        x = torch.zeros((b - a, cols), device="cuda", dtype=torch.float64)
        y = s["y"][a:b].double().contiguous().requires_grad_(True)
        gate = s["gate"][a:b].double().contiguous().requires_grad_(True) if "gate" in s else None
        given = s["h"][a:b].double().contiguous().requires_grad_(True)     # h as it was stored is what u was made of
        branch, pre = _step64(case, s, a, b, x, y, gate, vec)
        du = s["du"][a:b].double()
        pres = [k for k in names if k.endswith("pre")]
        through = torch.autograd.grad(pre(given), [given] + [vec[k] for k in pres], du)
        dx = s["dh"][a:b].double() + through[0]
        posts = [k for k in names if k.endswith("post")]
        leaves = [y] + ([gate] if gate is not None else [])
        back = torch.autograd.grad(branch, leaves + [vec[k] for k in posts], dx)
        out["dx"][a:b], out["dy"][a:b] = dx, back[0]
        if gate is not None:
            out["dgate"][a:b] = back[1]
        for k, v in zip(pres, through[1:]):
            out["d" + k] += v
        for k, v in zip(posts, back[len(leaves):]):
            out["d" + k] += v
    return out
