"""The residual step (norms per slice, gate, residual scale) and its gradient against the definition in 64 bits.

Tolerances, from the arithmetic (u = 2^-24; storage rounding 2^-9 for bf16).  A sum over a slice of w columns is added by
threads that each take at most 32 + w/32 elements in turn and then by a tree of at most 12 levels, so it is off by
T u sum|.| with T = w/32 + 48.  A normalised value t^ = (t - mean) r is then off by less than (T + 12) u H, where
H = |t^| + r (|t| + mean|t|) for the layer norm (the mean's own error) and H = |t^| for the plain one.  Every result below
is a sum of products of such values; with each factor replaced by its H, or by its absolute value, the error is at most
(8 T + 200) u times that sum: at most six factors with T + 12 each and a few single roundings.  Sums over n rows add n u.
"""
import numpy as np
import pytest

U32, UBF = 2.0 ** -24, 2.0 ** -9


def _make(rng, n, p, w, layer, gate, x=True, y=True, odd_rows=True):
    cols = p * w
    d = {"x": 1.3 * rng.standard_normal((n, cols)) if x else None, "y": 0.7 * rng.standard_normal((n, cols)) if y else None,
         "gate": 2.0 * rng.standard_normal((n, cols)) if gate else None}
    if odd_rows and n > 4:
        if y:
            d["y"][1] = 0.0                                # a block that gave nothing
            d["y"][2] = 3.0                                # a constant row: the layer norm's variance is zero
        if gate:
            d["gate"][3, ::2], d["gate"][3, 1::2] = 60.0, -200.0     # closed and open gates
    d["vec"] = {k: rng.standard_normal(cols) * 0.3 + 1.0 for k in ("w_post", "w_pre")}
    d["vec"].update({k: rng.standard_normal(cols) * 0.3 if layer else None for k in ("b_post", "b_pre")})
    return d


def _rounded(d, dt):
    import torch
    cast = (lambda a: torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16).double().numpy()) if dt == "bf16" else (lambda a: a.astype(np.float32).astype(np.float64))
    out = {k: None if d[k] is None else cast(d[k]) for k in ("x", "y", "gate")}
    out["vec"] = {k: None if v is None else v.astype(np.float32).astype(np.float64) for k, v in d["vec"].items()}
    return out


def _normal(t, layer, eps):
    """t^, H, r over the last axis."""
    c = t - t.mean(-1, keepdims=True) if layer else t
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    H = np.abs(c) * r + (r * (np.abs(t) + np.abs(t).mean(-1, keepdims=True)) if layer else 0.0)
    return c * r, H, r


def _sig(g):
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1.0, e) / (1.0 + e), e / (1.0 + e) ** 2


def _vec(d, k, p, w, default):
    v = d["vec"][k]
    return np.full((p, w), default) if v is None else v.reshape(p, w)


def _forward64(d, p, w, layer, s, eps):
    """h, u and their error magnitudes (to be multiplied by (8 T + 200) u)."""
    some = d["x"] if d["x"] is not None else d["y"]
    n = some.shape[0]
    h, mh = np.zeros((n, p, w)), np.zeros((n, p, w))
    if d["x"] is not None:
        h, mh = h + d["x"].reshape(n, p, w), mh + np.abs(d["x"].reshape(n, p, w))
    if d["y"] is not None:
        yhat, Y, _ = _normal(d["y"].reshape(n, p, w), layer, eps)
        g = _sig(d["gate"].reshape(n, p, w))[0] if d["gate"] is not None else 1.0
        wp, bp = _vec(d, "w_post", p, w, 1.0), _vec(d, "b_post", p, w, 0.0)
        h, mh = h + s * g * (yhat * wp + bp), mh + abs(s) * g * (Y * np.abs(wp) + np.abs(bp))
    hhat, H, r = _normal(h, layer, eps)
    wq, bq = _vec(d, "w_pre", p, w, 1.0), _vec(d, "b_pre", p, w, 0.0)
    u = hhat * wq + bq
    # an error of h moves its normal form by at most r (its own + the mean of all) + |h^| r (their root mean square)
    moved = r * (mh + mh.mean(-1, keepdims=True)) + np.abs(hhat) * r * np.sqrt((mh * mh).mean(-1, keepdims=True))
    mu = (H + moved) * np.abs(wq) + np.abs(bq)
    return [a.reshape(n, -1) for a in (h, u, mh, mu)]


def _backward64(d, h, dh, du, p, w, layer, s, eps):
    """Gradients and their error magnitudes."""
    n = (dh if dh is not None else du).shape[0]
    R = lambda a: a.reshape(n, p, w)                                             # noqa: E731
    D, mD = (R(dh).copy(), np.abs(R(dh))) if dh is not None else (np.zeros((n, p, w)), np.zeros((n, p, w)))
    out, mag = {}, {}
    mean = lambda a: a.mean(-1, keepdims=True)                                   # noqa: E731
    if du is not None:
        hhat, H, r = _normal(R(h), layer, eps)
        wq = _vec(d, "w_pre", p, w, 1.0)
        g = R(du) * wq
        D = D + r * (g - (mean(g) if layer else 0.0) - hhat * mean(g * hhat))
        mD = mD + r * (np.abs(g) + mean(np.abs(g)) + H * mean(np.abs(g) * H))
        out["dw_pre"], mag["dw_pre"] = (R(du) * hhat).sum(0), (np.abs(R(du)) * H).sum(0)
        out["db_pre"], mag["db_pre"] = R(du).sum(0), np.abs(R(du)).sum(0)
    out["dx"], mag["dx"] = D, mD
    if d["y"] is not None:
        yhat, Y, ry = _normal(R(d["y"]), layer, eps)
        sg, slope = _sig(R(d["gate"])) if d["gate"] is not None else (1.0, None)
        wp, bp = _vec(d, "w_post", p, w, 1.0), _vec(d, "b_post", p, w, 0.0)
        dt, mt = D * s * sg, mD * abs(s) * sg
        if slope is not None:
            out["dgate"], mag["dgate"] = D * s * slope * (yhat * wp + bp), mD * abs(s) * slope * (Y * np.abs(wp) + np.abs(bp))
        out["dw_post"], mag["dw_post"] = (dt * yhat).sum(0), (mt * Y).sum(0)
        out["db_post"], mag["db_post"] = dt.sum(0), mt.sum(0)
        g, mg = dt * wp, mt * np.abs(wp)
        out["dy"] = ry * (g - (mean(g) if layer else 0.0) - yhat * mean(g * yhat))
        mag["dy"] = ry * (mg + mean(mg) + Y * mean(mg * Y))
    flat = lambda a: a.reshape(-1) if a.ndim == 2 else a.reshape(n, -1)          # noqa: E731
    return {k: flat(v) for k, v in out.items()}, {k: flat(v) for k, v in mag.items()}


def _bound(w):
    return (8 * (w / 32 + 48) + 200) * U32


class _Device:
    """The same step on the GPU; every matrix sits inside a larger one whose other values must not change."""

    def __init__(self, d, n, p, w, layer, dt, s, eps, off=0, pad=0):
        import torch
        from paper_2408_11500_b200 import binding as B
        self.torch, self.B, self.n, self.p, self.w, self.off, self.ld = torch, B, n, p, w, off, off + p * w + pad
        self.type = torch.bfloat16 if dt == "bf16" else torch.float32
        self.d, self.big = d, []
        self.vec = {k: None if v is None else torch.from_numpy(v.astype(np.float32)).cuda() for k, v in d["vec"].items()}
        self.desc = B.make_residual_norm_desc(n, p, w, kind=B.ROWNORM_LAYER if layer else B.ROWNORM_RMS, dtype=B.BF16 if dt == "bf16" else B.F32,
                                              eps=eps, residual_scale=s, **self.vec,
                                              **{k + "_ld": self.ld for k in ("x", "y", "gate", "h", "u", "dh", "du", "dx", "dy", "dgate")})

    def put(self, a, dtype=None):
        if a is None:
            return None
        m = self.empty(dtype or self.type)
        m.copy_(self.torch.from_numpy(a).cuda())
        return m

    def empty(self, dtype=None):
        big = self.torch.full((self.n, self.ld), 5.0, device="cuda", dtype=dtype or self.type)
        part = big[:, self.off:self.off + self.p * self.w]
        part.fill_(float("nan"))
        self.big.append(big)
        return part

    def forward(self, h=True, u=True, in_place=False, stream=None):
        x, y, gate = (self.put(self.d[k]) for k in ("x", "y", "gate"))
        hh = x if in_place else self.empty() if h else None
        uu = self.empty() if u else None
        self.B.slicegcn_residual_norm_forward(self.desc, x, y, gate, hh, uu, stream)
        return hh, uu

    def backward(self, h, dh, du, in_place=False, skip=(), stream=None):
        f = self.torch.float32
        y, gate, h, dh, du = self.put(self.d["y"]), self.put(self.d["gate"]), self.put(h), self.put(dh, f), self.put(du, f)
        have = {"dx": True, "dy": y is not None, "dgate": gate is not None, "dw_post": y is not None, "db_post": y is not None,
                "dw_pre": du is not None, "db_pre": du is not None}
        out = {}
        for k, v in have.items():
            out[k] = None if not v or k in skip else self.empty(f) if k in ("dx", "dy", "dgate") else self.torch.full((self.p * self.w,), float("nan"), device="cuda")
        if in_place:
            out["dx"] = dh
        wsb = self.B.slicegcn_residual_norm_workspace_bytes(self.desc)
        ws = self.torch.randint(0, 256, (max(wsb, 1),), dtype=self.torch.uint8, device="cuda")
        self.B.slicegcn_residual_norm_backward(self.desc, y, gate, h, dh, du, out["dx"], out["dy"], out["dgate"], out["dw_post"], out["db_post"],
                                               out["dw_pre"], out["db_pre"], ws, wsb, stream)
        return {k: v for k, v in out.items() if v is not None}

    def untouched(self):
        for b in self.big:
            assert bool((b[:, :self.off] == 5).all()) and bool((b[:, self.off + self.p * self.w:] == 5).all())


def _close(got, want, mag, factor, u_out=0.0):
    got = got.double().cpu().numpy()
    want = want.astype(np.float32).astype(np.float64)     # a result is an fp32 number: what is far below its range (sigmoid(-200)) is zero
    err, allowed = np.abs(got - want), factor * mag + 2 * u_out * (np.abs(want) + factor * mag)
    assert np.all(err <= allowed), (float(np.max(err - allowed)), float(np.max(err / np.maximum(allowed, 1e-300))))


SHAPES = [(1, 1, 1), (5, 3, 1), (7, 1, 4), (300, 4, 4), (1000, 8, 32), (33, 4, 13), (257, 8, 16), (64, 1, 602), (130, 2, 100), (9, 1, 1024),
          (50, 1, 2000), (3, 1, 8192), (6, 64, 8), (2, 1, 16384), (21, 2, 1433), (40, 3, 171), (1, 1, 5000), (70, 1, 7), (1025, 2, 64),
          (19, 8, 512), (1200, 1, 256), (90, 1, 47)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,p,w", SHAPES)
@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
@pytest.mark.parametrize("dt,gate", [("f32", True), ("bf16", False), ("bf16", True)])
def test_step_and_gradient(n, p, w, layer, dt, gate):
    rng = np.random.default_rng(1000 * p + w)
    s, eps = 0.6, 1e-5
    d = _rounded(_make(rng, n, p, w, layer, gate), dt)
    dev = _Device(d, n, p, w, layer, dt, s, eps)
    h, u, mh, mu = _forward64(d, p, w, layer, s, eps)
    gh, gu = dev.forward()
    f, uo = _bound(w), UBF if dt == "bf16" else U32
    _close(gh, h, mh, f, uo)
    _close(gu, u, mu, f, uo)
    h = gh.double().cpu().numpy()                         # what the gradient starts from is the stored h
    dh, du = (rng.standard_normal((n, p * w)).astype(np.float32).astype(np.float64) for _ in range(2))
    want, mag = _backward64(d, h, dh, du, p, w, layer, s, eps)
    got = dev.backward(h, dh, du)
    assert set(got) == set(want)
    for k in want:
        _close(got[k], want[k], mag[k], f + (n * U32 if k[:2] in ("dw", "db") else 0.0))
    again = dev.backward(h, dh, du)
    assert all(dev.torch.equal(got[k], again[k]) for k in got)


@pytest.mark.gpu
@pytest.mark.parametrize("n,p,w,off,pad", [(100, 1, 602, 0, 6), (100, 8, 32, 8, 8), (77, 4, 13, 1, 2), (65, 2, 100, 3, 5), (12, 1, 4100, 2, 1), (300, 8, 32, 4, 0)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_strides_and_odd_starts(n, p, w, off, pad, dt):
    rng = np.random.default_rng(w)
    d = _rounded(_make(rng, n, p, w, True, True), dt)
    dev = _Device(d, n, p, w, True, dt, 1.0, 1e-5, off=off, pad=pad)
    h, u, mh, mu = _forward64(d, p, w, True, 1.0, 1e-5)
    gh, gu = dev.forward()
    f, uo = _bound(w), UBF if dt == "bf16" else U32
    _close(gh, h, mh, f, uo)
    _close(gu, u, mu, f, uo)
    h = gh.double().cpu().numpy()
    dh, du = (rng.standard_normal((n, p * w)).astype(np.float32).astype(np.float64) for _ in range(2))
    want, mag = _backward64(d, h, dh, du, p, w, True, 1.0, 1e-5)
    got = dev.backward(h, dh, du)
    for k in want:
        _close(got[k], want[k], mag[k], f + (n * U32 if k[:2] in ("dw", "db") else 0.0))
    dev.untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("n,p,w", [(300, 8, 32), (50, 1, 602), (17, 2, 3000)])
@pytest.mark.parametrize("parts", ["norm before alone", "norm after alone", "no residual", "only u", "no vectors"])
def test_parts_of_the_step(n, p, w, parts):
    rng = np.random.default_rng(w + len(parts))
    layer, s, eps = True, 0.5, 1e-6
    d = _make(rng, n, p, w, layer, gate=parts == "norm after alone", x=parts != "no residual", y=parts != "norm before alone")
    if parts == "no vectors":
        d["vec"] = dict.fromkeys(d["vec"])
    d = _rounded(d, "f32")
    dev = _Device(d, n, p, w, layer, "f32", s, eps)
    h, u, mh, mu = _forward64(d, p, w, layer, s, eps)
    with_h, with_u = parts not in ("only u", "norm before alone"), parts != "norm after alone"
    gh, gu = dev.forward(h=with_h, u=with_u)
    f = _bound(w)
    if with_h:
        _close(gh, h, mh, f, U32)
    if with_u:
        _close(gu, u, mu, f, U32)
    h = h.astype(np.float32).astype(np.float64)
    dh, du = (rng.standard_normal((n, p * w)).astype(np.float32).astype(np.float64) for _ in range(2))
    dh, du = None if parts in ("only u", "norm before alone") else dh, du if with_u else None
    want, mag = _backward64(d, h, dh, du, p, w, layer, s, eps)
    for skip in ((), ("dx",), ("dy", "dw_post"), ("dw_post", "db_post", "dw_pre", "db_pre")):
        got = dev.backward(h if du is not None else None, dh, du, skip=skip)
        assert set(got) == set(want) - set(skip)
        for k in got:
            _close(got[k], want[k], mag[k], f + (n * U32 if k[:2] in ("dw", "db") else 0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("n,p,w,dt", [(500, 8, 32, "bf16"), (500, 8, 32, "f32"), (40, 1, 602, "f32"), (33, 4, 13, "bf16"), (9, 1, 5000, "f32")])
def test_in_place_and_on_another_stream(n, p, w, dt):
    import torch
    rng = np.random.default_rng(w)
    d = _rounded(_make(rng, n, p, w, False, True), dt)
    dev = _Device(d, n, p, w, False, dt, 0.5, 1e-5)
    gh, gu = dev.forward()
    dh, du = (rng.standard_normal((n, p * w)).astype(np.float32).astype(np.float64) for _ in range(2))
    hs = gh.double().cpu().numpy()
    got = dev.backward(hs, dh, du)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ih, iu = dev.forward(in_place=True, stream=side.cuda_stream)
        there = dev.backward(hs, dh, du, in_place=True, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(ih, gh) and torch.equal(iu, gu)
    assert all(torch.equal(there[k], got[k]) for k in got)


@pytest.mark.gpu
def test_no_rows():
    rng = np.random.default_rng(0)
    d = _rounded(_make(rng, 0, 4, 8, True, True), "f32")
    dev = _Device(d, 0, 4, 8, True, "f32", 1.0, 1e-5)
    dev.forward()
    got = dev.backward(np.zeros((0, 32)), np.zeros((0, 32)), np.zeros((0, 32)))
    for k in ("dw_post", "db_post", "dw_pre", "db_pre"):
        assert bool((got[k] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("p,w", [(4, 32), (2, 50), (1, 700)])
def test_non_finite_values_stay_in_their_slice(layer, p, w):
    """A slice row that holds NaN or infinity spoils itself alone; the columns' gradients of that slice show it, no others."""
    import torch
    rng = np.random.default_rng(3)
    n = 40
    d = _rounded(_make(rng, n, p, w, layer, True, odd_rows=False), "f32")
    clean = _Device(d, n, p, w, layer, "f32", 1.0, 1e-5)
    ch, cu = clean.forward()
    dh, du = (rng.standard_normal((n, p * w)) for _ in range(2))
    cg = clean.backward(ch.double().cpu().numpy(), dh, du)
    bad = {k: (None if v is None else v.copy()) if k != "vec" else v for k, v in d.items()}
    bad["y"][5, 3], bad["y"][9, 1] = np.nan, np.inf
    dev = _Device(bad, n, p, w, layer, "f32", 1.0, 1e-5)
    gh, gu = dev.forward()
    keep = torch.ones((n, p * w), dtype=torch.bool, device="cuda")
    keep[5, :w] = False
    keep[9, :w] = False
    assert bool(torch.isnan(gh[5, :w]).all()) and bool(torch.isnan(gu[5, :w]).all())
    assert torch.equal(gh[keep], ch[keep]) and torch.equal(gu[keep], cu[keep])
    g = dev.backward(ch.double().cpu().numpy(), dh, du)
    assert torch.equal(g["dx"], cg["dx"])                  # h is clean
    assert torch.equal(g["dy"][keep], cg["dy"][keep]) and bool(torch.isnan(g["dy"][5, :w]).all())
    assert torch.equal(g["dw_post"][w:], cg["dw_post"][w:]) and torch.equal(g["dw_pre"], cg["dw_pre"])


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [False, True])
def test_gradient_matches_differences(layer):
    """Central differences of <dh, h> + <du, u> along a direction in every input, from the kernel's own forward pass.  The
    allowance is the truncation error of the same difference in 64 bits, and the rounding of the two sums over the step."""
    rng = np.random.default_rng(11)
    n, p, w, s, eps, t = 60, 2, 24, 0.8, 1e-3, 2.0 ** -5
    d = _rounded(_make(rng, n, p, w, layer, True, odd_rows=False), "f32")
    dh, du = (rng.standard_normal((n, p * w)).astype(np.float32).astype(np.float64) for _ in range(2))

    def value(dd, device):
        h, u, mh, mu = _forward64(dd, p, w, layer, s, eps)
        noise = _bound(w) * ((np.abs(dh) * mh).sum() + (np.abs(du) * mu).sum())
        if device:
            gh, gu = _Device(dd, n, p, w, layer, "f32", s, eps).forward()
            h, u = gh.double().cpu().numpy(), gu.double().cpu().numpy()
        return (dh * h).sum() + (du * u).sum(), noise
    h = _forward64(d, p, w, layer, s, eps)[0].astype(np.float32).astype(np.float64)
    got = {k: v.double().cpu().numpy() for k, v in _Device(d, n, p, w, layer, "f32", s, eps).backward(h, dh, du).items()}
    want = _backward64(d, _forward64(d, p, w, layer, s, eps)[0], dh, du, p, w, layer, s, eps)[0]
    names = [("x", "dx"), ("y", "dy"), ("gate", "dgate"), ("w_post", "dw_post"), ("w_pre", "dw_pre")]
    names += [("b_post", "db_post"), ("b_pre", "db_pre")] if layer else []
    for name, grad in names:
        where = d if name in d else d["vec"]
        kept = where[name]
        step = (rng.integers(0, 2, kept.shape) * 2 - 1) * t
        vals = {}
        for sign in (1, -1):
            where[name] = (kept + sign * step).astype(np.float32).astype(np.float64)
            vals[sign] = value(d, True), value(d, False), where[name]
        where[name] = kept
        moved = vals[1][2] - vals[-1][2]
        slope = (got[grad].reshape(kept.shape) * moved).sum()
        truth = (want[grad].reshape(kept.shape) * moved).sum()
        truncation = abs(vals[1][1][0] - vals[-1][1][0] - truth)
        noise = vals[1][0][1] + vals[-1][0][1] + abs(moved).max() * (np.abs(got[grad]).sum() * (_bound(w) + n * U32)) * 10
        assert abs(vals[1][0][0] - vals[-1][0][0] - slope) <= 1.01 * truncation + noise, name


@pytest.mark.gpu
def test_offsets_past_32_bits():
    import torch
    from paper_2408_11500_b200 import binding as B
    n, p, w = 2_449_029, 4, 256
    assert n * p * w > 2 ** 31
    x, u = torch.zeros((n, p * w), device="cuda", dtype=torch.bfloat16), torch.full((n, p * w), 7.0, device="cuda", dtype=torch.bfloat16)
    x[-3:] = torch.randn((3, p * w), device="cuda").to(torch.bfloat16)
    B.slicegcn_residual_norm_forward(B.make_residual_norm_desc(n, p, w, dtype=B.BF16), x, None, None, None, u)
    t = x[-3:].double().view(3, p, w)
    want = (t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + 1e-5)).view(3, -1)
    assert bool(((u[-3:].double() - want).abs() <= (_bound(w) + 2 * UBF) * want.abs()).all()) and int(torch.count_nonzero(u[:-3])) == 0


def test_refusals():
    from paper_2408_11500_b200 import binding as B
    b = np.zeros(1 << 16, np.float32)                      # host memory: every call below is refused before a launch
    ok = dict(n=4, num_slices=2, h_s=8)

    def refused(status, call):
        with pytest.raises(B.SliceGCNError) as e:
            call()
        assert e.value.status == status and str(e.value)

    def fwd(d, x=b, y=b, gate=b, h=b, u=b):
        return lambda: B.slicegcn_residual_norm_forward(d, x, y, gate, h, u)

    def bwd(d, y=b, gate=b, h=b, dh=b, du=b, dx=b, dy=b, dgate=b, v=(b, b, b, b), ws=b, wsb=b.nbytes):
        return lambda: B.slicegcn_residual_norm_backward(d, y, gate, h, dh, du, dx, dy, dgate, *v, ws, wsb)
    for bad in (dict(n=-1), dict(num_slices=0), dict(h_s=0), dict(kind=2), dict(dtype=9), dict(eps=0.0), dict(eps=float("nan"))):
        d = B.make_residual_norm_desc(**{**ok, **bad})
        for call in (fwd(d), bwd(d), lambda: B.slicegcn_residual_norm_workspace_bytes(d)):
            refused(B.ERR_INVALID_ARG, call)
    for bad in (dict(num_slices=65), dict(h_s=B.MAX_NORM_WIDTH + 1)):
        d = B.make_residual_norm_desc(**{**ok, **bad})
        for call in (fwd(d), bwd(d)):
            refused(B.ERR_UNSUPPORTED, call)
    refused(B.ERR_OVERFLOW, fwd(B.make_residual_norm_desc(4, 64, 1 << 26)))
    for k in ("x", "y", "gate", "h", "u"):
        refused(B.ERR_INVALID_ARG, fwd(B.make_residual_norm_desc(**ok, **{k + "_ld": 15})))
    for k in ("y", "gate", "h", "dh", "du", "dx", "dy", "dgate"):
        refused(B.ERR_INVALID_ARG, bwd(B.make_residual_norm_desc(**ok, **{k + "_ld": 15})))
    d = B.make_residual_norm_desc(**ok)
    none = (None,) * 4
    for call in (fwd(d, x=None, y=None, gate=None), fwd(d, y=None), fwd(d, h=None, u=None), fwd(d, x=b.ctypes.data + 2),
                 bwd(d, dh=None, du=None, v=none), bwd(d, h=None), bwd(d, y=None, gate=None, dgate=None), bwd(d, y=None, dy=None),
                 bwd(d, gate=None), bwd(d, du=None), bwd(d, y=None, gate=None, dy=None, dgate=None), bwd(d, dx=b.ctypes.data + 2),
                 bwd(d, v=(b.ctypes.data + 1, b, b, b)), bwd(d, ws=b.ctypes.data + 4)):
        refused(B.ERR_INVALID_ARG, call)
    refused(B.ERR_INVALID_ARG, fwd(B.make_residual_norm_desc(**ok, w_pre=b.ctypes.data + 2)))
    need = B.slicegcn_residual_norm_workspace_bytes(d)
    assert need > 0
    refused(B.ERR_ALLOC, bwd(d, wsb=need - 1))
    refused(B.ERR_ALLOC, bwd(d, ws=None, wsb=need))
    with pytest.raises(TypeError):
        B.make_residual_norm_desc(**ok, z_ld=16)
