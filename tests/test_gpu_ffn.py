"""Feed-forward projections and their gradients, against the definition in 64 bits.

Tolerances.  With K terms of a sum the error is bounded against the sum of magnitudes, not the result: by S below, the
definition with |x|, |W|, |b| and the activation's largest slope.  fp32: operands are exact sums of three parts, products of
parts beyond the 24th bit are left out (2^-24 each, three of them at most 2^-22 in all), and the tensor cores' additions cut off up to
2^-23 of the running sum each: 20 of them at its full size per chunk of 128 (six products: the five small ones lie 2^-7 down), and half as
much for each of the K / 128 additions in registers, so (16 + 8 + K / 256) 2^-23 S covers them; activations add 8 * 2^-24.  bf16: products are exact, additions as above without chunks
(K / 16) 2^-23 S, and results are rounded once, half a step or 2^-8 of the value at most.
Gradients in bf16 round da and dc first: another 2^-8 of the sum of magnitudes.
"""
import math

import numpy as np
import pytest

U32, UBF = 2.0 ** -24, 2.0 ** -8
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


def act64(name, a):
    import torch
    if name == "none":
        return a, torch.ones_like(a)
    if name == "relu":
        return a.clamp(min=0), (a > 0).double()
    if name == "silu":
        q = torch.sigmoid(a)
        return a * q, q * (1 + a * (1 - q))
    u = math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)
    t = torch.tanh(u)
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * a * a)


class Problem:
    """Inputs of a call; leading dimensions `pad` wider than the rows, whose extra columns hold NaN and must not matter."""

    def __init__(self, n, p, ins, outs, gated, act, dtype, grad="same", pad=0, bias=True, residual=False, scale=0.75, seed=0, offset=0):
        import torch
        from paper_2408_11500_b200 import binding as B
        self.__dict__.update(n=n, p=p, ins=ins, outs=outs, gated=gated, act=act, scale=scale)
        self.dt = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.gt = self.dt if grad == "same" else torch.float32 if grad == "fp32" else torch.bfloat16
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def mat(cols, t, std=1.0):
            ld = cols + pad
            buf = torch.full((n * ld + 64,), float("nan"), device="cuda", dtype=t)
            m = buf[offset:offset + n * ld].view(n, ld)[:, :cols] if n else torch.empty((0, ld), device="cuda", dtype=t)[:, :cols]
            m.copy_(torch.randn((n, cols), generator=g, device="cuda") * std)
            return m
        self.x, self.dout = mat(p * ins, self.dt), mat(p * outs, self.gt)
        self.r = mat(p * outs, self.dt) if residual else None
        self.W = (torch.randn((p, ins, outs), generator=g, device="cuda") / math.sqrt(ins)).to(self.dt)
        self.W2 = (torch.randn((p, ins, outs), generator=g, device="cuda") / math.sqrt(ins)).to(self.dt) if gated else None
        self.b = torch.randn((p, outs), generator=g, device="cuda") * 0.3 if bias else None
        self.b2 = torch.randn((p, outs), generator=g, device="cuda") * 0.3 if bias and gated else None
        self.out, self.dx = mat(p * outs, self.dt), mat(p * ins, self.gt)
        code = lambda t: B.F32 if t == torch.float32 else B.BF16   # noqa: E731
        lds = {k + "_ld": getattr(self, k).stride(0) for k in ("x", "r", "out", "dout", "dx") if getattr(self, k) is not None}
        self.d = B.make_ffn_desc(n, p, ins, outs, self.W, self.W2, self.b, self.b2, act=ACTS[act], dtype=code(self.dt), grad_dtype=code(self.gt),
                                 scale=scale, **lds)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def _ws(self, back):
        import torch
        from paper_2408_11500_b200 import binding as B
        need = B.slicegcn_ffn_workspace_bytes(self.d, self.x, self.dout if back else None)
        return torch.randint(0, 256, (max(need, 1),), dtype=torch.uint8, device="cuda"), need

    def forward(self, stream=None):
        from paper_2408_11500_b200 import binding as B
        ws, need = self._ws(False)
        B.slicegcn_ffn_forward(self.d, self.x, self.r, self.out, self.status, ws, need, stream)
        assert int(self.status) == 0
        return self.out

    def backward(self, want=("dx", "dW", "dW2", "db", "db2"), stream=None):
        import torch
        from paper_2408_11500_b200 import binding as B
        ws, need = self._ws(True)
        shape = (self.p, self.ins, self.outs)
        g = {"dx": self.dx, "dW": torch.full(shape, float("nan"), device="cuda", dtype=self.gt), "db": torch.full((self.p, self.outs), float("nan"), device="cuda")}
        g["dW2"], g["db2"] = (torch.full_like(g["dW"], float("nan")), torch.full_like(g["db"], float("nan"))) if self.gated else (None, None)
        g = {k: v if k in want else None for k, v in g.items()}
        B.slicegcn_ffn_backward(self.d, self.x, self.dout, g["dx"], g["dW"], g["dW2"], g["db"], g["db2"], self.status, ws, need, stream)
        assert int(self.status) == 0
        return {k: v for k, v in g.items() if v is not None}

    # ---- 64 bits
    def _pre(self):
        import torch
        x = self.x.double().reshape(self.n, self.p, self.ins).transpose(0, 1)

        def one(W, b):
            a, s = torch.matmul(x, W.double()), torch.matmul(x.abs(), W.double().abs())
            return (a, s) if b is None else (a + b.double()[:, None], s + b.double().abs()[:, None])
        a, sa = one(self.W, self.b)
        c, sc = one(self.W2, self.b2) if self.gated else (torch.ones_like(a), torch.ones_like(a))
        return x, a, sa, c, sc

    def adds(self, k):
        """Relative error of a sum of k terms against the sum of magnitudes."""
        import torch
        return (24 + k / 256) * 2 * U32 if self.dt == torch.float32 or self.gt == torch.float32 else (2 + k / 16) * 2 * U32

    def check_forward(self, out):
        import torch
        _, a, sa, c, sc = self._pre()
        y, dy = act64(self.act, a)
        e = self.adds(self.ins)
        want = y * c if self.gated else y
        # |act'| <= 1.13; the product's two errors
        err = 1.13 * e * sa * (c.abs() if self.gated else 1) + (y.abs() * e * sc if self.gated else 0) + 16 * U32 * want.abs()
        err = err + 16 * U32 * sa * (c.abs() if self.gated else 1)
        want, err = ((t * abs(self.scale) if t is err else t * self.scale).transpose(0, 1).reshape(self.n, -1) for t in (want, err))
        if self.r is not None:
            want = want + self.r.double()
            err = err + 2 * U32 * self.r.double().abs()
        u = 0.0 if self.dt == torch.float32 else UBF
        off = (out.double() - want).abs()
        assert bool(torch.isfinite(out).all())
        bound = err + (u + 2 * U32) * want.abs() + 1e-30
        assert bool((off <= bound).all()), float((off / bound).max())

    def check_backward(self, got):
        import torch
        x, a, sa, c, sc = self._pre()
        y, dy = act64(self.act, a)
        g = self.dout.double().reshape(self.n, self.p, self.outs).transpose(0, 1) * self.scale
        e = self.adds(self.ins)
        da, dc = g * dy * c if self.gated else g * dy, g * y
        # act'' <= 1 for silu and gelu; ReLU's step is handled by the callers (inputs without a pre-activation near zero)
        bend = 0.0 if self.act in ("none", "relu") else 1.2
        eda = g.abs() * (bend * e * sa * c.abs() + (1.13 * e * sc if self.gated else 0)) + 32 * U32 * g.abs() * c.abs() * (1 + sa * bend)
        edc = g.abs() * 1.13 * e * sa + 16 * U32 * (dc.abs() + g.abs() * sa)
        round_z = UBF if self.gt == torch.bfloat16 and (self.act != "none" or self.gated) else 0.0
        u = UBF if self.gt == torch.bfloat16 else 0.0
        xt = x.transpose(1, 2)

        def close(name, want, err):
            off = (got[name].double() - want).abs()
            bound = err + (u if got[name].dtype == torch.bfloat16 else 2 * U32) * want.abs() + 1e-30
            assert bool(torch.isfinite(got[name]).all()), name
            assert bool((off <= bound).all()), (name, float((off / bound).max()))
        parts = [("dW", "db", da, eda, self.W)] + ([("dW2", "db2", dc, edc, self.W2)] if self.gated else [])
        dx = edx = 0.0
        for dw, db, z, ez, W in parts:
            mag = z.abs()
            ez2 = ez + round_z * mag
            rows = (24 + min(self.n, 4096) / 16 + self.n / 256) * 2 * U32
            if dw in got:
                close(dw, torch.matmul(xt, z), torch.matmul(xt.abs(), ez2 + rows * mag))
            if db in got:
                close(db, z.sum(1), (ez + (8 + math.sqrt(self.n)) * 2 * U32 * mag).sum(1))
            Wt = W.double().transpose(1, 2)
            dx = dx + torch.matmul(z, Wt)
            edx = edx + torch.matmul(ez2 + self.adds(2 * self.outs) * mag, Wt.abs())
        if "dx" in got:
            close("dx", dx.transpose(0, 1).reshape(self.n, -1), edx.transpose(0, 1).reshape(self.n, -1))


SHAPES = [(1, 1, 4, 4), (5, 1, 64, 64), (300, 1, 256, 256), (257, 4, 32, 64), (1000, 1, 602, 130), (129, 8, 16, 8), (700, 2, 100, 47), (64, 1, 1433, 16),
          (2048, 1, 128, 1024), (33, 3, 7, 11), (511, 1, 1024, 200), (9, 1, 513, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
def test_forward(shape, gated, dtype):
    for act, pad, residual in (("silu", 0, False), ("gelu", 8, True), ("none", 3, True), ("relu", 0, True)):
        q = Problem(*shape, gated, act, dtype, pad=pad, residual=residual, seed=len(act))
        q.check_forward(q.forward())


@pytest.mark.gpu
@pytest.mark.parametrize("types", ["bf16", "fp32", "bf16/fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
def test_backward(shape, gated, types):
    dtype, grad = types.split("/") if "/" in types else (types, "same")
    for act, pad in (("silu", 0), ("gelu", 8), ("none", 3)):
        q = Problem(*shape, gated, act, dtype, grad, pad=pad, seed=len(act))
        q.check_backward(q.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("types", ["bf16", "fp32", "bf16/fp32"])
@pytest.mark.parametrize("shape", [(30_000, 8, 48, 40), (50_001, 1, 300, 72), (40_000, 2, 72, 300), (20_000, 1, 700, 700)], ids=str)
def test_many_tiles_per_pair_of_sms(shape, types):
    """Several tiles one after another on every pair of SMs, of half and of whole width, with one and with many chunks of k."""
    dtype, grad = types.split("/") if "/" in types else (types, "same")
    for gated in (False, True):
        q = Problem(*shape, gated, "silu", dtype, grad)
        q.check_forward(q.forward())
        q.check_backward(q.backward())
        q = Problem(*shape, gated, "none", dtype, grad)
        q.check_backward(q.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 2, 4, 5, 8, 9])
def test_a_few_rows(n, dtype):
    """Serving: up to eight rows go another way than more do."""
    for p, ins, outs, pad in ((1, 256, 1024, 0), (1, 4096, 260, 3), (4, 33, 129, 1), (1, 1433, 6, 0), (2, 3, 1, 5), (8, 700, 128, 8), (1, 16384, 40, 0), (1, 20000, 12, 0)):
        for gated, act, residual in ((False, "gelu", True), (True, "silu", False), (False, "none", False)):
            q = Problem(n, p, ins, outs, gated, act, dtype, pad=pad, residual=residual, bias=act != "none", seed=n)
            q.check_forward(q.forward())


@pytest.mark.gpu
@pytest.mark.parametrize("types", ["bf16", "fp32", "bf16/fp32"])
@pytest.mark.parametrize("shape", [(100, 1, 4096, 64), (2708, 1, 1433, 16), (16, 1, 64, 2500), (700, 1, 2000, 130), (40, 2, 900, 300), (5, 1, 513, 2100), (5000, 1, 800, 72)], ids=str)
def test_products_in_pieces(shape, types):
    """Few tiles with a long sum: pieces of it are added up by a second kernel."""
    dtype, grad = types.split("/") if "/" in types else (types, "same")
    for gated, act, pad, residual in ((False, "silu", 1, True), (True, "gelu", 0, True), (False, "none", 0, False)):
        q = Problem(*shape, gated, act, dtype, grad, pad=pad, residual=residual)
        q.check_forward(q.forward())
        q.check_backward(q.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("types", ["bf16", "fp32", "bf16/fp32"])
@pytest.mark.parametrize("shape", [(3000, 8, 14, 23), (777, 8, 4, 193), (5000, 6, 20, 64), (1000, 64, 1, 3), (2000, 4, 32, 32), (300, 12, 5, 1), (20_001, 8, 32, 64)], ids=str)
def test_narrow_slices(shape, types):
    """Slices of few columns are computed several at a time."""
    dtype, grad = types.split("/") if "/" in types else (types, "same")
    for gated, act, pad, residual in ((False, "silu", 1, True), (True, "gelu", 0, False), (False, "none", 5, True)):
        q = Problem(*shape, gated, act, dtype, grad, pad=pad, residual=residual)
        q.check_forward(q.forward())
        q.check_backward(q.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1000, 1, 25, 14), (513, 2, 300, 9), (3000, 1, 16, 16), (129, 8, 13, 10), (70, 4, 7, 375), (65, 1, 100, 100), (10, 1, 4, 64), (20_000, 1, 1213, 5), (999, 1, 64, 61)], ids=str)
def test_little_work(shape, dtype):
    """Sizes and layouts that plain multiply-adds take, aligned (pad 4) and not."""
    for gated, act, pad, residual in ((False, "silu", 1, True), (True, "gelu", 4, False), (False, "none", 0, False), (True, "relu", 3, True)):
        q = Problem(*shape, gated, act, dtype, pad=pad, residual=residual, offset=pad)
        q.check_forward(q.forward())


@pytest.mark.gpu
@pytest.mark.parametrize("pad,offset", [(0, 0), (4, 4), (2, 2), (1, 0), (8, 8), (4, 2)], ids=str)
@pytest.mark.parametrize("shape,types", [((700, 1, 300, 132), ("fp32", "fp32")), ((333, 2, 260, 96), ("fp32", "fp32")), ((260, 3, 150, 70), ("fp32", "fp32")),
                                         ((700, 1, 900, 136), ("bf16", "bf16")), ((300, 1, 1000, 131), ("bf16", "fp32"))], ids=str)
def test_layouts_of_sums_emptied_into_registers(shape, types, pad, offset):
    """r, dout and results by 16, 8 and single elements at a time."""
    for gated, act, residual in ((False, "gelu", True), (True, "silu", False), (True, "relu", True)):
        q = Problem(*shape, gated, act, types[0], grad=types[1], pad=pad, residual=residual, offset=offset)
        q.check_forward(q.forward())
        q.check_backward(q.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("ins", [1024, 4096])
def test_biases_gradients_of_long_sums(ins):
    """Additions cut in one direction, so that a sum over rows keeps a relative error that stays what an element's is.  512 k are 32
    additions that cut half of 2^-23 of a running sum that grows to the whole: 32 * 2^-24 / 2 = 2^-20 on average; twice that is allowed."""
    import torch
    q = Problem(300, 1, ins, 64, True, "silu", "bf16")
    got = q.backward(("db", "db2"))
    x, a, _, c, _ = q._pre()
    y, dy = act64("silu", a)
    g = q.dout.double()[None] * q.scale
    for name, want in (("db", (g * dy * c).sum(1)), ("db2", (g * y).sum(1))):
        assert float((got[name].double() - want).norm() / want.norm()) < 2.0 ** -19


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 31, 33, 512, 513])
@pytest.mark.parametrize("types", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")], ids=str)
def test_biases_gradients_of_few_rows(n, types):
    for p, gated in ((1, True), (3, False)):
        q = Problem(n, p, 72, 200, gated, "gelu", types[0], grad=types[1])
        q.check_backward(q.backward())
        for want in (("db",), ("dW", "db"), ("dx",)):
            q.check_backward(q.backward(want))
