"""Feed-forward projections at the edges of their number ranges: tiny and large fp32 numbers in the form that the tensor cores
take, activations and derivatives far from zero, NaN before an activation, biases' gradients of middling sums."""
import math

import pytest

from test_gpu_ffn import U32, UBF, Problem, act64

pytestmark = pytest.mark.gpu

LOST = 2.0 ** -133     # what the three bf16 parts of an fp32 number leave out at most: the last bit of the least of them


def _adds(k):
    """Relative error of a sum of k fp32 products against the sum of magnitudes, as `test_gpu_ffn.py` derives it."""
    return (24 + k / 256) * 2 * U32


def _ranged(n, cols, lo, hi, seed):
    """Rows of normal numbers times powers of two from 2^lo to 2^hi."""
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    scale = torch.linspace(lo, hi, n, device="cuda", dtype=torch.float64).round().exp2()
    return (torch.randn((n, cols), generator=g, device="cuda", dtype=torch.float64) * scale[:, None]).float()


def test_fp32_numbers_of_every_magnitude_in_three_parts():
    """Rows from 2^-120 (and single numbers below the normal ones) to 2^90; the weights are large enough for the products to be normal.
    A number keeps its 24 bits from 2^-110 up; below that what it loses is less than 2^-133."""
    import torch
    from paper_2408_11500_b200 import binding as B
    n, ins, outs = 3000, 512, 256
    g = torch.Generator("cuda").manual_seed(1)
    x, dout = _ranged(n, ins, -120, 90, 2), _ranged(n, outs, -120, 90, 3)
    W = torch.randn((1, ins, outs), generator=g, device="cuda") * 2.0 ** 16
    out, dx = torch.empty((n, outs), device="cuda"), torch.empty((n, ins), device="cuda")
    d = B.make_ffn_desc(n, 1, ins, outs, W)
    need = B.slicegcn_ffn_workspace_bytes(d, x)
    assert need >= 6 * n * ins                       # parts of x are laid out: this is no plain product
    ws = torch.empty(max(need, B.slicegcn_ffn_workspace_bytes(d, x, dout)), dtype=torch.uint8, device="cuda")
    B.slicegcn_ffn_forward(d, x, None, out, None, ws, ws.numel())
    B.slicegcn_ffn_backward(d, x, dout, dx, None, None, None, None, None, ws, ws.numel())
    w = W[0].double()
    for got, a, b in ((out, x.double(), w), (dx, dout.double(), w.t())):
        want, mag, lost = a @ b, a.abs() @ b.abs(), LOST * b.abs().sum(0)
        bound = (_adds(a.shape[1]) + 2 * U32) * mag + lost
        off = (got.double() - want).abs()
        assert bool((off <= bound).all()), float((off / bound).max())


def test_tiny_gradients_in_three_parts():
    """da and dc of rows from 2^-120 to 2^60 on their way through memory, gated without an activation: da = g c, dc = g a."""
    import torch
    from paper_2408_11500_b200 import binding as B
    n, ins, outs = 2000, 256, 320
    g = torch.Generator("cuda").manual_seed(4)
    x, dout = torch.randn((n, ins), generator=g, device="cuda"), _ranged(n, outs, -120, 60, 5)
    W, W2 = (torch.randn((1, ins, outs), generator=g, device="cuda") * 16 for _ in range(2))
    dx = torch.empty((n, ins), device="cuda")
    d = B.make_ffn_desc(n, 1, ins, outs, W, W2)
    ws = torch.empty(B.slicegcn_ffn_workspace_bytes(d, x, dout), dtype=torch.uint8, device="cuda")
    B.slicegcn_ffn_backward(d, x, dout, dx, None, None, None, None, None, ws, ws.numel())
    X, G, w, w2 = x.double(), dout.double(), W[0].double(), W2[0].double()
    want, bound = 0.0, 0.0
    for here, other in ((w, w2), (w2, w)):
        z, s = G * (X @ other), G.abs() * (X.abs() @ other.abs())
        want = want + z @ here.t()
        bound = bound + ((_adds(ins) + 4 * U32) * s + LOST) @ here.abs().t() + (_adds(2 * outs) + 2 * U32) * (z.abs() @ here.abs().t())
    off = (dx.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


#: rows, columns: tiles; pieces of k and the kernel that ends them
GRAD_PATHS = [(600, 64), (16, 2048), (300, 1024)]
TYPES = [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")]


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("n,ins", GRAD_PATHS, ids=str)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_nan_before_an_activation_leaves_no_finite_gradient(act, gated, n, ins, types):
    """Of its row in dx, and of the biases' and weights' sums that it enters; other rows keep theirs."""
    import torch
    q = Problem(n, 1, ins, 72, gated, act, types[0], grad=types[1])
    clean = q.backward()["dx"].clone()
    q.x[4, 7] = float("nan")
    got = q.backward()
    keep = torch.arange(n, device="cuda") != 4
    assert torch.equal(got["dx"][keep], clean[keep])
    assert bool(torch.isnan(got["dx"][4]).all()) and bool(torch.isnan(got["db"]).all()) and bool(torch.isnan(got["dW"]).all())


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("n,ins", GRAD_PATHS, ids=str)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_derivatives_far_from_zero(act, gated, n, ins, types):
    """W is the unit matrix in its first rows, so that x's first columns are the pre-activations: the derivative is 1 far above zero and
    0 far below.  Everything is a power of two or a sum of two, so that results are exact."""
    import torch
    outs = 64
    q = Problem(n, 1, ins, outs, gated, act, types[0], grad=types[1], scale=1.0, bias=False)
    q.x.zero_(), q.W.zero_(), q.dout.fill_(0.5)
    q.W[0, :outs] = torch.eye(outs, device="cuda", dtype=q.dt)
    e = torch.arange(20, 20 + outs, device="cuda")                       # 2^20 .. 2^83; squares pass fp32's range from 2^64 on
    sign = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1.0, -1.0)[:, None]
    q.x[:, :outs] = (sign * torch.exp2(e.double())).to(q.dt)
    if gated:                                                            # c = 4 x_0 2^-20 = +-4
        q.W2.zero_()
        q.W2[0, 0] = 2.0 ** -18
    got = q.backward(("dx",))["dx"].double()
    c = 4.0 * sign.double() if gated else torch.ones_like(sign, dtype=torch.float64)
    want = torch.zeros_like(got)
    want[:, :outs] = 0.5 * c * (sign > 0)
    if gated:                                                            # dc = g act(a), all of it to x_0
        total = (0.5 * torch.exp2(e.double())).sum() * 2.0 ** -18
        want[:, :1] += total * (sign > 0)
        # the sum of 64 powers of two is rounded: additions as in every product, and dc's own roundings
        slack = (_adds(outs) if q.dt == torch.float32 or q.gt == torch.float32 else (2 + outs / 16) * 2 * U32) + (2 * UBF if q.gt == torch.bfloat16 else 8 * U32)
        off = (got[:, 0] - want[:, 0]).abs()
        assert bool((off <= slack * want[:, 0].abs()).all())
        got, want = got[:, 1:], want[:, 1:]
    assert torch.equal(got, want), (got - want).abs().max()


#: rows, columns: a few rows; plain multiply-adds; tiles; pieces of k and the kernel that ends them
PATHS = [(5, 64), (200, 25), (40_000, 400), (100, 4096)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,ins", PATHS, ids=str)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activations_far_below_zero(act, n, ins, dtype):
    """Where 1 + exp(-w) passes fp32's range the activation is still a normal number.  x is zero, so that the biases are the
    pre-activations.  The exponential and the quotient are off by 2 units each; w by 4 of its own roundings.  Results of bf16 may take a
    gate below 2^-126 for zero."""
    import torch
    outs = 256
    q = Problem(n, 1, ins, outs, False, act, dtype, scale=1.0)
    q.x.zero_()
    q.b.copy_(torch.linspace(-100.0, -60.0, outs, device="cuda") if act == "silu" else torch.linspace(-11.0, -7.0, outs, device="cuda"))
    a = q.b[0].double()
    w = -a if act == "silu" else -2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)
    want = a * torch.exp(-w) / (1 + torch.exp(-w))
    got = q.forward().double()
    bound = (16 + 4 * w.abs()) * U32 * want.abs() + 2 * a.abs() * 2.0 ** -149
    if dtype == "bf16":
        bound = bound + UBF * want.abs() + a.abs() * 2.0 ** -126
    off = (got - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("ins", [256, 320, 512, 768, 1024])
def test_biases_gradients_of_middling_sums(ins):
    """Biases' gradients are fp32 beside gradients of bf16 too.  An addition of 16 columns in tensor memory cuts half of 2^-23 of a running
    sum that grows to the whole: ins / 16 * 2^-24 / 2 on average, up to 768 columns; longer sums are emptied every 512.  Twice that is
    allowed."""
    q = Problem(300, 1, ins, 64, True, "silu", "bf16")
    got = q.backward(("db", "db2"))
    x, a, _, c, _ = q._pre()
    y, dy = act64("silu", a)
    g = q.dout.double()[None] * q.scale
    columns = ins if ins <= 768 else 512
    for name, want in (("db", (g * dy * c).sum(1)), ("db2", (g * y).sum(1))):
        assert float((got[name].double() - want).norm() / want.norm()) < columns / 16 * 2.0 ** -24, name


def test_weights_gradients_of_many_rows_are_not_cut_short():
    """Additions in tensor memory cut in one direction: 512 rows are 32 of them, half of 2^-24 each of a sum that grows to the whole, 2^-20 on
    average; what 512 rows give is then added with rounding.  The mean of a bf16 result's distance to the rightly rounded one is
    that shift (results on the other side of a rounding's border make up for those that did not move); twice 2^-20 is allowed."""
    import torch
    from paper_2408_11500_b200 import binding as B
    n, ins, outs = 300_000, 1024, 512
    g = torch.Generator("cuda").manual_seed(6)

    def positive(cols):
        t = torch.rand((n, cols), generator=g, device="cuda").add_(0.5).mul_(torch.rand(cols, generator=g, device="cuda").add_(1.0))
        return t.to(torch.bfloat16)
    x, dout = positive(ins), positive(outs)
    W, dW = (torch.zeros((1, ins, outs), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    d = B.make_ffn_desc(n, 1, ins, outs, W, dtype=B.BF16)
    ws = torch.empty(B.slicegcn_ffn_workspace_bytes(d, x, dout), dtype=torch.uint8, device="cuda")
    B.slicegcn_ffn_backward(d, x, dout, None, dW, None, None, None, None, ws, ws.numel())
    want = torch.zeros((ins, outs), device="cuda", dtype=torch.float64)
    for s in range(0, n, 50_000):
        want += x[s:s + 50_000].double().t() @ dout[s:s + 50_000].double()
    short = ((want.to(torch.bfloat16).double() - dW[0].double()) / want).mean()
    assert abs(float(short)) < 2 * 2.0 ** -20, float(short)
