"""The accuracy of the residual step's gate, which the sums over a slice (and their tolerances) hide elsewhere.

With y = 1 in every column, no residual and a plain norm, h = sigmoid(g) b with the same b in every column: an open gate (infinity)
shows b.  In units of u = 2^-24: 2^x is off by at most 4, the constant ln 2 puts 0.05 |g| into e^-g, each of the product and the sum
1 + e rounds once, 1 / x is off by 2 and the product with b by 1: 9 + 0.05 |g| for h.  The slope e / (1 + e)^2 takes two
reciprocals and two products more (15 + 0.05 |g|), dgate three products and the norm's root besides (30 + 0.05 |g|).
"""
import math

import pytest

U32 = 2.0 ** -24


def _call(gate, w):
    import torch
    from paper_2408_11500_b200 import binding as B
    n = gate.shape[0]
    y, h, dh, dx, dy, dgate = (torch.ones((n, w), device="cuda") for _ in range(6))
    d = B.make_residual_norm_desc(n, 1, w)
    wsb = B.slicegcn_residual_norm_workspace_bytes(d)
    ws = torch.empty(max(wsb, 1), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    B.slicegcn_residual_norm_forward(d, None, y, gate, h, None, st)
    B.slicegcn_residual_norm_backward(d, y, gate, None, dh, None, dx, dy, dgate, None, None, None, None, ws, wsb, st)
    return h.double(), dgate.double()


@pytest.mark.gpu
@pytest.mark.parametrize("w", [32, 101, 300, 1000, 4000])
def test_gate_and_its_slope(w):
    import torch
    n = 50
    gate = torch.linspace(-80, 80, n * w, device="cuda").view(n, w)
    h, dgate = _call(gate, w)
    b = _call(torch.full((n, w), math.inf, device="cuda"), w)[0]
    g = gate.double()
    want, slope = torch.sigmoid(g), torch.sigmoid(g) * torch.sigmoid(-g)
    assert bool(((h / b / want - 1).abs() <= (10 + 0.05 * g.abs()) * U32).all())
    assert bool(((dgate / (slope / math.sqrt(1 + 1e-5)) - 1).abs() <= (30 + 0.05 * g.abs()) * U32).all())


@pytest.mark.gpu
@pytest.mark.parametrize("w", [32, 101, 300, 1000, 4000])
def test_gates_past_every_exponent(w):
    import torch
    values = [math.inf, -math.inf, 3e38, -3e38, 200.0, -200.0, 128.5, -88.5, 0.0, -0.0, math.nan]
    gate = torch.tensor(values, device="cuda")[:, None].expand(-1, w).contiguous()
    h, dgate = _call(gate, w)
    b = h[0]
    for k, v in enumerate(values[:8]):
        assert bool((h[k] == (b if v > 0 else 0.0)).all()), v
        assert bool((dgate[k].abs() <= 1e-38).all()), v
    assert bool((h[8] == b / 2).all()) and bool((h[9] == b / 2).all())
    assert bool(torch.isnan(h[10]).all()) and bool(torch.isnan(dgate[10]).all())
