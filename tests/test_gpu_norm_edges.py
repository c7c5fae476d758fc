"""What a call leaves out has no say in it, and an eps below fp32's range is not zero."""
import pytest

WIDTHS = [(50, 4, 32), (50, 2, 13), (50, 1, 300), (40, 1, 1000), (9, 1, 3000)]


def _desc(n, p, w, **more):
    from paper_2408_11500_b200 import binding as B
    return B.make_residual_norm_desc(n, p, w, **more)


def _backward(d, y, gate, h, dh, du):
    import torch
    from paper_2408_11500_b200 import binding as B
    dx = torch.full_like(h, float("nan"))
    dy = torch.full_like(h, float("nan")) if y is not None else None
    wsb = B.slicegcn_residual_norm_workspace_bytes(d)
    ws = torch.empty(max(wsb, 1), dtype=torch.uint8, device="cuda")
    B.slicegcn_residual_norm_backward(d, y, gate, h, dh, du, dx, dy, None, None, None, None, None, ws, wsb, torch.cuda.current_stream().cuda_stream)
    return dx, dy


@pytest.mark.gpu
@pytest.mark.parametrize("n,p,w", WIDTHS)
@pytest.mark.parametrize("kind", [0, 1], ids=["rms", "layer"])
def test_weights_of_a_norm_that_a_call_does_not_take(n, p, w, kind):
    """After the last block there is no u: whatever its weights hold, the gradient of h goes through as it is.  Before the first
    block there is no y: its weights stay out of u's gradient."""
    import torch
    torch.manual_seed(w)
    h, dh, y = (torch.randn((n, p * w), device="cuda") for _ in range(3))
    bad, good = torch.full((p * w,), float("nan"), device="cuda"), torch.rand(p * w, device="cuda") + 0.5
    want = _backward(_desc(n, p, w, kind=kind, w_post=good), y, None, h, dh, None)
    got = _backward(_desc(n, p, w, kind=kind, w_post=good, w_pre=bad, b_pre=bad), y, None, h, dh, None)
    assert torch.equal(got[0], dh) and torch.equal(got[1], want[1])
    want = _backward(_desc(n, p, w, kind=kind, w_pre=good), None, None, h, dh, y)[0]
    got = _backward(_desc(n, p, w, kind=kind, w_pre=good, w_post=bad, b_post=bad), None, None, h, dh, y)[0]
    assert bool(torch.isfinite(got).all()) and torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("n,p,w", WIDTHS)
@pytest.mark.parametrize("kind", [0, 1], ids=["rms", "layer"])
def test_rows_of_zeros_with_the_least_eps(n, p, w, kind):
    """0 / sqrt(0 + eps) is 0 however small eps is."""
    import torch
    from paper_2408_11500_b200 import binding as B
    x, y = torch.randn((n, p * w), device="cuda"), torch.randn((n, p * w), device="cuda")
    y[3], x[3] = 0.0, 0.0
    y[5], x[5] = 2.0, 0.0
    h, u = torch.empty_like(x), torch.empty_like(x)
    d = _desc(n, p, w, kind=kind, eps=1e-60)
    B.slicegcn_residual_norm_forward(d, x, y, None, h, u, torch.cuda.current_stream().cuda_stream)
    assert bool((h[3] == 0).all()) and bool((u[3] == 0).all())
    assert bool(torch.isfinite(h).all()) and bool(torch.isfinite(u).all())
    zero = torch.zeros_like(x)
    dx, dy = _backward(d, y, None, h, zero, zero)
    assert bool((dx == 0).all()) and bool((dy == 0).all())
