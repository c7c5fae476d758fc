"""The residual step where a thread works on many rows: stages of the copies are used again, the last round is a part of one, and
the columns' sums take many rows each.  Rows against the 64-bit definition with the tolerances of `test_gpu_residual_norm.py` (a
spread sample of them, since rows do not depend on one another); sums over the rows on values that make them exact in any order.
"""
import numpy as np
import pytest

from test_gpu_residual_norm import UBF, U32, _backward64, _bound, _close, _Device, _forward64, _make, _rounded

# rows at a time are 1,184 to 151,552 by lanes (forward: 8 CTAs per SM; gradient: 2), about 1,776 staged, 592 beyond 1,024 columns
SHAPES = [(45_003, 8, 32, 0, 0), (45_003, 1, 128, 0, 0), (90_001, 4, 13, 0, 0), (700_001, 1, 5, 0, 0), (45_001, 2, 100, 1, 3), (30_001, 4, 18, 0, 0),
          (45_001, 1, 256, 0, 0), (8_001, 1, 171, 0, 0), (5_501, 2, 200, 0, 0), (8_001, 1, 400, 4, 4), (9_001, 1, 602, 0, 6), (8_003, 1, 1000, 0, 0), (6_001, 1, 700, 1, 1),
          (2_003, 1, 1100, 0, 0), (1_501, 2, 1433, 0, 0)]


def _sample(n):
    some = np.unique(np.concatenate([np.arange(min(n, 200)), np.arange(max(0, n - 300), n), np.random.default_rng(n).integers(0, n, 1500)]))
    return some


def _rows(d, some):
    return {k: (None if v is None else v[some]) if k != "vec" else v for k, v in d.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("n,p,w,off,pad", SHAPES)
@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
@pytest.mark.parametrize("dt,gate", [("f32", True), ("bf16", True), ("bf16", False)])
def test_many_rows(n, p, w, off, pad, layer, dt, gate):
    rng = np.random.default_rng(w)
    s, eps = 0.6, 1e-5
    d = _rounded(_make(rng, n, p, w, layer, gate), dt)
    dev = _Device(d, n, p, w, layer, dt, s, eps, off=off, pad=pad)
    some = _sample(n)
    part, f, uo = _rows(d, some), _bound(w), UBF if dt == "bf16" else U32
    h, u, mh, mu = _forward64(part, p, w, layer, s, eps)
    gh, gu = dev.forward()
    _close(gh[some], h, mh, f, uo)
    _close(gu[some], u, mu, f, uo)
    ih, iu = dev.forward(in_place=True)                    # rows are on their way while others are written
    assert dev.torch.equal(ih, gh) and dev.torch.equal(iu, gu)
    h = gh.double().cpu().numpy()
    dh, du = (rng.standard_normal((n, p * w)).astype(np.float32).astype(np.float64) for _ in range(2))
    want, mag = _backward64(part, h[some], dh[some], du[some], p, w, layer, s, eps)
    got = dev.backward(h, dh, du)
    for k in ("dx", "dy") + (("dgate",) if gate else ()):
        _close(got[k][some], want[k], mag[k], f)
    there = dev.backward(h, dh, du, in_place=True)
    assert all(dev.torch.equal(there[k], got[k]) for k in got)
    dev.untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("n,p,w,off,pad", SHAPES + [(45_003, 4, 64, 0, 0), (9_001, 1, 512, 0, 0), (5_001, 1, 1024, 0, 0), (2_003, 1, 2048, 0, 0)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_sums_over_the_rows(n, p, w, off, pad, dt):
    """Whole numbers in dh and du, scale 1 and no gate: the biases' gradients are their column sums, and with rows of +-1 and a width
    that is a power of two (plain norm, N = the row itself) so are the weights' of the products; fp32 holds them all exactly."""
    rng = np.random.default_rng(n)
    sign = lambda: rng.integers(0, 2, (n, p * w)) * 2.0 - 1.0                       # noqa: E731
    d = {"x": None, "y": sign(), "gate": None, "vec": dict.fromkeys(("w_post", "b_post", "w_pre", "b_pre"))}
    h = sign()
    dh, du = (rng.integers(-3, 4, (n, p * w)).astype(np.float64) for _ in range(2))
    dev = _Device(d, n, p, w, False, dt, 1.0, 1e-30, off=off, pad=pad)
    exact = w & (w - 1) == 0

    def same(got, k, want):
        assert np.array_equal(got[k].double().cpu().numpy(), want.sum(0)), k
    got = dev.backward(h, None, du)                        # D is not whole here, but du's sums are
    same(got, "db_pre", du)
    if exact:
        same(got, "dw_pre", du * h)
    got = dev.backward(h, dh, None)                        # D = dh
    same(got, "db_post", dh)
    if exact:
        same(got, "dw_post", dh * d["y"])
    without = dev.backward(h, dh, du, skip=("db_post", "db_pre"))
    if exact:
        same(without, "dw_pre", du * h)
    dev.untouched()
