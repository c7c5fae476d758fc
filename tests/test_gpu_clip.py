"""The global gradient norm and clipping by it, against the definition in 64 bits.

Tolerances: the squares are taken and added in 64 bits (errors below 1e-9 at these sizes), so the norm is off by its
rounding to fp32, 2^-24, and a clipped fp32 value by the rounding of the factor and of the product, 2 * 2^-24 (doubled for
second-order terms); bf16 values by one more rounding, 2^-9.
"""
import math

import numpy as np
import pytest

U32, UBF = 2.0 ** -24, 2.0 ** -9


def _clip(tensors, max_norm, in_place=False, norm_only=False, stream=None):
    import torch
    from paper_2408_11500_b200 import binding as B
    dst = None if norm_only else tensors if in_place else [torch.full_like(t, float("nan")) for t in tensors]
    norm = torch.full((1,), float("nan"), device="cuda")
    wsb = B.slicegcn_clip_workspace_bytes()
    ws = torch.randint(0, 256, (wsb,), dtype=torch.uint8, device="cuda")
    B.slicegcn_clip_grads(B.make_tensor_list(tensors, dst), max_norm, norm, ws, wsb, stream)
    return dst, norm


def _check(src, dst, norm, max_norm):
    true = math.sqrt(sum(float(t.double().pow(2).sum()) for t in src))
    assert abs(float(norm) - true) <= 2 * U32 * true
    f = max_norm / true if true > max_norm else 1.0
    for a, b in zip(src, dst or []):
        want = a.double() * f
        u = UBF if b.element_size() == 2 else 0.0
        assert bool(((b.double() - want).abs() <= (4 * U32 + 2 * u) * want.abs()).all())
        if true < max_norm * (1 - 1e-6):
            assert bool((a == b).all())


SIZES = [[1], [5, 0, 3], [1000, 1, 4096, 4097], [1433 * 16, 16, 16 * 7, 7], [200_003, 64, 65_536, 13, 100], [7] * 300, [2_000_001],
         [169_343 * 128, 4096, 32, 256 * 256, 40], [64 * 1024 * 1024 + 5, 17], [128] * 512]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES, ids=[str(k) for k in range(len(SIZES))])
@pytest.mark.parametrize("types", ["f32", "bf16", "mixed"])
def test_clipping(sizes, types):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(len(sizes))
    pick = {"f32": lambda i: torch.float32, "bf16": lambda i: torch.bfloat16, "mixed": lambda i: (torch.float32, torch.bfloat16)[i % 2]}[types]
    src = [torch.randn(n, generator=g, device="cuda").mul_(0.1).to(pick(i)) for i, n in enumerate(sizes)]
    true = math.sqrt(sum(float(t.double().pow(2).sum()) for t in src))
    for max_norm in (0.3 * true, 2.0 * true, math.inf):
        dst, norm = _clip(src, max_norm)
        _check(src, dst, norm, max_norm)
        again, norm2 = _clip(src, max_norm)
        assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(dst, again))
        assert torch.equal(_clip(src, max_norm, norm_only=True)[1], norm)
    copies = [t.clone() for t in src]
    _clip(copies, 0.3 * true, in_place=True)
    want = _clip(src, 0.3 * true)[0]
    assert all(torch.equal(a, b) for a, b in zip(copies, want))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("a,b", [(1, 1), (1, 2), (3, 0), (2, 6), (4, 4)])
def test_odd_starts(dt, a, b):
    """Sources and destinations that start off any 16-byte boundary, each at its own place; neighbours stay as they are."""
    import torch
    t = torch.float32 if dt == "f32" else torch.bfloat16
    base, out = torch.randn(30_020, device="cuda").to(t), torch.full((30_020,), 9.0, device="cuda", dtype=t)
    from paper_2408_11500_b200 import binding as B
    norm, wsb = torch.zeros(1, device="cuda"), B.slicegcn_clip_workspace_bytes()
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    B.slicegcn_clip_grads(B.make_tensor_list([base[a:a + 30_001]], [out[b:b + 30_001]]), 2.0, norm, ws, wsb)
    _check([base[a:a + 30_001]], [out[b:b + 30_001]], norm, 2.0)
    assert bool((out[:b] == 9).all()) and bool((out[b + 30_001:] == 9).all())


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e20, 3e38])
def test_squares_outside_fp32(size):
    """Gradients whose squares (or their sum) fp32 cannot hold still have a norm and are clipped by it."""
    import torch
    src = [torch.full((1000,), size, device="cuda"), torch.full((17,), -size, device="cuda")]
    true = float(src[0][0].double()) * math.sqrt(1017)
    dst, norm = _clip(src, size / 2)
    if true < 3.4e38:
        assert abs(float(norm) - true) <= 2 * U32 * true
    else:
        assert math.isinf(float(norm))                     # the norm itself is past fp32; the factor is not
    want = size / 2 / math.sqrt(1017)
    assert bool(((dst[0].double() - want).abs() <= 8 * U32 * want).all()) and bool(((dst[1].double() + want).abs() <= 8 * U32 * want).all())


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_changes_nothing(value):
    import torch
    src = [torch.randn(5000, device="cuda"), torch.randn(33, device="cuda").to(torch.bfloat16)]
    src[0][4321] = value
    dst, norm = _clip(src, 1.0)
    assert not math.isfinite(float(norm))
    assert all(torch.equal(torch.nan_to_num(a, nan=123.0), torch.nan_to_num(b, nan=123.0)) for a, b in zip(src, dst))


@pytest.mark.gpu
def test_zero_gradients_and_empty_lists():
    import torch
    src = [torch.zeros(100, device="cuda"), torch.empty(0, device="cuda")]
    dst, norm = _clip(src, 1.0)
    assert float(norm) == 0.0 and bool((dst[0] == 0).all())
    assert float(_clip([], 1.0)[1]) == 0.0
    assert float(_clip([torch.empty(0, device="cuda")], 1.0)[1]) == 0.0


@pytest.mark.gpu
def test_on_another_stream():
    import torch
    side = torch.cuda.Stream()
    src = [torch.zeros(3_000_000, device="cuda"), torch.zeros(77, device="cuda")]
    host = [torch.randn(t.numel()).pin_memory() for t in src]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for t, h in zip(src, host):
            t.copy_(h, non_blocking=True)
        dst, norm = _clip(src, 1.0, stream=side.cuda_stream)
    side.synchronize()
    _check(src, dst, norm, 1.0)


@pytest.mark.gpu
def test_more_elements_than_32_bits_hold():
    import torch
    src = torch.zeros(2 ** 31 + 100, device="cuda", dtype=torch.bfloat16)
    src[-1], src[-2], src[0] = 3.0, 4.0, 12.0
    dst, norm = _clip([src], 6.5)
    assert float(norm) == 13.0 and float(dst[0][-1]) == 1.5 and float(dst[0][0]) == 6.0 and int(torch.count_nonzero(dst[0])) == 3


def test_refusals():
    from paper_2408_11500_b200 import binding as B
    import ctypes
    b = np.zeros(4096, np.float32)                         # host memory: every call below is refused before a launch
    at = b.ctypes.data

    def tl(count=1, src=(at,), dst=(at,), elems=(8,), dtypes=(0,), drop=()):
        d = B.TensorList()
        keep = ((ctypes.c_void_p * len(src))(*src), (ctypes.c_void_p * len(dst))(*dst), (ctypes.c_int64 * len(elems))(*elems),
                (ctypes.c_int32 * len(dtypes))(*dtypes))
        d.count = count
        for (k, t), v in zip(B.TensorList._fields_[1:], keep):
            if k not in drop:
                setattr(d, k, ctypes.cast(v, t))
        d._keep = keep
        return B._with_address(d)

    def refused(status, lst, max_norm=1.0, norm=b, ws=b, wsb=b.nbytes):
        with pytest.raises(B.SliceGCNError) as e:
            B.slicegcn_clip_grads(lst, max_norm, norm, ws, wsb)
        assert e.value.status == status and str(e.value)
    for bad in (dict(count=-1), dict(drop=("src",)), dict(drop=("elems",)), dict(src=(None,)), dict(dst=(None,)), dict(elems=(-1,)),
                dict(dtypes=(5,)), dict(src=(at + 2,)), dict(dst=(at + 1,))):
        refused(B.ERR_INVALID_ARG, tl(**bad))
    many = B.MAX_TENSORS + 1
    refused(B.ERR_UNSUPPORTED, tl(many, (at,) * many, (at,) * many, (1,) * many, (0,) * many))
    for max_norm in (0.0, -1.0, math.nan):
        refused(B.ERR_INVALID_ARG, tl(), max_norm=max_norm)
    refused(B.ERR_INVALID_ARG, tl(drop=("dst",)), norm=None)
    refused(B.ERR_INVALID_ARG, tl(), norm=at + 2)
    refused(B.ERR_INVALID_ARG, tl(), ws=at + 4)
    need = B.slicegcn_clip_workspace_bytes()
    refused(B.ERR_ALLOC, tl(), wsb=need - 1)
    refused(B.ERR_ALLOC, tl(), ws=None)
