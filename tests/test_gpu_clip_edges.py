"""Clipping where its kernels have the least to do and the least room: lists of no or few pieces (CTAs of the cluster that own
nothing), the tolerances being those of the 64-bit definition in `test_gpu_clip.py`.
"""
import math

import pytest

U32 = 2.0 ** -24


def _call(src, max_norm, times=1):
    """`times` calls back to back on their own outputs."""
    import torch
    from paper_2408_11500_b200 import binding as B
    wsb = B.slicegcn_clip_workspace_bytes()
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    outs = [[torch.full_like(t, math.nan) for t in src] for _ in range(times)]
    norms = torch.full((times,), math.nan, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    lists = [B.make_tensor_list(src, o) for o in outs]
    for k, t in enumerate(lists):
        B.slicegcn_clip_grads(t, max_norm, norms[k:], ws, wsb, st)
    return outs, norms


@pytest.mark.gpu
@pytest.mark.parametrize("pieces", [0, 1, 2, 7, 8, 9, 63, 64])
def test_clusters_with_ctas_that_own_nothing(pieces):
    """Tensors of a few numbers, one piece each; many launches behind one another, all of which must give the same."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(pieces)
    src = [torch.randn(3 + k, generator=g, device="cuda") for k in range(min(pieces, 32))]
    if pieces > 32:
        src[-1] = torch.randn((pieces - 32) * 4096 + 1, generator=g, device="cuda")     # 16 KB a piece
    true = math.sqrt(sum(float(t.double().pow(2).sum()) for t in src))
    outs, norms = _call(src, 0.5 * true if pieces else 1.0, times=100)
    assert bool(((norms.double() - true).abs() <= 2 * U32 * true).all())
    for out in outs:
        for a, b in zip(src, out):
            assert bool(((b.double() - 0.5 * a.double()).abs() <= 4 * U32 * a.double().abs()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("count", [1017, 2_000_001])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size,max_norm", [(3e38, 1e-3), (3e38, 1e-5), (1e37, 1e-6), (1e30, 1e-20), (2.0, 1e-37)])
def test_factors_below_the_normal_numbers(size, max_norm, dt, count):
    """One rounding of the product, which may itself lie below the normal numbers (2^-149 apart)."""
    import torch
    src = torch.full((count,), size, device="cuda", dtype=torch.float32 if dt == "f32" else torch.bfloat16)
    src[1::2] *= -0.37
    true = math.sqrt(float(src.double().pow(2).sum()))
    (out,), norm = (v[0] for v in _call([src], max_norm))
    want = src.double() * (max_norm / true)
    u = U32 if dt == "f32" else 2.0 ** -9
    assert bool(((out.double() - want).abs() <= 2 * u * want.abs() + (2.0 ** -149 if dt == "f32" else 2.0 ** -133)).all())
    assert bool((out != 0).any())
    assert math.isinf(float(norm)) if true > 3.41e38 else abs(float(norm) - true) <= 2 * U32 * true
