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
