"""Embedding lookup and its gradient against the definition in 64 bits (numpy, on the host).

Tolerances, from the arithmetic.  u = 2^-24 (fp32), 2^-9 (bf16).  Lookup: scale is rounded to fp32, one product, one
rounding to the output type: |err| <= (2u + u_out)|value|, doubled for second order terms.  Gradient: every summand is one
fp32 product with a rounded scale (2u), and any order of adding m of them in fp32 is off by at most m u sum|summand|:
|err| <= (m + 3) u sum|summand|.
"""
import numpy as np
import pytest

U32, UBF = 2.0 ** -24, 2.0 ** -9


def _ids(rng, n, vocab, kind):
    if kind == "hub":                      # one id holds most positions, the rest are spread
        ids = rng.integers(0, vocab, n)
        ids[rng.random(n) < 0.7] = vocab // 2
    elif kind == "same":
        ids = np.full(n, vocab - 1)
    elif kind == "own":
        ids = rng.permutation(vocab)[:n]
    elif kind == "none":
        ids = np.full(n, -1)
    else:
        ids = rng.integers(0, vocab, n)
        ids[rng.random(n) < 0.2] = -1
    return ids.astype(np.int32)


def _backward(torch, B, ids, dout, vocab, width, scale, dtable=None, accumulate=False, status=None, stream=None):
    if dtable is None:
        dtable = torch.full((vocab, width), float("nan"), device="cuda")
    d = B.make_embed_desc(ids.numel(), vocab, width, scale=scale, accumulate=accumulate, dout_ld=dout.stride(0) if dout.dim() else width,
                          dtable_ld=dtable.stride(0))
    wsb = B.slicegcn_embed_workspace_bytes(d)
    ws = torch.randint(0, 256, (wsb,), dtype=torch.uint8, device="cuda")     # contents undefined: anything must do
    B.slicegcn_embed_backward(d, ids, dout, dtable, status, ws, wsb, stream)
    return dtable


def _check_gradient(got, ids, dout, vocab, scale, base=None):
    ok = ids >= 0
    want, size, count = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1])), np.zeros(vocab)
    np.add.at(want, ids[ok], scale * dout[ok].astype(np.float64))
    np.add.at(size, ids[ok], np.abs(scale * dout[ok].astype(np.float64)))
    np.add.at(count, ids[ok], 1)
    if base is not None:
        want, size, count = want + base, size + np.abs(base), count + 1
    assert np.all(np.abs(got - want) <= (count[:, None] + 3) * U32 * size)


CASES = [(1, 7, 128, "spread"), (33, 5, 13, "hub"), (1000, 40, 1, "spread"), (2708, 1433, 16, "spread"), (4097, 300, 100, "hub"),
         (5000, 70001, 32, "spread"), (20000, 3, 47, "hub"), (9000, 9000, 128, "own"), (300, 50, 1433, "hub"), (513, 1, 4, "same"),
         (12289, 256, 260, "spread"), (40000, 65536, 8, "spread"), (700, 91, 600, "none"), (60000, 17, 64, "same"), (31, 300000, 24, "spread")]


@pytest.mark.gpu
@pytest.mark.parametrize("n,vocab,width,kind", CASES)
@pytest.mark.parametrize("tdt,odt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_lookup(n, vocab, width, kind, tdt, odt):
    import torch
    from paper_2408_11500_b200 import binding as B
    rng = np.random.default_rng(n + width)
    types = {"f32": (torch.float32, B.F32, 0.0), "bf16": (torch.bfloat16, B.BF16, UBF)}
    ids = _ids(rng, n, vocab, kind)
    table = torch.from_numpy(rng.standard_normal((vocab, width)).astype(np.float32)).cuda().to(types[tdt][0])
    out = torch.full((n, width), float("nan"), device="cuda", dtype=types[odt][0])
    scale = 3.3
    d = B.make_embed_desc(n, vocab, width, scale=scale, table_dtype=types[tdt][1], out_dtype=types[odt][1])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.slicegcn_embed_forward(d, torch.from_numpy(ids).cuda(), table, out, status, torch.cuda.current_stream().cuda_stream)
    want = np.where((ids >= 0)[:, None], scale * table.double().cpu().numpy()[np.maximum(ids, 0)], 0.0)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= 2 * (2 * U32 + types[odt][2]) * np.abs(want))
    assert status.item() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n,vocab,width,kind", CASES)
def test_gradient(n, vocab, width, kind):
    import torch
    from paper_2408_11500_b200 import binding as B
    rng = np.random.default_rng(n + width)
    ids, dout = _ids(rng, n, vocab, kind), rng.standard_normal((n, width)).astype(np.float32)
    args = (torch.from_numpy(ids).cuda(), torch.from_numpy(dout).cuda(), vocab, width, 0.7)
    got = _backward(torch, B, *args)
    _check_gradient(got.double().cpu().numpy(), ids, dout, vocab, 0.7)
    assert torch.equal(got, _backward(torch, B, *args))                       # the order of the sums is fixed
    base = torch.from_numpy(rng.standard_normal((vocab, width)).astype(np.float32)).cuda()
    keep = base.double().cpu().numpy()
    _backward(torch, B, *args, dtable=base, accumulate=True)
    _check_gradient(base.double().cpu().numpy(), ids, dout, vocab, 0.7, base=keep)


@pytest.mark.gpu
@pytest.mark.parametrize("width,off,pad", [(16, 1, 3), (100, 2, 5), (13, 4, 7), (128, 0, 4), (128, 4, 1), (47, 3, 0), (260, 1, 1)])
def test_strides_and_odd_starts(width, off, pad):
    """Columns of a wider matrix, at a start and a leading dimension that allow no wide accesses; neighbours stay as they are."""
    import torch
    from paper_2408_11500_b200 import binding as B
    rng = np.random.default_rng(width)
    n, vocab, ld = 777, 91, off + width + pad
    ids = _ids(rng, n, vocab, "spread")
    ids_d = torch.from_numpy(ids).cuda()
    dout = torch.from_numpy(rng.standard_normal((n, ld)).astype(np.float32)).cuda()
    dtable = torch.full((vocab, ld), 5.0, device="cuda")
    _backward(torch, B, ids_d, dout[:, off:off + width], vocab, width, 1.5, dtable=dtable[:, off:off + width])
    got = dtable.double().cpu().numpy()
    _check_gradient(got[:, off:off + width], ids, dout.cpu().numpy()[:, off:off + width], vocab, 1.5)
    assert np.all(got[:, :off] == 5) and np.all(got[:, off + width:] == 5)
    for odt, code, u in ((torch.float32, B.F32, 0.0), (torch.bfloat16, B.BF16, UBF)):
        table = torch.from_numpy(rng.standard_normal((vocab, ld)).astype(np.float32)).cuda()
        out = torch.full((n, ld), 5.0, device="cuda", dtype=odt)
        d = B.make_embed_desc(n, vocab, width, scale=1.5, out_dtype=code, table_ld=ld, out_ld=ld)
        B.slicegcn_embed_forward(d, ids_d, table[:, off:off + width], out[:, off:off + width])
        got = out.double().cpu().numpy()
        want = np.where((ids >= 0)[:, None], 1.5 * table.double().cpu().numpy()[np.maximum(ids, 0), off:off + width], 0.0)
        assert np.all(np.abs(got[:, off:off + width] - want) <= 2 * (2 * U32 + u) * np.abs(want))
        assert np.all(got[:, :off] == 5) and np.all(got[:, off + width:] == 5)


@pytest.mark.gpu
def test_bad_ids_are_skipped_and_reported():
    import torch
    from paper_2408_11500_b200 import binding as B
    rng = np.random.default_rng(0)
    n, vocab, width = 500, 37, 20
    ids = _ids(rng, n, vocab, "spread")
    ids[[3, 90, 91, 499]] = [vocab, 2 ** 31 - 1, -2, -2 ** 31]
    dout = rng.standard_normal((n, width)).astype(np.float32)
    dout[ids < 0] = np.nan                        # a row without an id takes no part, whatever it holds
    dout[ids >= vocab] = np.inf
    clean = np.where((ids >= 0) & (ids < vocab), ids, -1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = _backward(torch, B, torch.from_numpy(ids).cuda(), torch.from_numpy(dout).cuda(), vocab, width, 2.0, status=status)
    _check_gradient(got.double().cpu().numpy(), clean, np.where(clean[:, None] >= 0, dout, 0).astype(np.float32), vocab, 2.0)
    assert status.item() == B.DEVSTATUS_BAD_ID
    _backward(torch, B, torch.from_numpy(ids).cuda(), torch.from_numpy(dout).cuda(), vocab, width, 2.0)       # nobody asks: still skipped
    table, out = torch.randn((vocab, width), device="cuda"), torch.full((n, width), 9.0, device="cuda")
    status.zero_()
    d = B.make_embed_desc(n, vocab, width)
    B.slicegcn_embed_forward(d, torch.from_numpy(ids).cuda(), table, out, status)
    assert status.item() == B.DEVSTATUS_BAD_ID
    assert torch.equal(out, torch.where(torch.from_numpy(clean).cuda()[:, None] >= 0, table[torch.from_numpy(np.maximum(clean, 0)).cuda().long()], 0.0))


@pytest.mark.gpu
def test_no_ids():
    import torch
    from paper_2408_11500_b200 import binding as B
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    got = _backward(torch, B, empty, torch.empty((0, 12), device="cuda"), 9, 12, 1.0)
    assert torch.equal(got, torch.zeros_like(got))
    kept = torch.randn((9, 12), device="cuda")
    want = kept.clone()
    _backward(torch, B, empty, torch.empty((0, 12), device="cuda"), 9, 12, 1.0, dtable=kept, accumulate=True)
    assert torch.equal(kept, want)
    B.slicegcn_embed_forward(B.make_embed_desc(0, 9, 12), None, kept, None)


@pytest.mark.gpu
def test_non_finite_values_stay_in_their_rows():
    import torch
    from paper_2408_11500_b200 import binding as B
    ids = torch.tensor([0, 2, 2, 1, 3, 0], dtype=torch.int32, device="cuda")
    dout = torch.ones((6, 8), device="cuda")
    dout[1, 3], dout[3, 0] = float("inf"), float("nan")
    got = _backward(torch, B, ids, dout, 5, 8, 1.0)
    want = torch.tensor([2.0, 1.0, 2.0, 1.0, 0.0], device="cuda")[:, None].repeat(1, 8)
    want[2, 3], want[1, 0] = float("inf"), float("nan")
    assert torch.equal(torch.nan_to_num(got, nan=77.0), torch.nan_to_num(want, nan=77.0))


@pytest.mark.gpu
def test_gradient_is_the_adjoint_and_matches_differences():
    """The lookup is linear in the table: <lookup(T), G> = <T, gradient(G)>, and a step in one entry moves the sum by its gradient."""
    import torch
    from paper_2408_11500_b200 import binding as B
    rng = np.random.default_rng(5)
    n, vocab, width, scale = 3000, 211, 24, 1.25
    ids = torch.from_numpy(_ids(rng, n, vocab, "hub")).cuda()
    T, G = torch.randn((vocab, width), device="cuda"), torch.randn((n, width), device="cuda")
    d = B.make_embed_desc(n, vocab, width, scale=scale)

    def value(table):
        out = torch.empty((n, width), device="cuda")
        B.slicegcn_embed_forward(d, ids, table, out)
        return float((out.double() * G.double()).sum())
    grad = _backward(torch, B, ids, G, vocab, width, scale)
    size = float((T.double().abs() * grad.double().abs()).sum())
    assert abs(value(T) - float((T.double() * grad.double()).sum())) <= 3000 * U32 * size
    for v, c in [(105, 0), (3, 7), (210, 23)]:
        step = T.clone()
        step[v, c] += 0.5
        moved = float(step[v, c].double() - T[v, c].double())
        # both sides are sums over the positions of v: rounding of each lookup, then of the gradient's own sum
        rows = (ids == v).nonzero()[:, 0]
        bound = float(G[rows, c].double().abs().sum()) * scale * (4 * abs(float(step[v, c])) + rows.numel() + 4) * U32
        assert abs((value(step) - value(T)) - moved * float(grad[v, c])) <= 2 * bound


@pytest.mark.gpu
def test_on_another_stream():
    import torch
    from paper_2408_11500_b200 import binding as B
    rng = np.random.default_rng(8)
    n, vocab, width = 30000, 500, 64
    ids, dout = _ids(rng, n, vocab, "hub"), rng.standard_normal((n, width)).astype(np.float32)
    side = torch.cuda.Stream()
    ids_d, dout_d = torch.from_numpy(ids).cuda(), torch.zeros((n, width), device="cuda")
    src = torch.from_numpy(dout).pin_memory()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        dout_d.copy_(src, non_blocking=True)
        got = _backward(torch, B, ids_d, dout_d, vocab, width, 1.0, stream=side.cuda_stream)
    side.synchronize()
    _check_gradient(got.double().cpu().numpy(), ids, dout, vocab, 1.0)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A table and a gradient of more than 2^31 elements: the last rows are found and written."""
    import torch
    from paper_2408_11500_b200 import binding as B
    vocab, width = 4_300_000, 512
    assert vocab * width > 2 ** 31
    table = torch.zeros((vocab, width), device="cuda", dtype=torch.bfloat16)
    ids = torch.tensor([vocab - 1, 0, vocab - 2, vocab - 1, -1], dtype=torch.int32, device="cuda")
    table[-2:] = torch.randn((2, width), device="cuda").to(torch.bfloat16)
    out = torch.empty((5, width), device="cuda")
    B.slicegcn_embed_forward(B.make_embed_desc(5, vocab, width, scale=2.0, table_dtype=B.BF16), ids, table, out)
    want = 2.0 * table[ids.clamp(min=0).long()].float()
    want[4] = 0
    assert torch.equal(out, want)
    del table
    dout = torch.randn((5, width), device="cuda")
    got = _backward(torch, B, ids, dout, vocab, width, 1.0)
    assert torch.equal(got[vocab - 1], dout[0] + dout[3]) and torch.equal(got[vocab - 2], dout[2]) and torch.equal(got[0], dout[1])
    assert int(torch.count_nonzero(got[1:vocab - 2])) == 0 and int(torch.isnan(got).sum()) == 0


def test_refusals():
    from paper_2408_11500_b200 import binding as B
    buf = np.zeros(4096, np.float32)                       # host memory: every call below is refused before a launch
    ok = dict(n=4, vocab=8, width=4)

    def refused(status, call):
        with pytest.raises(B.SliceGCNError) as e:
            call()
        assert e.value.status == status and str(e.value)
    for bad in (dict(n=-1), dict(vocab=0), dict(width=0)):
        d = B.make_embed_desc(**{**ok, **bad})
        refused(B.ERR_INVALID_ARG, lambda: B.slicegcn_embed_forward(d, buf, buf, buf))
        refused(B.ERR_INVALID_ARG, lambda: B.slicegcn_embed_workspace_bytes(d))
        refused(B.ERR_INVALID_ARG, lambda: B.slicegcn_embed_backward(d, buf, buf, buf, None, buf, buf.nbytes))
    for bad in (dict(n=2 ** 31), dict(vocab=2 ** 31 - 1)):
        d = B.make_embed_desc(**{**ok, **bad})
        refused(B.ERR_OVERFLOW, lambda: B.slicegcn_embed_workspace_bytes(d))
    refused(B.ERR_UNSUPPORTED, lambda: B.slicegcn_embed_workspace_bytes(B.make_embed_desc(4, 8, (1 << 20) + 1)))
    for bad in (dict(table_ld=3), dict(out_ld=3), dict(table_dtype=7), dict(out_dtype=-1)):
        d = B.make_embed_desc(**{**ok, **bad})
        refused(B.ERR_INVALID_ARG, lambda: B.slicegcn_embed_forward(d, buf, buf, buf))
    for bad in (dict(dout_ld=3), dict(dtable_ld=3)):
        d = B.make_embed_desc(**{**ok, **bad})
        refused(B.ERR_INVALID_ARG, lambda: B.slicegcn_embed_backward(d, buf, buf, buf, None, buf, buf.nbytes))
    d = B.make_embed_desc(**ok)
    for args in ((None, buf, buf), (buf, None, buf), (buf, buf, None), (buf.ctypes.data + 2, buf, buf), (buf, buf.ctypes.data + 1, buf)):
        refused(B.ERR_INVALID_ARG, lambda: B.slicegcn_embed_forward(d, *args))
        refused(B.ERR_INVALID_ARG, lambda: B.slicegcn_embed_backward(d, *args, None, buf, buf.nbytes))
    refused(B.ERR_INVALID_ARG, lambda: B.slicegcn_embed_backward(d, buf, buf, buf, None, buf.ctypes.data + 4, 4000))
    need = B.slicegcn_embed_workspace_bytes(d)
    refused(B.ERR_ALLOC, lambda: B.slicegcn_embed_backward(d, buf, buf, buf, None, buf, need - 1))
    refused(B.ERR_ALLOC, lambda: B.slicegcn_embed_backward(d, buf, buf, buf, None, None, need))
