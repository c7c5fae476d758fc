"""The embedding gradient where there are very many ids: runs that do not stay in registers, three passes of the sort, several
batches per unit of the sums, ids that reach over many CTAs, and the largest number of ids a call takes.

The values are small whole numbers and the scale is a power of two, so that every sum is exact in fp32 in any order: results have
to be equal.
"""
import pytest


def _gradient(ids, dout, vocab, scale):
    import torch
    from paper_2408_11500_b200 import binding as B
    n, width = dout.shape
    d = B.make_embed_desc(n, vocab, width, scale=scale, dout_ld=dout.stride(0))
    wsb = B.slicegcn_embed_workspace_bytes(d)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = torch.full((vocab, width), float("nan"), device="cuda")
    B.slicegcn_embed_backward(d, ids, dout, out, None, ws, wsb, torch.cuda.current_stream().cuda_stream)
    return out


@pytest.mark.gpu
def test_as_many_ids_as_31_bits_hold():
    """Position i has id i mod V and the value (i div V) mod 5 - 2: the sum over an id with c positions is known."""
    import torch
    n, vocab, chunk = 2 ** 31 - 1, 300_007, 1 << 27
    ids = torch.empty(n, dtype=torch.int32, device="cuda")
    dout = torch.empty((n, 1), device="cuda")
    for a in range(0, n, chunk):
        i = torch.arange(a, min(n, a + chunk), device="cuda")
        ids[a:a + chunk] = i % vocab
        dout[a:a + chunk, 0] = (i // vocab) % 5 - 2
    got = _gradient(ids, dout, vocab, 2.0)
    count = (n - torch.arange(vocab, device="cuda") + vocab - 1) // vocab
    first = torch.tensor([0, -2, -3, -3, -2], device="cuda")     # of the first c mod 5 values; five in a row add up to nothing
    assert torch.equal(got[:, 0], 2.0 * first[count % 5])


# many positions per unit and per CTA, runs of the sort that are read again, three digits, ids over 2 to 16 CTAs of the sums and over more
CASES = [(2_449_029, 2_449_029, 4, "own"), (2_449_029, 2_449_029, 7, "own"), (1_500_000, 300_007, 8, "zipf"), (2_000_003, 262_144, 16, "uniform"),
         (2_449_029, 200_003, 100, "zipf"), (1_300_000, 2_000_000, 7, "zipf"), (300_000, 1_500_000, 33, "zipf"), (1_600_000, 5, 12, "uniform"),
         (1_500_000, 100, 3, "uniform"), (1_250_000, 3, 32, "hub"), (160_000, 70_001, 131, "zipf"), (2_400_000, 40, 20, "runs"), (700_000, 1_000, 300, "zipf"),
         (20_000, 2_000_000, 20, "zipf"), (100_000, 400_000, 131, "zipf"), (9_000, 500_000, 5, "uniform"), (30_001, 120_004, 130, "uniform"),
         (8_192, 900_001, 33, "zipf"), (5_000, 300_000, 262, "zipf"), (1_000, 60_000, 1_433, "uniform"), (8, 1_000_003, 6, "uniform"), (0, 100_003, 9, "uniform"),
         (70_000, 280_000, 1, "uniform"), (50_000, 3_000, 2, "zipf"), (60_000, 60_000, 6, "own"), (400_000, 20, 6, "hub"), (90_000, 2, 8, "uniform"), (5, 1, 3, "uniform"), (1_024, 1, 5, "uniform"), (1_025, 1, 5, "uniform"), (4_096, 4, 33, "uniform"), (8_192, 8, 131, "hub"), (8_192, 7, 131, "hub"), (8_000, 20, 12, "zipf"), (300, 400, 40_000, "uniform"), (8_192, 9_699_000, 2, "uniform"), (8_000, 40_000, 2, "zipf"), (17, 90_000, 3, "uniform")]


def _ids(n, vocab, kind):
    import math
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(n + vocab)
    if kind == "own":
        ids = torch.randperm(vocab, generator=g, device="cuda")[:n]
    elif kind == "runs":                                   # every id as often, in order: sums of many CTAs each
        ids = torch.arange(n, device="cuda") * vocab // n
    else:
        ids = torch.randint(0, vocab, (n,), generator=g, device="cuda")
        if kind == "zipf":
            ids = torch.exp(torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * math.log(vocab + 1.0)).long().sub_(1).clamp_(0, vocab - 1)
            ids = (ids * 1_000_003 + 7) % vocab
        if kind == "hub":
            ids[torch.rand(n, generator=g, device="cuda") < 0.7] = vocab - 1
        ids[torch.rand(n, generator=g, device="cuda") < 0.02] = -1
    return ids.to(torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("n,vocab,width,kind", CASES)
@pytest.mark.parametrize("gap,start", [(0, 0), (4, 0), (3, 1)], ids=["dense", "rows apart", "odd start"])
def test_sums_are_exact(n, vocab, width, kind, gap, start):
    """Overwriting and adding, in tables whose rows follow one another or lie apart; nothing outside the rows changes."""
    import torch
    from paper_2408_11500_b200 import binding as B
    ids = _ids(n, vocab, kind)
    g = torch.Generator(device="cuda")
    g.manual_seed(width)
    dout = torch.randint(-3, 4, (n, width), generator=g, device="cuda").float()
    known = (ids >= 0).nonzero()[:, 0]
    want = torch.zeros((vocab, width), device="cuda", dtype=torch.float64).index_add_(0, ids[known].long(), dout[known].double()).mul_(2.0)
    big = torch.full((vocab * (width + gap) + start + 8,), 9.0, device="cuda")
    table = big[start:start + vocab * (width + gap)].view(vocab, width + gap)[:, :width]
    for accumulate in (False, True):
        table.fill_(3.0 if accumulate else float("nan"))
        d = B.make_embed_desc(n, vocab, width, scale=2.0, accumulate=accumulate, dtable_ld=width + gap)
        wsb = B.slicegcn_embed_workspace_bytes(d)
        ws = torch.randint(0, 256, (wsb,), dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.slicegcn_embed_backward(d, ids, dout, table, status, ws, wsb, torch.cuda.current_stream().cuda_stream)
        assert torch.equal(table.double(), want + (3.0 if accumulate else 0.0)) and status.item() == 0
        assert bool((big[:start] == 9).all()) and bool((big[start + vocab * (width + gap):] == 9).all())
        if gap:
            assert bool((big[start:start + vocab * (width + gap)].view(vocab, width + gap)[:, width:] == 9).all())


@pytest.mark.gpu
@pytest.mark.parametrize("width", [1, 2, 3, 5, 6, 7, 8, 11, 33, 130])
@pytest.mark.parametrize("n,vocab,kind", [(20_000, 700, "zipf"), (30_000, 30_000, "own"), (2_000, 90, "zipf")])
@pytest.mark.parametrize("ld,start", [(0, 1), (0, 3), (3, 2), (4, 0)])
def test_rows_of_dout_at_every_start(n, vocab, kind, width, ld, start):
    """What lies between the rows, before the first and behind the last is never taken (NaN)."""
    import torch
    from paper_2408_11500_b200 import binding as B
    ids = _ids(n, vocab, kind)
    big = torch.full((n * (width + ld) + start + 3,), float("nan"), device="cuda")
    dout = big[start:start + n * (width + ld)].view(n, width + ld)[:, :width]
    g = torch.Generator(device="cuda")
    g.manual_seed(width)
    dout.copy_(torch.randint(-3, 4, (n, width), generator=g, device="cuda").float())
    known = (ids >= 0).nonzero()[:, 0]
    want = torch.zeros((vocab, width), device="cuda", dtype=torch.float64).index_add_(0, ids[known].long(), dout[known].double())
    d = B.make_embed_desc(n, vocab, width, dout_ld=width + ld)
    wsb = B.slicegcn_embed_workspace_bytes(d)
    ws = torch.randint(0, 256, (wsb,), dtype=torch.uint8, device="cuda")
    out = torch.full((vocab, width), float("nan"), device="cuda")
    B.slicegcn_embed_backward(d, ids, dout, out, None, ws, wsb, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(out.double(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("n,vocab,width", [(3_000, 700_001, 33), (3_000, 700_001, 64), (20_000, 300_000, 7), (20_000, 300_000, 131), (300_000, 270_000, 5), (60_000, 60_000, 40)])
def test_replayed_and_on_another_stream(n, vocab, width):
    """Launches that overlap do so in a graph and on a side stream as well; every replay starts from other contents."""
    import torch
    from paper_2408_11500_b200 import binding as B
    ids = _ids(n, vocab, "zipf")
    dout = torch.randint(-3, 4, (n, width), device="cuda").float()
    want = _gradient(ids, dout, vocab, 2.0)
    out = torch.empty_like(want)
    d = B.make_embed_desc(n, vocab, width, scale=2.0)
    wsb = B.slicegcn_embed_workspace_bytes(d)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out.fill_(5.0)
        B.slicegcn_embed_backward(d, ids, dout, out, None, ws, wsb, torch.cuda.current_stream().cuda_stream)
        doubled = out * 2.0
    for _ in range(20):
        graph.replay()
        assert torch.equal(out, want) and torch.equal(doubled, 2.0 * want)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            out.fill_(float("nan"))
            B.slicegcn_embed_backward(d, ids, dout, out, None, ws, wsb, side.cuda_stream)
            assert torch.equal(out, want)
