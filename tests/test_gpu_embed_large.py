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
