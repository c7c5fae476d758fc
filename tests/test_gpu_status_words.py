"""A status word that several calls share keeps what each of them has set."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,vocab", [(300, 40), (200_000, 1000)], ids=str)
def test_bad_ids_leave_an_expired_wait_in_the_word(n, vocab):
    """Lookup and gradient, small and sorted forms, in a word that holds the bit of a wait that ran out."""
    import torch
    from paper_2408_11500_b200 import binding as B
    ids = torch.randint(0, vocab, (n,), dtype=torch.int32, device="cuda")
    ids[n // 2] = vocab
    table, out = torch.randn((vocab, 8), device="cuda"), torch.empty((n, 8), device="cuda")
    d = B.make_embed_desc(n, vocab, 8)
    ws = torch.empty(B.slicegcn_embed_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    status = torch.tensor([B.DEVSTATUS_WAIT], dtype=torch.int32, device="cuda")
    B.slicegcn_embed_forward(d, ids, table, out, status)
    assert int(status) == B.DEVSTATUS_WAIT | B.DEVSTATUS_BAD_ID
    status.fill_(B.DEVSTATUS_WAIT)
    B.slicegcn_embed_backward(d, ids, out, table, status, ws, ws.numel())
    assert int(status) == B.DEVSTATUS_WAIT | B.DEVSTATUS_BAD_ID
    assert B.DEVSTATUS_WAIT & B.DEVSTATUS_BAD_ID == 0


def test_feed_forward_calls_leave_bad_ids_in_the_word():
    from paper_2408_11500_b200 import binding as B
    import torch
    n, k = 500, 96
    x, W, out = torch.randn((n, k), device="cuda"), torch.randn((1, k, k), device="cuda"), torch.empty((n, k), device="cuda")
    d = B.make_ffn_desc(n, 1, k, k, W, act=B.ACT_SILU)
    need = max(B.slicegcn_ffn_workspace_bytes(d, x), B.slicegcn_ffn_workspace_bytes(d, x, out))
    ws, status = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.tensor([B.DEVSTATUS_BAD_ID], dtype=torch.int32, device="cuda")
    B.slicegcn_ffn_forward(d, x, None, out, status, ws, need)
    B.slicegcn_ffn_backward(d, x, out, torch.empty_like(x), torch.empty_like(W), None, None, None, status, ws, need)
    assert int(status) == B.DEVSTATUS_BAD_ID


def test_the_deep_model_reports_an_expired_wait_as_such():
    """Not as bad ids, and not silently."""
    from test_gpu_ffn_deep import _ff_model
    from paper_2408_11500_b200 import binding as B
    m, _ = _ff_model(100, 20, 32, 4, 1, 5, 2)
    m.step(0.1)
    m.check()
    assert int(m.waits) == 0 and int(m.status) == 0
    m.ids[3] = 20
    m.step(0.1)
    m.check()
    assert int(m.waits) == 0 and int(m.status) == B.DEVSTATUS_BAD_ID
    m.waits.fill_(B.DEVSTATUS_WAIT)                  # as a kernel leaves it
    with pytest.raises(RuntimeError, match="gave up a wait"):
        m.check()
    m.B.slicegcn_graph_destroy(m.g)
