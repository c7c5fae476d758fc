"""The operators together (`deep_epochs.py`): one step's gradients against 64-bit automatic differentiation of the whole
model with a dense aggregation matrix, clipping, and a few steps of training."""
import math

import numpy as np
import pytest

from helpers import rel_inf

pytestmark = pytest.mark.gpu


def _model(n, vocab, hidden, p, layers, classes, seed=0):
    import torch
    from deep_epochs import DeepSlicedGCN
    from oracle import slicegcn_oracle as orc
    from paper_2408_11500_b200 import binding as B, synth
    src, dst = synth.chung_lu_powerlaw(n, 4 * n, 2.2, 60, seed=seed)
    g = B.slicegcn_graph_create(n, src, dst, B.SYMMETRIZE | B.ADD_SELF_LOOPS)
    A = orc.spmm(orc.build_graph(n, src, dst, True, True), np.eye(n))
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, vocab, n).astype(np.int32)
    ids[::17] = -1
    m = DeepSlicedGCN(g, torch.from_numpy(ids).cuda(), torch.from_numpy(synth.uniform_labels(n, classes, seed)).cuda(), vocab, hidden, p, layers, classes)
    return m, torch.from_numpy(A).cuda()


def _loss64(m, A, P):
    """The model in 64 bits, from its definition."""
    import torch

    def norm(t):
        t = t.view(m.n, m.p, m.h_s)
        return (t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + 1e-5)).reshape(m.n, -1)
    known = (m.ids >= 0)[:, None]
    x = torch.where(known, m.scale * P["table"][m.ids.clamp(min=0).long()], 0.0)
    u = norm(x) * P["w_pre.0"]
    for i in range(m.layers):
        agg, blocks = A @ u, []
        for k in range(m.p):
            cols = slice(k * m.h_s, (k + 1) * m.h_s)
            blocks.append(torch.relu(P[f"b.{i}"][k] + agg[:, cols] @ P[f"W_agg.{i}"][k]) + u[:, cols] @ P[f"W_self.{i}"][k])
        x = x + m.s * torch.sigmoid(u) * (norm(torch.cat(blocks, 1)) * P[f"w_post.{i}"])
        u = norm(x) * P[f"w_pre.{i + 1}"]
    logits = u @ P["Wc"] + P["bc"]
    return torch.nn.functional.cross_entropy(logits, m.labels), logits


@pytest.mark.parametrize("n,vocab,hidden,p,layers", [(300, 40, 32, 4, 3), (257, 257, 96, 1, 2), (200, 7, 24, 2, 5)])
def test_gradients_of_the_whole_model(n, vocab, hidden, p, layers):
    """The framework's own gate for fp32 gradients, 1e-4 of the largest entry per tensor."""
    import torch
    m, A = _model(n, vocab, hidden, p, layers, 5)
    P = {k: v.double().requires_grad_(True) for k, v in m.params.items()}
    want_loss, want_logits = _loss64(m, A, P)
    grads = torch.autograd.grad(want_loss, list(P.values()))
    logits = m.forward()
    loss = m.backward(logits)
    assert rel_inf(logits.cpu().numpy(), want_logits.detach().cpu().numpy()) <= 1e-4
    assert abs(float(loss) - want_loss.item()) <= 1e-4 * want_loss.item()
    for (k, got), want in zip(m.grads.items(), grads):
        assert rel_inf(got.cpu().numpy(), want.cpu().numpy()) <= 1e-4, k
    m.max_norm = 1e-3
    m.clip()
    true = math.sqrt(sum(float(v.double().pow(2).sum()) for v in m.grads.values()))
    assert true > m.max_norm and abs(float(m.norm) - true) <= 1e-6 * true
    assert all(rel_inf(m.clipped[k].cpu().numpy(), (m.grads[k].double() * (m.max_norm / true)).cpu().numpy()) <= 1e-6 for k in m.grads)
    assert int(m.status) == 0
    m.B.slicegcn_graph_destroy(m.g)


def test_training_reduces_the_loss():
    m, _ = _model(400, 400, 64, 4, 6, 7, seed=3)
    losses = [float(m.step(0.5)) for _ in range(40)]
    assert np.isfinite(losses).all() and losses[-1] < 0.7 * losses[0]
    m.B.slicegcn_graph_destroy(m.g)


def test_every_call_can_be_captured_in_a_graph():
    """No call allocates, synchronises or reads back, so a step of all of them replays from a CUDA graph, small and large forms."""
    import torch
    from paper_2408_11500_b200 import binding as B
    torch.manual_seed(0)
    for n, vocab, p, w, extra in [(900, 70, 4, 24, 10), (30_000, 500, 1, 300, 400_000), (50, 9, 1, 1500, 7)]:
        cols = p * w
        ids = torch.randint(0, vocab, (n,), dtype=torch.int32, device="cuda")
        table, dtable = torch.randn((vocab, cols), device="cuda"), torch.empty((vocab, cols), device="cuda")
        x, y, h, u, dx, dy = (torch.randn((n, cols), device="cuda") for _ in range(6))
        dw, big, out = torch.empty(cols, device="cuda"), torch.randn(extra, device="cuda"), torch.empty(extra, device="cuda")
        norm = torch.zeros(1, device="cuda")
        e, r = B.make_embed_desc(n, vocab, cols), B.make_residual_norm_desc(n, p, w)
        clipped = torch.empty_like(dtable)
        t = B.make_tensor_list([dtable, big], [clipped, out])
        wsb = max(B.slicegcn_embed_workspace_bytes(e), B.slicegcn_residual_norm_workspace_bytes(r), B.slicegcn_clip_workspace_bytes())
        ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")

        def step():
            st = torch.cuda.current_stream().cuda_stream
            B.slicegcn_embed_forward(e, ids, table, x, None, st)
            B.slicegcn_residual_norm_forward(r, x, y, None, h, u, st)
            B.slicegcn_residual_norm_backward(r, y, None, h, u, x, dx, dy, None, None, None, dw, None, ws, wsb, st)
            B.slicegcn_embed_backward(e, ids, dx, dtable, None, ws, wsb, st)
            B.slicegcn_clip_grads(t, 1.0, norm, ws, wsb, st)
        step()
        torch.cuda.synchronize()
        want = [v.clone() for v in (x, h, u, dx, dy, dw, dtable, clipped, out, norm)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for v in (x, h, u, dx, dy, dw, dtable, clipped, out, norm):
            v.fill_(7.0)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((x, h, u, dx, dy, dw, dtable, clipped, out, norm), want))
