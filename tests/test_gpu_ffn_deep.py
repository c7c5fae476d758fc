"""The feed-forward blocks and AdamW as `deep_epochs.py` uses them, and the calls that its steps do not make: captured, on two
streams at once, in place, with outputs left out, on matrices whose offsets pass 32 bits."""
import math

import numpy as np
import pytest

from helpers import rel_inf
from test_gpu_deep import _model
from test_gpu_ffn import Problem

pytestmark = pytest.mark.gpu


def _ff_model(n, vocab, hidden, p, layers, classes, ff, adamw="", seed=0):
    import torch
    from deep_epochs import DeepSlicedGCN
    base, A = _model(n, vocab, hidden, p, layers, classes, seed)
    m = DeepSlicedGCN(base.g, base.ids, base.labels.int(), vocab, hidden, p, layers, classes, ff=ff, adamw=adamw)
    for k, v in m.params.items():                    # biases and scales that matter
        if k.startswith(("f.", "f_out.", "w_ff.")):
            v += torch.randn(v.shape, generator=torch.Generator("cuda").manual_seed(len(k)), device="cuda") * 0.2
    return m, A


def _loss64(m, A, P):
    import torch

    def norm(t):
        t = t.view(m.n, m.p, m.h_s)
        return (t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + 1e-5)).reshape(m.n, -1)

    def per_slice(t, W):
        return torch.einsum("nsi,sio->nso", t.view(m.n, m.p, -1), W)
    known = (m.ids >= 0)[:, None]
    x = torch.where(known, m.scale * P["table"][m.ids.clamp(min=0).long()], 0.0)
    u = norm(x) * P["w_pre.0"]
    for i in range(m.layers):
        M = per_slice(A @ u, P[f"W_agg.{i}"]) + P[f"b.{i}"]
        y = torch.relu(M) + per_slice(u, P[f"W_self.{i}"])
        x = x + m.s * torch.sigmoid(u) * (norm(y.reshape(m.n, -1)) * P[f"w_post.{i}"])
        u = norm(x) * P[f"w_ff.{i}"]
        a = per_slice(u, P[f"F_gate.{i}"]) + P[f"f.{i}"]
        h = a * torch.sigmoid(a) * per_slice(u, P[f"F_up.{i}"])
        x = x + m.s * (per_slice(h.reshape(m.n, -1), P[f"F_out.{i}"]) + P[f"f_out.{i}"]).reshape(m.n, -1)
        u = norm(x) * P[f"w_pre.{i + 1}"]
    return torch.nn.functional.cross_entropy(u @ P["Wc"] + P["bc"], m.labels)


@pytest.mark.parametrize("n,vocab,hidden,p,layers,ff", [(300, 40, 32, 4, 3, 2), (257, 257, 96, 1, 2, 3), (900, 70, 256, 8, 2, 4)])
def test_gradients_of_the_model_with_blocks(n, vocab, hidden, p, layers, ff):
    """The framework's own gate for fp32 gradients, 1e-4 of the largest entry per tensor; then differences along the gradient."""
    import torch
    m, A = _ff_model(n, vocab, hidden, p, layers, 5, ff)
    P = {k: v.double().requires_grad_(True) for k, v in m.params.items()}
    want = _loss64(m, A, P)
    grads = torch.autograd.grad(want, list(P.values()))
    loss = m.backward(m.forward())
    assert abs(float(loss) - want.item()) <= 1e-4 * want.item() and int(m.status) == 0
    for (k, got), g in zip(m.grads.items(), grads):
        assert rel_inf(got.cpu().numpy(), g.cpu().numpy()) <= 1e-4, k
    # the 64-bit loss moves along the call's own gradient as that gradient says
    for k in ("F_gate.0", "F_up.0", "F_out.0", "f.0", "f_out.0"):
        g = m.grads[k].double()
        step = 1e-4 / float(g.norm())
        hi, lo = (float(_loss64(m, A, {**{q: v.detach() for q, v in P.items()}, k: P[k].detach() + s * step * g})) for s in (1, -1))
        assert abs((hi - lo) / 2 - step * float(g.square().sum())) <= 1e-3 * step * float(g.square().sum()) + 1e-12, k
    m.B.slicegcn_graph_destroy(m.g)


@pytest.mark.parametrize("adamw", ["32bit", "8bit"])
def test_a_training_step_with_blocks_and_adamw(adamw):
    """Parameters after a step are those of the formula with the step's own gradients, and the steps run on."""
    import torch
    m, _ = _ff_model(300, 40, 32, 4, 2, 5, 2, adamw)
    m.max_norm = m.adamw.max_norm = 1e-3
    before = {k: v.double().clone() for k, v in m.params.items()}
    m.step(1e-3)
    true = math.sqrt(sum(float(v.double().pow(2).sum()) for v in m.grads.values()))
    for k, v in m.params.items():
        g = m.grads[k].double() * min(1.0, 1e-3 / true)
        keep = 1 - 1e-5 if v.dim() > 1 and not k.startswith(("b.", "f.", "f_out.")) else 1.0
        want = before[k] * keep - 1e-3 * g / (g.abs() + 1e-8)      # the first step's averages are the gradient's own
        # where |g| is far below eps the norm's and the factor's roundings (a few 2^-24) count by themselves
        assert bool(((v.double() - want).abs() <= 8 * 2.0 ** -24 * before[k].abs() + 1e-3 * 2e-5).all()), k
    losses = [float(m.step(1e-3)) for _ in range(5)]
    assert np.isfinite(losses).all() and m.count.tolist() == [6, 0]
    m.B.slicegcn_graph_destroy(m.g)


def test_captured_in_graphs_that_share_a_workspace():
    """Forward and gradients of several shapes and types, each in a graph of its own over one workspace, replayed one after another."""
    import torch
    from paper_2408_11500_b200 import binding as B
    shapes = [(3, 1, 256, 1024, True, "silu", "bf16"), (5000, 8, 32, 64, True, "gelu", "bf16"), (300, 1, 602, 130, False, "relu", "fp32"), (2708, 1, 1433, 16, False, "none", "fp32"),
              (20_000, 1, 128, 256, False, "none", "bf16")]
    problems = [Problem(*s, residual=True) for s in shapes]
    sizes = [max(B.slicegcn_ffn_workspace_bytes(q.d, q.x), B.slicegcn_ffn_workspace_bytes(q.d, q.x, q.dout)) for q in problems]
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")

    def grads(q):
        g = [torch.empty((q.p, q.ins, q.outs), device="cuda", dtype=q.gt), torch.empty((q.p, q.outs), device="cuda")]
        return g + ([torch.empty_like(g[0]), torch.empty_like(g[1])] if q.gated else [None, None])

    def go(q, g):
        st = torch.cuda.current_stream().cuda_stream
        B.slicegcn_ffn_forward(q.d, q.x, q.r, q.out, q.status, ws, ws.numel(), st)
        B.slicegcn_ffn_backward(q.d, q.x, q.dout, q.dx, g[0], g[2], g[1], g[3], q.status, ws, ws.numel(), st)
    outs, want, graphs = [grads(q) for q in problems], [], []
    for q, g in zip(problems, outs):
        go(q, g)
        want.append([t.clone() for t in [q.out, q.dx] + g if t is not None])
    for q, g in zip(problems, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go(q, g)
        graphs.append(graph)
        for t in [q.out, q.dx] + g:
            if t is not None:
                t.fill_(7.0)
    for _ in range(2):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for q, g, w in zip(problems, outs, want):
        assert all(torch.equal(a, b) for a, b in zip([t for t in [q.out, q.dx] + g if t is not None], w)) and int(q.status) == 0


def test_two_streams_at_once():
    """Calls that overlap, each with a workspace of its own, give what they give alone."""
    import torch
    a, b = Problem(30_000, 1, 256, 512, True, "silu", "bf16", seed=1), Problem(3_000, 4, 100, 47, False, "gelu", "fp32", pad=1, residual=True, seed=2)
    want = [(q.forward().clone(), {k: v.clone() for k, v in q.backward().items()}) for q in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for q, s in zip((a, b), streams):
            with torch.cuda.stream(s):                       # its workspace and gradients come from that stream too
                got.append((q.forward(s.cuda_stream), q.backward(stream=s.cuda_stream)))
        torch.cuda.synchronize()
        for (out, g), (w, wg) in zip(got, want):
            assert torch.equal(out, w) and all(torch.equal(g[k], wg[k]) for k in wg)


@pytest.mark.parametrize("dtype,shape", [("bf16", (3000, 1, 256, 320)), ("bf16", (700, 2, 100, 47)), ("fp32", (900, 4, 32, 64)), ("fp32", (6, 1, 100, 50)), ("fp32", (200, 1, 3000, 40))])
def test_the_result_in_the_residual_s_place(dtype, shape):
    import torch
    q = Problem(*shape, True, "silu", dtype, residual=True)
    want = q.forward().clone()
    q.out = q.r
    q.d.out_ld = q.d.r_ld
    assert torch.equal(q.forward(), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_outputs_left_out(dtype):
    import torch
    for gated, act in ((True, "silu"), (False, "none")):
        q = Problem(1000, 2, 72, 130, gated, act, dtype)
        whole = {k: v.clone() for k, v in q.backward().items()}
        for want in (("dx",), ("dW",), ("db",), ("dW2",), ("db2", "dx"), ("dW", "db2"), ()):
            want = [k for k in want if k in whole]
            got = q.backward(want)
            assert set(got) == set(want) and all(torch.equal(got[k], whole[k]) for k in want)


def test_no_rows():
    import torch
    q = Problem(0, 2, 24, 16, True, "silu", "bf16")
    q.forward()
    g = q.backward()
    assert all(bool((g[k] == 0).all()) for k in ("dW", "dW2", "db", "db2"))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_neighbours_keep_their_values(dtype):
    """Columns beside a row, rows behind the last, and what follows dense gradients."""
    import torch
    from paper_2408_11500_b200 import binding as B
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    for n, p, ins, outs in ((130, 2, 40, 24), (257, 1, 70, 33), (5, 1, 64, 100), (3000, 8, 14, 23)):
        W, out, dx = (torch.randn(s, device="cuda").to(t) for s in ((p, ins, outs), (n + 3, p * outs + 9), (n + 3, p * ins + 9)))
        x, g = torch.randn((n, p * ins), device="cuda").to(t), torch.randn((n, p * outs), device="cuda").to(t)
        out.fill_(9.0), dx.fill_(9.0)
        dW, db = torch.full((p * ins * outs + 8,), 9.0, device="cuda", dtype=t), torch.full((p * outs + 8,), 9.0, device="cuda")
        d = B.make_ffn_desc(n, p, ins, outs, W, act=B.ACT_GELU, dtype=B.BF16 if dtype == "bf16" else B.F32, out_ld=out.stride(0), dx_ld=dx.stride(0))
        need = max(B.slicegcn_ffn_workspace_bytes(d, x), B.slicegcn_ffn_workspace_bytes(d, x, g))
        ws = torch.full((need + 256,), 9, device="cuda", dtype=torch.uint8)
        B.slicegcn_ffn_forward(d, x, None, out, None, ws, need)
        B.slicegcn_ffn_backward(d, x, g, dx, dW, None, db, None, None, ws, need)
        for m, cols in ((out, p * outs), (dx, p * ins)):
            assert bool((m[n:] == 9).all()) and bool((m[:, cols:] == 9).all()) and not bool((m[:n, :cols] == 9).all())
        assert bool((dW[-8:] == 9).all()) and bool((db[-8:] == 9).all()) and bool((ws[need:] == 9).all())


def test_offsets_past_32_bits():
    """Matrices of more than 2^32 bytes and 2^31 elements; the last rows are compared."""
    import torch
    from paper_2408_11500_b200 import binding as B
    n, ins, outs = 1_100_003, 256, 2048
    g = torch.Generator("cuda").manual_seed(0)
    x = torch.randn((n, ins), generator=g, device="cuda", dtype=torch.bfloat16)
    W, W2 = (torch.randn((1, ins, outs), generator=g, device="cuda").div_(16).to(torch.bfloat16) for _ in range(2))
    out = torch.empty((n, outs), device="cuda", dtype=torch.bfloat16)
    dx, dW, dW2 = torch.empty_like(x), torch.empty_like(W), torch.empty_like(W)
    d = B.make_ffn_desc(n, 1, ins, outs, W, W2, act=B.ACT_SILU, dtype=B.BF16)
    need = B.slicegcn_ffn_workspace_bytes(d, x, out)
    ws, status = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.slicegcn_ffn_forward(d, x, None, out, status, ws, need)
    part = slice(n - 300, n)

    def pre():
        a, c = (x[part].double() @ w[0].double() for w in (W, W2))
        return a, c, torch.sigmoid(a)
    a, c, q = pre()
    want = a * q * c
    assert bool(((out[part].double() - want).abs() <= 2.0 ** -7 * want.abs() + 1e-3).all())
    out.normal_(generator=g)
    out.mul_(1e-2)
    B.slicegcn_ffn_backward(d, x, out, dx, dW, dW2, None, None, status, ws, need)
    gr = out[part].double()
    da, dc = gr * c * (q + a * q * (1 - q)), gr * a * q
    want = da @ W[0].double().t() + dc @ W2[0].double().t()
    mag = da.abs() @ W[0].double().abs().t() + dc.abs() @ W2[0].double().abs().t()
    assert bool(((dx[part].double() - want).abs() <= 2.0 ** -7 * mag).all()) and int(status) == 0
    total = torch.zeros((ins, outs), device="cuda", dtype=torch.float64)
    for s in range(0, n, 100_000):
        part = slice(s, min(n, s + 100_000))
        a, c, q = pre()
        total += x[part].double().t() @ (out[part].double() * a * q)
    # roundings of dc and of the result, half a step each; the rows' products have random signs
    assert float((dW2[0].double() - total).norm() / total.norm()) <= 2 * 2.0 ** -8


@pytest.mark.parametrize("types", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")], ids=str)
@pytest.mark.parametrize("shape", [(3001, 1, 300, 132), (2500, 2, 1000, 76), (700, 1, 64, 40)], ids=str)
def test_neighbours_of_aligned_rows_keep_their_values(shape, types):
    """The same where rows start on 16 bytes, widths do not end there, and results leave by tensor copies."""
    import torch
    from paper_2408_11500_b200 import binding as B
    n, p, ins, outs = shape
    t, gt = (torch.bfloat16 if k == "bf16" else torch.float32 for k in types)
    code = lambda k: B.BF16 if k == torch.bfloat16 else B.F32   # noqa: E731
    wide = lambda cols: (cols + 7) // 8 * 8 + 16   # noqa: E731
    W, W2 = (torch.randn((p, ins, outs), device="cuda").to(t) for _ in range(2))
    x, g = torch.randn((n, wide(p * ins)), device="cuda").to(t), torch.randn((n, wide(p * outs)), device="cuda").to(gt)
    x[:, p * ins:], g[:, p * outs:] = float("nan"), float("nan")
    out, dx = torch.full((n + 2, wide(p * outs)), 9.0, device="cuda", dtype=t), torch.full((n + 2, wide(p * ins)), 9.0, device="cuda", dtype=gt)
    r = torch.full((n, wide(p * outs)), float("nan"), device="cuda", dtype=t)
    r[:, :p * outs] = 1.0
    d = B.make_ffn_desc(n, p, ins, outs, W, W2, act=B.ACT_SILU, dtype=code(t), grad_dtype=code(gt), x_ld=x.stride(0), r_ld=r.stride(0), out_ld=out.stride(0),
                        dout_ld=g.stride(0), dx_ld=dx.stride(0))
    need = max(B.slicegcn_ffn_workspace_bytes(d, x), B.slicegcn_ffn_workspace_bytes(d, x, g))
    ws = torch.full((need + 256,), 9, device="cuda", dtype=torch.uint8)
    dW, dW2 = (torch.empty((p, ins, outs), device="cuda", dtype=gt) for _ in range(2))
    B.slicegcn_ffn_forward(d, x, r, out, None, ws, need)
    B.slicegcn_ffn_backward(d, x, g, dx, dW, dW2, None, None, None, ws, need)
    for m, cols in ((out, p * outs), (dx, p * ins)):
        assert bool((m[n:] == 9).all()) and bool((m[:, cols:] == 9).all()) and bool(torch.isfinite(m[:n, :cols]).all())
    assert bool(torch.isfinite(dW).all()) and bool(torch.isfinite(dW2).all()) and bool((ws[need:] == 9).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_with_infinities_and_nan_stay_in_their_rows(dtype):
    import torch
    for n in (7, 600):
        q = Problem(n, 1, 200, 72, True, "silu", dtype)
        clean = q.forward().clone()
        q.x[2, 5], q.x[4, 7] = float("inf"), float("nan")
        out = q.forward()
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        keep[2] = keep[4] = False
        assert torch.equal(out[keep], clean[keep]) and bool(torch.isnan(out[4]).all()) and not bool(torch.isfinite(out[2]).any())


def test_large_and_tiny_fp32_numbers():
    """Magnitudes up to fp32's range and down to its least normal numbers in separate rows."""
    import torch
    from paper_2408_11500_b200 import binding as B
    n, ins, outs = 64, 96, 40
    x = torch.randn((n, ins), device="cuda")
    scale = torch.logspace(-30, 34, n, device="cuda", dtype=torch.float64)
    x = (x.double() * scale[:, None]).float()
    W = torch.randn((1, ins, outs), device="cuda")
    out, ws_d = torch.empty((n, outs), device="cuda"), B.make_ffn_desc(n, 1, ins, outs, W)
    need = B.slicegcn_ffn_workspace_bytes(ws_d, x)
    B.slicegcn_ffn_forward(ws_d, x, None, out, None, torch.empty(need, dtype=torch.uint8, device="cuda"), need)
    want, mag = x.double() @ W[0].double(), x.double().abs() @ W[0].double().abs()
    assert bool(((out.double() - want).abs() <= 2.0 ** -20 * mag).all())
