"""Training a deep sliced GCN whose nodes are given by ids: embedding lookup, sliced layers between norms with gated
residuals, a linear head, and clipping by the global gradient norm, on one GPU.

    python deep_epochs.py --workload citation --layers 8 --vocab 40009 --epochs 20

The features are `scale * table[ids]` (one learned vector per node, or per category with --vocab); layer l reads
u = N(x), and the residual stream becomes x + s * sigmoid(u) * N(layer(u)).  Everything but the head (one matrix product
and a softmax in torch) and the update itself runs in the library.  Prints one JSON line.
"""
from __future__ import annotations

import argparse
import json
import math

import numpy as np


class DeepSlicedGCN:
    """Parameters, activations and gradients of the model above; `step()` is one full-batch training step."""

    def __init__(self, g, ids, labels, vocab: int, hidden: int, num_slices: int, layers: int, classes: int, seed: int = 0,
                 residual_scale: float = 0.5, max_norm: float = 1.0):
        import torch
        from paper_2408_11500_b200 import binding as B
        self.torch, self.B, self.g = torch, B, g
        self.n, self.vocab, self.p, self.h_s, self.layers, self.classes = ids.numel(), vocab, num_slices, hidden // num_slices, layers, classes
        self.width = self.p * self.h_s
        self.scale, self.s, self.max_norm = math.sqrt(self.width), residual_scale, max_norm
        self.ids, self.labels = ids, labels.long()
        shapes = {"table": (vocab, self.width), "w_pre.0": (self.width,)}
        for layer in range(layers):
            shapes.update({f"W_agg.{layer}": (self.p, self.h_s, self.h_s), f"W_self.{layer}": (self.p, self.h_s, self.h_s),
                           f"b.{layer}": (self.p, self.h_s), f"w_post.{layer}": (self.width,), f"w_pre.{layer + 1}": (self.width,)})
        shapes.update({"Wc": (self.width, classes), "bc": (classes,)})
        self.params, self.grads, self.clipped = ({k: torch.zeros(s, device="cuda") for k, s in shapes.items()} for _ in range(3))
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        for k, v in self.params.items():
            if k.startswith("w_p"):
                v.fill_(1.0)
            elif k == "table":
                v.normal_(0.0, 1.0 / self.width, generator=gen)
            elif v.dim() > 1 and not k.startswith("b."):
                v.normal_(0.0, math.sqrt(2.0 / (v.shape[-2] + v.shape[-1])), generator=gen)

        def mat():
            return torch.empty((self.n, self.width), device="cuda")
        self.x = [mat() for _ in range(layers + 1)]          # residual stream
        self.u = [mat() for _ in range(layers + 1)]          # normalised: layer inputs, then the head's
        self.y = [mat() for _ in range(layers)]              # layer outputs
        self.dx, self.du, self.dy, self.dgate = mat(), mat(), mat(), mat()
        self.norm = torch.zeros(1, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        P = self.params
        self.embed = B.make_embed_desc(self.n, vocab, self.width, scale=self.scale)
        self.first_norm = B.make_residual_norm_desc(self.n, self.p, self.h_s, w_pre=P["w_pre.0"])
        self.norms = [B.make_residual_norm_desc(self.n, self.p, self.h_s, residual_scale=self.s, w_post=P[f"w_post.{i}"], w_pre=P[f"w_pre.{i + 1}"])
                      for i in range(layers)]
        starts = [i * self.h_s for i in range(self.p)]
        self.layer = [B.make_layer_desc(self.p, starts, self.h_s, self.width, self.width, self.h_s, self.width, B.F32, B.ORDER_AUTO,
                                        P[f"W_agg.{i}"], P[f"W_self.{i}"], P[f"b.{i}"]) for i in range(layers)]
        self.saved_bytes = B.slicegcn_layer_saved_bytes(g, self.layer[0])
        self.saved = [torch.empty(self.saved_bytes, dtype=torch.uint8, device="cuda") for _ in range(layers)]
        self.tensors = B.make_tensor_list(list(self.grads.values()), list(self.clipped.values()))
        self.ws_bytes = max(B.slicegcn_layer_workspace_bytes(g, self.layer[0]), B.slicegcn_embed_workspace_bytes(self.embed),
                            B.slicegcn_residual_norm_workspace_bytes(self.norms[0]), B.slicegcn_clip_workspace_bytes())
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device="cuda")   # the calls follow one another on one stream

    def forward(self):
        B, st = self.B, self.torch.cuda.current_stream().cuda_stream
        B.slicegcn_embed_forward(self.embed, self.ids, self.params["table"], self.x[0], self.status, st)
        B.slicegcn_residual_norm_forward(self.first_norm, self.x[0], None, None, None, self.u[0], st)
        for i in range(self.layers):
            B.slicegcn_layer_forward(self.g, self.layer[i], self.u[i], self.y[i], self.saved[i], self.saved_bytes, self.ws, self.ws_bytes, st)
            B.slicegcn_residual_norm_forward(self.norms[i], self.x[i], self.y[i], self.u[i], self.x[i + 1], self.u[i + 1], st)
        return self.u[-1] @ self.params["Wc"] + self.params["bc"]

    def backward(self, logits):
        """Gradients of the mean cross entropy; returns the loss."""
        torch, B, G = self.torch, self.B, self.grads
        st = torch.cuda.current_stream().cuda_stream
        log_p = torch.log_softmax(logits, 1)
        loss = -log_p.gather(1, self.labels[:, None]).mean()
        d = log_p.exp()
        d[torch.arange(self.n, device="cuda"), self.labels] -= 1.0
        d /= self.n
        torch.matmul(self.u[-1].t(), d, out=G["Wc"])
        torch.sum(d, 0, out=G["bc"])
        torch.matmul(d, self.params["Wc"].t(), out=self.du)
        dh = None
        for i in reversed(range(self.layers)):
            B.slicegcn_residual_norm_backward(self.norms[i], self.y[i], self.u[i], self.x[i + 1], dh, self.du, self.dx, self.dy, self.dgate,
                                              G[f"w_post.{i}"], None, G[f"w_pre.{i + 1}"], None, self.ws, self.ws_bytes, st)
            dh = self.dx
            B.slicegcn_layer_backward(self.g, self.layer[i], self.u[i], self.saved[i], self.dy, self.width, self.du, self.width, G[f"W_agg.{i}"],
                                      G[f"W_self.{i}"], G[f"b.{i}"], None, None, self.ws, self.ws_bytes, st)
            self.du += self.dgate                            # u is the layer's input and the gate
        B.slicegcn_residual_norm_backward(self.first_norm, None, None, self.x[0], dh, self.du, self.dx, None, None, None, None, G["w_pre.0"], None,
                                          self.ws, self.ws_bytes, st)
        B.slicegcn_embed_backward(self.embed, self.ids, self.dx, G["table"], self.status, self.ws, self.ws_bytes, st)
        return loss

    def clip(self):
        self.B.slicegcn_clip_grads(self.tensors, self.max_norm, self.norm, self.ws, self.ws_bytes, self.torch.cuda.current_stream().cuda_stream)

    def step(self, lr: float):
        loss = self.backward(self.forward())
        self.clip()
        self.torch._foreach_add_(list(self.params.values()), list(self.clipped.values()), alpha=-lr)
        return loss


def main() -> None:
    import torch
    from paper_2408_11500_b200 import binding as B, synth
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="citation", choices=sorted(synth.WORKLOADS))
    ap.add_argument("--fraction", type=float, default=1.0, help="scale the workload's nodes and edges")
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--vocab", type=int, default=0, help="categories (0: a vector of its own for every node)")
    ap.add_argument("--epochs", type=int, default=20)
    ap.add_argument("--warmup", type=int, default=3)
    ap.add_argument("--lr", type=float, default=0.5)
    args = ap.parse_args()
    w = dict(synth.WORKLOADS[args.workload])
    if args.fraction < 1.0:
        w["n"], w["m"] = max(int(w["n"] * args.fraction), 64), max(int(w["m"] * args.fraction), 64)
        if "max_degree" in w:
            w["max_degree"] = max(w["max_degree"] * args.fraction, 16)
    src, dst = synth.make_graph(w, 0)
    g = B.slicegcn_graph_create(w["n"], src, dst, B.SYMMETRIZE | B.ADD_SELF_LOOPS)
    rng = np.random.default_rng(0)
    vocab = args.vocab or w["n"]
    ids = rng.integers(0, vocab, w["n"]) if args.vocab else np.arange(w["n"])
    model = DeepSlicedGCN(g, torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(synth.uniform_labels(w["n"], w["classes"], 0)).cuda(),
                          vocab, w["hidden"], w["p"], args.layers, w["classes"])
    losses = [model.step(args.lr) for _ in range(args.warmup)]
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    t0.record()
    for _ in range(args.epochs):
        losses.append(model.step(args.lr))
    t1.record()
    torch.cuda.synchronize()
    ms = t0.elapsed_time(t1) / args.epochs
    print(json.dumps({"metric": "full-graph training throughput of a deep sliced GCN from ids", "unit": "epochs/s", "value": 1e3 / ms,
                      "ms_per_epoch": ms, "workload": args.workload, "nodes": w["n"], "layers": args.layers, "vocab": vocab,
                      "first_loss": float(losses[0]), "final_loss": float(losses[-1]), "gradient_norm": float(model.norm),
                      "bad_ids": int(model.status)}))
    B.slicegcn_graph_destroy(g)


if __name__ == "__main__":
    main()
