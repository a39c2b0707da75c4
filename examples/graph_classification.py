"""Graph classification with every operator of the library in one training step.

A batch of dense random graphs; every node has one of a few types, and the mix of types tells the class of its graph.

    h = embedding(types)            embedding_fwd       grad of the table:  embedding_bwd
    a = mean over neighbours of h   Hag.aggregate_fwd   grad of h:          Hag.aggregate_bwd
    y = layer norm of a @ W1        layer_norm_fwd      grads of W1, w, b:  layer_norm_bwd
    p = mean over a graph, relu(y)  graph_pool_fwd      grad of relu(y):    graph_pool_bwd
    logits = p @ W2, cross entropy

then clip_grad_norm over all gradients, in place, and one step of plain gradient descent.  The two matrix products, the
relu and the loss are torch's.

    python examples/graph_classification.py [--graphs 400] [--steps 30] [--dtype f32|bf16]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1906_03707_b200 as hb  # noqa: E402
from paper_1906_03707_b200 import synth  # noqa: E402

TYPES, CLASSES = 20, 3


class Batch:
    """Graphs side by side: their HAG on the device, the nodes' types, the graphs' rows and classes."""

    def __init__(self, n_graphs: int, seed: int = 0):
        w = synth.workload(4, scale=n_graphs / 5000)
        self.graph = w.graph
        self.n = w.graph.n
        self.hag = hb.Hag.build(w.graph.row_ptr, w.graph.col_idx, w.capacity).to_device(0)
        rng = np.random.default_rng(seed)
        self.seg_ptr = torch.arange(0, self.n + 1, 100, dtype=torch.int32, device="cuda")
        n_graphs = self.seg_ptr.numel() - 1
        labels = rng.integers(0, CLASSES, n_graphs)
        mix = rng.dirichlet(np.full(TYPES, 0.5), CLASSES)
        types = np.concatenate([rng.choice(TYPES, 100, p=mix[c]) for c in labels])
        types[::97] = -1                                        # nodes without a type: zero features, no gradient
        self.types = torch.from_numpy(types.astype(np.int32)).cuda()
        self.labels = torch.from_numpy(labels).cuda()


class Model:
    def __init__(self, width: int = 64, dtype=torch.float32, seed: int = 1):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale):
            return (scale * torch.randn(shape, generator=gen, device="cuda")).to(dtype)

        self.table = normal(TYPES, width, scale=1.0)
        self.w1 = normal(width, width, scale=width ** -0.5)
        self.gain = torch.ones(width, device="cuda", dtype=dtype)
        self.bias = torch.zeros(width, device="cuda", dtype=dtype)
        self.w2 = normal(width, CLASSES, scale=width ** -0.5)

    def parameters(self):
        return [self.table, self.w1, self.gain, self.bias, self.w2]

    def loss_and_gradients(self, batch: Batch):
        """The loss and the gradients in the order of ``parameters``."""
        h = hb.embedding_fwd(batch.types, self.table)
        a = batch.hag.aggregate_fwd(h, reduce="mean")
        y, mean, rstd = hb.layer_norm_fwd(z := a @ self.w1, self.gain, self.bias)
        r = y.clamp(min=0)
        p = hb.graph_pool_fwd(batch.seg_ptr, r, reduce="mean")
        logits = (p @ self.w2).float()
        loss = torch.nn.functional.cross_entropy(logits, batch.labels)

        g = torch.softmax(logits, 1)
        g[torch.arange(g.shape[0], device=g.device), batch.labels] -= 1
        g = (g / g.shape[0]).to(p.dtype)
        grad_w2 = p.t() @ g
        grad_r = hb.graph_pool_bwd(batch.seg_ptr, g @ self.w2.t(), batch.n, reduce="mean")
        grad_y = grad_r * (y > 0)
        grad_z, grad_gain, grad_bias = hb.layer_norm_bwd(grad_y, z, mean, rstd, self.gain, out=grad_y)
        grad_w1 = a.t() @ grad_z
        grad_h = batch.hag.aggregate_bwd(grad_z @ self.w1.t(), reduce="mean")
        grad_table = hb.embedding_bwd(batch.types, grad_h, TYPES)
        return loss, [grad_table, grad_w1, grad_gain, grad_bias, grad_w2]

    def step(self, batch: Batch, rate: float = 0.5, max_norm: float = 1.0):
        loss, grads = self.loss_and_gradients(batch)
        _, norm = hb.clip_grad_norm(grads, max_norm, out=grads)
        for p, g in zip(self.parameters(), grads):
            p.add_(g, alpha=-rate)
        return loss, norm


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--graphs", type=int, default=400)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args()
    batch = Batch(a.graphs)
    model = Model(dtype=torch.float32 if a.dtype == "f32" else torch.bfloat16)
    for k in range(a.steps):
        loss, norm = model.step(batch)
        if k % 5 == 0 or k == a.steps - 1:
            print(f"step {k:3d}  loss {float(loss):.4f}  gradient norm {float(norm):.4f}")


if __name__ == "__main__":
    main()
