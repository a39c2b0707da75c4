"""Graph classification by a stack of residual layers, trained with AdamW.

The batch of examples/graph_classification.py; a stream s carries the features from layer to layer.

    s = embedding(types)                     embedding_fwd
    per layer:  y, s = norm(b + s)           rms_norm_fwd, residual = s; the first layer has no b yet
                b = relu(mean over neighbours of y, times W)        Hag.aggregate_fwd
    y = norm(b + s), p = mean over a graph   rms_norm_fwd, graph_pool_fwd
    logits = p @ W2, cross entropy

Backwards each norm's gradient meets the one that arrives along the stream (rms_norm_bwd, grad_total).  Then grad_norm and
one adamw_step over all parameters: clipping included, no weight decay on gains, states in 32 or 8 bits (those rounded by
chance, so that they follow gradients that shrink).  With bf16 layers
the parameters stay in fp32 and the step writes the bf16 copies that the next pass reads.

    python examples/residual_adamw.py [--graphs 400] [--layers 3] [--steps 30] [--dtype f32|bf16] [--bits 32|8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path[:0] = [ROOT, os.path.join(ROOT, "examples")]
import paper_1906_03707_b200 as hb  # noqa: E402
from graph_classification import CLASSES, TYPES, Batch  # noqa: E402


class Model:
    def __init__(self, width: int = 64, layers: int = 3, dtype=torch.float32, bits: int = 32, seed: int = 1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape, scale: scale * torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
        self.layers = layers
        self.table = normal(TYPES, width, scale=1.0)
        self.w = [normal(width, width, scale=(2 / width) ** 0.5) for _ in range(layers)]
        self.gain = [torch.ones(width, device="cuda") for _ in range(layers + 1)]
        self.w2 = normal(width, CLASSES, scale=width ** -0.5)
        self.decay = [0.0] + [0.01] * layers + [0.0] * (layers + 1) + [0.01]
        # what the passes read: the parameters, or their bf16 copies
        self.copies = None if dtype is torch.float32 else [p.to(dtype) for p in self.parameters()]
        self.state = hb.adamw_state(self.parameters(), bits)
        self.steps, self.seed = 0, seed

    def parameters(self):
        return [self.table, *self.w, *self.gain, self.w2]

    def loss_and_gradients(self, batch: Batch):
        """The loss and the gradients in the order of ``parameters``."""
        read = self.copies or self.parameters()
        n = self.layers
        table, w, gain, w2 = read[0], read[1:1 + n], read[1 + n:2 + 2 * n], read[-1]
        y, stream, rstd = hb.rms_norm_fwd(hb.embedding_fwd(batch.types, table), gain[0])
        kept = []                                               # of each layer: stream, rstd, aggregate, branch
        for k in range(n):
            a = batch.hag.aggregate_fwd(y, reduce="mean")
            b = (a @ w[k]).clamp_(min=0)
            kept.append((stream, rstd, a, b))
            y, stream, rstd = hb.rms_norm_fwd(b, gain[k + 1], residual=stream)
        p = hb.graph_pool_fwd(batch.seg_ptr, y, reduce="mean")
        logits = (p @ w2).float()
        loss = torch.nn.functional.cross_entropy(logits, batch.labels)

        g = torch.softmax(logits, 1)
        g[torch.arange(g.shape[0], device=g.device), batch.labels] -= 1
        g = (g / g.shape[0]).to(p.dtype)
        grad_w, grad_gain, grad_w2 = [None] * n, [None] * (n + 1), p.t() @ g
        grad_y = hb.graph_pool_bwd(batch.seg_ptr, g @ w2.t(), batch.n, reduce="mean")
        along = None
        for k in reversed(range(n)):
            grad_b, along, grad_gain[k + 1] = hb.rms_norm_bwd(grad_y, stream, rstd, gain[k + 1], grad_total=along)
            stream, rstd, a, b = kept[k]
            grad_z = grad_b * (b > 0)
            grad_w[k] = a.t() @ grad_z
            grad_y = batch.hag.aggregate_bwd(grad_z @ w[k].t(), reduce="mean")
        grad_s, _, grad_gain[0] = hb.rms_norm_bwd(grad_y, stream, rstd, gain[0], grad_total=along)
        return loss, [hb.embedding_bwd(batch.types, grad_s, TYPES), *grad_w, *grad_gain, grad_w2]

    def step(self, batch: Batch, rate: float = 1e-2, max_norm: float = 1.0):
        loss, grads = self.loss_and_gradients(batch)
        norm = hb.grad_norm(grads)
        self.steps += 1
        hb.adamw_step(self.parameters(), grads, self.state, self.steps, lr=rate, weight_decay=self.decay, total_norm=norm, max_norm=max_norm,
                      copies=self.copies, seed=self.seed)
        return loss, norm


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--graphs", type=int, default=400)
    ap.add_argument("--layers", type=int, default=3)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args()
    batch = Batch(a.graphs)
    model = Model(layers=a.layers, dtype=torch.float32 if a.dtype == "f32" else torch.bfloat16, bits=a.bits)
    for k in range(a.steps):
        loss, norm = model.step(batch)
        if k % 5 == 0 or k == a.steps - 1:
            print(f"step {k:3d}  loss {float(loss):.4f}  gradient norm {float(norm):.4f}")


if __name__ == "__main__":
    main()
