"""A residual network on the active rows, trained on labels: a class per active vertex.

``LabelHead`` takes the rows that a mask picks from a batch of bodies through residual
blocks to a class each, of any number of classes, and trains on labels; a vertex without
a label (any number outside of the classes) is left out:

    h0 = gather(x) + scale * E[v]          shc_gather_rows, shc_embed_rows
    y0 = layer_norm(h0) gamma + beta       shc_layer_norm
    y  = y + gelu(y W1 + b1) W2 + b2       shc_linear, twice a block
    loss, dy, dT                           shc_linear_cross_entropy_step: classes' rows T
    gradients of the blocks                shc_linear_backward, the residual's added by dy
    dh0, dgamma, dbeta, dE                 shc_layer_norm_backward, shc_embed_rows_backward
    clipping                               shc_grad_norm, shc_clip_grads

All arithmetic of the forward and backward pass but the sum of a block's two gradients
runs in the library's kernels; PyTorch holds the memory and applies the plain gradient
step to the fp32 parameters.  Buffers are made once, for all B * V rows active.

``python -m paper_2608_09388_amd.label_head`` trains one on synthetic bodies whose labels
follow a fixed random network and prints the mean loss.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as shc

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


class LabelHead:
    """B bodies of V vertices, C channels, `hidden` of a block, `classes`, any numbers (C as
    the gather takes it)."""

    def __init__(self, B: int, V: int, C: int, hidden: int, classes: int, blocks: int = 2,
                 max_norm: float = 1.0, dtype: str = "bf16", seed: int = 0, device: str = "cuda"):
        self.B, self.V, self.C, self.classes, self.blocks = B, V, C, classes, blocks
        self.max_norm = max_norm
        dt, f32 = DTYPE[dtype], torch.float32
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def new(*shape, dtype=dt):
            return torch.empty(shape, dtype=dtype, device=device)

        def randn(*shape, scale):
            return torch.randn(shape, generator=g, dtype=f32, device=device) * scale

        # parameters in fp32; the layers read their matrices in the compute dtype
        self.params = dict(E=randn(V, C, scale=C ** -0.5), gamma=torch.ones(C, device=device),
                           beta=torch.zeros(C, device=device),
                           T=randn(classes, C, scale=C ** -0.5))
        for k in range(blocks):
            self.params[f"W1.{k}"] = randn(C, hidden, scale=C ** -0.5)
            self.params[f"b1.{k}"] = torch.zeros(hidden, device=device)
            self.params[f"W2.{k}"] = randn(hidden, C, scale=0.5 * hidden ** -0.5)
            self.params[f"b2.{k}"] = torch.zeros(C, device=device)
        matrix = {k for k, v in self.params.items() if v.dim() == 2}
        self.weights = {k: new(*self.params[k].shape) for k in matrix}
        # gradients of the layers' matrices come in the compute dtype, of E in fp32
        self.grads = {k: torch.zeros_like(v, dtype=dt if k in matrix and k != "E" else f32)
                      for k, v in self.params.items()}
        self._refresh()
        self.scale = math.sqrt(C)
        rows = B * V
        self.coords = new(rows, 2, dtype=torch.int32)
        self.inv, self.row_ptr = new(rows, dtype=torch.int32), new(B + 1, dtype=torch.int32)
        self.count = new(1, dtype=torch.int32)
        self.compact_ws = new(max(16, shc.compact_mask_workspace(B, V)), dtype=torch.uint8)
        self.S, self.h0, self.dh0 = new(rows, C), new(rows, C), new(rows, C)
        self.y = [new(rows, C) for _ in range(blocks + 1)]
        self.pre = [new(rows, hidden) for _ in range(blocks)]
        self.act = [new(rows, hidden) for _ in range(blocks)]
        self.dy, self.dz, self.db = new(rows, C), new(rows, hidden), new(rows, C)
        self.mean, self.rstd, self.loss, self.weight = (new(rows, dtype=f32) for _ in range(4))
        self.norm = new(1, dtype=f32)
        code = shc.SHC_BF16 if dtype == "bf16" else shc.SHC_F32
        self.ws = new(max(
            shc.linear_workspace(rows, C, hidden, code), shc.linear_workspace(rows, hidden, C, code),
            shc.linear_backward_workspace(rows, C, hidden, code, shc.SHC_ACT_GELU),
            shc.linear_backward_workspace(rows, hidden, C, code),
            shc.linear_cross_entropy_workspace(rows, C, classes, code),
            shc.layer_norm_backward_workspace(rows, C),
            shc.embed_rows_backward_workspace(rows, V, C),
            shc.grad_norm_workspace(self.grads.values())), dtype=torch.uint8)

    def _refresh(self):
        for k, w in self.weights.items():
            w.copy_(self.params[k])

    def compact(self, mask: torch.Tensor) -> int:
        """The active rows of mask [B*V]: their number."""
        return shc.compact_mask(mask, self.B, self.V, self.coords, self.inv, self.row_ptr,
                                self.count, self.compact_ws)

    def forward(self, x: torch.Tensor, n: int) -> torch.Tensor:
        """The last block's rows [n][C] of the active rows of x [B*V][C]."""
        if n == 0:
            return self.y[-1][:0]
        p, w = self.params, self.weights
        shc.gather_rows(x, self.coords, n, self.B, self.V, self.S)
        shc.embed_rows(w["E"], self.coords[:n, 1], self.h0, self.scale, self.S)
        shc.layer_norm(self.h0[:n], p["gamma"], p["beta"], self.y[0], self.mean, self.rstd)
        for k in range(self.blocks):
            shc.linear(self.y[k][:n], w[f"W1.{k}"], p[f"b1.{k}"], self.act[k], shc.SHC_ACT_GELU,
                       pre=self.pre[k], ws=self.ws)
            shc.linear(self.act[k][:n], w[f"W2.{k}"], p[f"b2.{k}"], self.y[k + 1],
                       residual=self.y[k], ws=self.ws)
        return self.y[-1][:n]

    def losses(self, labels: torch.Tensor, n: int) -> torch.Tensor:
        """Loss [n] of the rows that forward left, without gradients."""
        return shc.linear_cross_entropy(self.y[-1][:n], self.weights["T"], labels, loss=self.loss[:n],
                                        ws=self.ws)

    def backward(self, labels: torch.Tensor, n: int) -> torch.Tensor:
        """Loss [n] against labels [n], and self.grads of the mean over the labelled rows,
        clipped to max_norm together."""
        p, w, g = self.params, self.weights, self.grads
        self.there = ((labels >= 0) & (labels < self.classes)).sum().clamp_(min=1)
        if n == 0:
            for t in (*g.values(), self.norm):
                t.zero_()
            return self.loss[:0]
        self.weight[:n] = 1.0 / self.there
        shc.linear_cross_entropy_step(self.y[-1][:n], w["T"], labels, self.weight, None, self.loss,
                                      self.dy, g["T"], ws=self.ws)
        for k in reversed(range(self.blocks)):
            shc.linear_backward(self.dy[:n], self.act[k], w[f"W2.{k}"], None, self.dz, g[f"W2.{k}"],
                                g[f"b2.{k}"], ws=self.ws)
            shc.linear_backward(self.dz[:n], self.y[k], w[f"W1.{k}"], self.pre[k], self.db,
                                g[f"W1.{k}"], g[f"b1.{k}"], shc.SHC_ACT_GELU, ws=self.ws)
            self.dy[:n].add_(self.db[:n])
        shc.layer_norm_backward(self.dy[:n], self.h0, p["gamma"], self.mean, self.rstd, self.dh0,
                                g["gamma"], g["beta"], ws=self.ws)
        shc.embed_rows_backward(self.dh0, self.coords[:n, 1], g["E"], self.scale, ws=self.ws)
        shc.grad_norm(g.values(), self.norm, ws=self.ws)
        shc.clip_grads(g.values(), self.norm, self.max_norm)
        return self.loss[:n]

    def mean_loss(self, loss: torch.Tensor) -> torch.Tensor:
        """The mean that the last backward's gradients are of, from its losses: over the rows
        with a label (0 without one)."""
        return loss.sum() / self.there

    def update(self, lr: float):
        for k, v in self.params.items():
            v.sub_(self.grads[k], alpha=lr)
        self._refresh()

    def step(self, x, mask, labels, lr: float) -> torch.Tensor:
        """One training step; labels(coords [n][2]) gives the active rows' labels [n].
        Returns the loss of every active row (0 without a label)."""
        n = self.compact(mask)
        self.forward(x, n)
        loss = self.backward(labels(self.coords[:n]), n)
        self.update(lr)
        return loss


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--bodies", type=int, default=64)
    ap.add_argument("--vertices", type=int, default=655)
    ap.add_argument("--channels", type=int, default=128)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--classes", type=int, default=655)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--dtype", choices=sorted(DTYPE), default="bf16")
    a = ap.parse_args()
    B, V = a.bodies, a.vertices
    head = LabelHead(B, V, a.channels, a.hidden, a.classes, a.blocks, dtype=a.dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    # a vertex has the same class in every body; a tenth of the vertices have none
    table = torch.randint(0, a.classes, (V,), generator=g, device="cuda")
    table[torch.rand(V, generator=g, device="cuda") < 0.1] = -1

    def labels(coords):
        return table[coords[:, 1].long()]

    for s in range(a.steps):
        x = torch.randn((B * V, a.channels), generator=g, device="cuda").to(DTYPE[a.dtype])
        mask = (torch.rand(B * V, generator=g, device="cuda") < 0.1).to(torch.uint8)
        loss = head.step(x, mask, labels, a.lr)
        if s % 10 == 0 or s == a.steps - 1:
            print(f"step {s}: {loss.numel()} rows, mean loss {float(head.mean_loss(loss)):.4f}, "
                  f"gradient norm {float(head.norm):.4f}", flush=True)


if __name__ == "__main__":
    main()
