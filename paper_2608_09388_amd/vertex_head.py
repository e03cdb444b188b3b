"""A trained head on the active rows: per-vertex classes distilled from a teacher.

``VertexHead`` classifies every active vertex of a batch of bodies and learns
from a teacher's top logits at those vertices:

    h = gather(x) + scale * E[v]        shc_gather_rows, shc_embed_rows: a learned
                                        row per vertex, looked up by the vertex
                                        column of the coordinate list
    y = layer_norm(h) gamma + beta      shc_layer_norm
    z = y W + b                         shc_sparse_linear
    loss, dz                            shc_distill_top_step
    dy, dW, db                          shc_sparse_linear_backward
    dh, dgamma, dbeta                   shc_layer_norm_backward
    dE                                  shc_embed_rows_backward, by sorted ids

All arithmetic of the forward and backward pass runs in the library's kernels;
PyTorch holds the memory, and applies the plain gradient step to the fp32
parameters.  Buffers are made once, for all B * V rows active.

``python -m paper_2608_09388_amd.vertex_head`` trains one on synthetic bodies
with a fixed random teacher and prints the mean loss.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as shc

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


class VertexHead:
    """B bodies of V vertices, C channels, `classes` of a multiple of 16 up to 256."""

    def __init__(self, B: int, V: int, C: int, classes: int, top: int = 8,
                 temperature: float = 2.0, dtype: str = "bf16", seed: int = 0,
                 device: str = "cuda"):
        self.B, self.V, self.C, self.classes, self.T = B, V, C, classes, temperature
        self.top = top  # entries a row that it asks of its teacher
        dt, f32 = DTYPE[dtype], torch.float32
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def new(*shape, dtype=dt):
            return torch.empty(shape, dtype=dtype, device=device)

        def randn(*shape):
            return torch.randn(shape, generator=g, dtype=f32, device=device)

        # parameters in fp32; the layers read E and W in the compute dtype
        self.params = dict(E=randn(V, C) / math.sqrt(C), W=randn(C, classes) / math.sqrt(C),
                           b=torch.zeros(classes, device=device),
                           gamma=torch.ones(C, device=device), beta=torch.zeros(C, device=device))
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.E, self.W = new(V, C), new(C, classes)
        self._refresh()
        self.scale = math.sqrt(C)
        rows = B * V
        self.coords = new(rows, 2, dtype=torch.int32)
        self.inv, self.row_ptr = new(rows, dtype=torch.int32), new(B + 1, dtype=torch.int32)
        self.count = new(1, dtype=torch.int32)
        self.compact_ws = new(max(16, shc.compact_mask_workspace(B, V)), dtype=torch.uint8)
        self.S, self.h, self.y, self.dy, self.dh = (new(rows, C) for _ in range(5))
        self.z, self.dz = new(rows, classes), new(rows, classes)
        self.mean, self.rstd, self.loss, self.weight = (new(rows, dtype=f32) for _ in range(4))
        self.linear_ws = new(max(16, shc.sparse_linear_backward_workspace(
            rows, C, classes, shc.SHC_BF16 if dtype == "bf16" else shc.SHC_F32)),
            dtype=torch.uint8)
        self.norm_ws = new(shc.layer_norm_backward_workspace(rows, C), dtype=torch.uint8)
        self.embed_ws = new(shc.embed_rows_backward_workspace(rows, V, C), dtype=torch.uint8)

    def _refresh(self):
        self.E.copy_(self.params["E"])
        self.W.copy_(self.params["W"])

    def compact(self, mask: torch.Tensor) -> int:
        """The active rows of mask [B*V]: their number."""
        return shc.compact_mask(mask, self.B, self.V, self.coords, self.inv, self.row_ptr,
                                self.count, self.compact_ws)

    def forward(self, x: torch.Tensor, n: int) -> torch.Tensor:
        """Logits [n][classes] of the active rows of x [B*V][C]."""
        if n == 0:
            return self.z[:0]
        p = self.params
        shc.gather_rows(x, self.coords, n, self.B, self.V, self.S)
        shc.embed_rows(self.E, self.coords[:n, 1], self.h, self.scale, self.S)
        shc.layer_norm(self.h[:n], p["gamma"], p["beta"], self.y, self.mean, self.rstd)
        shc.sparse_linear(self.y, n, self.W, p["b"], self.z, shc.SHC_ACT_NONE)
        return self.z[:n]

    def backward(self, top_ids: torch.Tensor, top_logits: torch.Tensor, n: int) -> torch.Tensor:
        """Loss [n] against the teacher's entries [n][k], and self.grads of its mean."""
        if n == 0:
            for g in self.grads.values():
                g.zero_()
            return self.loss[:0]
        p, g = self.params, self.grads
        self.weight[:n] = 1.0 / n
        shc.distill_top_step(self.z[:n], top_ids, top_logits, self.weight, self.loss, self.dz,
                             self.T)
        shc.sparse_linear_backward(self.y, self.W, None, self.dz, n, self.dy, g["W"], g["b"],
                                   shc.SHC_ACT_NONE, self.linear_ws)
        shc.layer_norm_backward(self.dy[:n], self.h, p["gamma"], self.mean, self.rstd, self.dh,
                                g["gamma"], g["beta"], ws=self.norm_ws)
        shc.embed_rows_backward(self.dh, self.coords[:n, 1], g["E"], self.scale,
                                ws=self.embed_ws)
        return self.loss[:n]

    def update(self, lr: float):
        for k, v in self.params.items():
            v.sub_(self.grads[k], alpha=lr)
        self._refresh()

    def step(self, x, mask, teacher, lr: float) -> torch.Tensor:
        """One training step; teacher(coords [n][2]) gives (top_ids, top_logits).
        Returns the loss of every active row."""
        n = self.compact(mask)
        self.forward(x, n)
        loss = self.backward(*teacher(self.coords[:n]), n)
        self.update(lr)
        return loss


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--bodies", type=int, default=64)
    ap.add_argument("--vertices", type=int, default=655)
    ap.add_argument("--channels", type=int, default=128)
    ap.add_argument("--classes", type=int, default=48)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--dtype", choices=sorted(DTYPE), default="bf16")
    a = ap.parse_args()
    B, V = a.bodies, a.vertices
    head = VertexHead(B, V, a.channels, a.classes, dtype=a.dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    # the teacher prefers the same classes at a vertex in every body
    table = 3.0 * torch.randn((V, a.classes), generator=g, device="cuda")
    top_logits, top_ids = table.topk(head.top, dim=1)
    top_ids = top_ids.to(torch.int32)

    def teacher(coords):
        v = coords[:, 1].long()
        return top_ids[v], top_logits[v]

    for s in range(a.steps):
        x = torch.randn((B * V, a.channels), generator=g, device="cuda").to(DTYPE[a.dtype])
        mask = (torch.rand(B * V, generator=g, device="cuda") < 0.1).to(torch.uint8)
        loss = head.step(x, mask, teacher, a.lr)
        if s % 10 == 0 or s == a.steps - 1:
            print(f"step {s}: {loss.numel()} rows, mean loss {float(loss.mean()):.4f}", flush=True)


if __name__ == "__main__":
    main()
