"""A layer's training step on matrices that lie in blocks over P ranks, with its
weights kept in 4 bits and its activation kept in 8 bits for the backward pass.

    python examples/few_bit_layer.py [--tokens T] [--inputs K] [--outputs N] [--steps S]

The weights W (outputs x inputs) and the activation X (tokens x inputs) are
block-cyclic float32 matrices.  A step
  1. quantises W out of its blocks, both ways in one read: mx(W) for the forward
     product, mx(W^T) for the gradient of the input;
  2. quantises X^T out of its blocks to 8 bits (the checkpoint) and brings X itself
     together with a transform;
  3. forward Y = X W^T;  backward dX = dY W and dW = dY^T X from the 8-bit
     checkpoint, summed in 32 bits;
  4. updates the distributed W with a transform: W <- -rate dW + W.
Prints the loss |X W^T - target|^2 / 2, which falls.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2106_06601_amd as costa  # noqa: E402


class Dealt:
    """A float32 matrix in blocks over a grid of ranks, and its place in one piece."""

    def __init__(self, rows, cols, mb, nb, prow, pcol):
        self.layout = costa.Layout.block_cyclic(rows, cols, mb, nb, prow, pcol)
        self.whole = costa.Layout.general(rows, cols, [0, rows], [0, cols], [0], prow * pcol, "row")
        self.local = [torch.empty(self.layout.local_elems(r), device="cuda") for r in range(prow * pcol)]

    def put(self, x, alpha=1.0, beta=0.0):
        """self <- alpha x + beta self"""
        costa.costa_transform("f32", "N", alpha, beta, self.layout, self.local, self.whole,
                              [x] + [None] * (len(self.local) - 1))

    def get(self, x):
        costa.costa_transform("f32", "N", 1.0, 0.0, self.whole, [x] + [None] * (len(self.local) - 1), self.layout,
                              self.local)
        return x


def train(tokens=512, inputs=384, outputs=256, steps=8, rate=None, seed=0):
    """Runs the steps; returns the losses."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    new = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
    W, X = Dealt(outputs, inputs, 64, 32, 2, 2), Dealt(tokens, inputs, 128, 64, 2, 2)
    true = torch.randn(outputs, inputs, generator=gen, device="cuda") / inputs**0.5
    W.put(torch.zeros_like(true))
    wq, wqt = costa.MxMatrix.empty(4, outputs, inputs), costa.MxMatrix.empty(4, inputs, outputs)
    xt = costa.MxMatrix.empty(8, inputs, tokens)
    x, y, dx, dw = new(tokens, inputs), new(tokens, outputs), new(tokens, inputs), new(outputs, inputs)
    rate = rate or 1.0 / tokens
    losses = []
    for _ in range(steps):
        fresh = torch.randn(tokens, inputs, generator=gen, device="cuda")
        X.put(fresh)
        target = fresh @ true.t()
        costa.costa_mx_quantize_layout("f32", 1.0, W.layout, W.local, wq, wqt)
        costa.costa_mx_quantize_layout("f32", 1.0, X.layout, X.local, None, xt)
        costa.costa_mx_product_real(1.0, "N", X.get(x), wq, 0.0, y)
        dy = y - target
        losses.append(float(dy.square().sum()) / (2 * tokens))
        costa.costa_mx_product_real(1.0, "N", dy, wqt, 0.0, dx)  # (for the layer below)
        costa.costa_mx_product_real(1.0, "T", dy, xt, 0.0, dw)
        W.put(dw, -rate, 1.0)
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--inputs", type=int, default=384)
    ap.add_argument("--outputs", type=int, default=256)
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    for k, loss in enumerate(train(a.tokens, a.inputs, a.outputs, a.steps)):
        print(f"step {k}: loss {loss:.4f}")
