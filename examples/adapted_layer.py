"""A training step of low-rank adapters beside frozen weights in 4 bits, up to the loss over a
vocabulary, for the rows of several requests at once.

    python examples/adapted_layer.py [--tokens T] [--inputs K] [--words N] [--requests R] [--steps S]

    h1 = x             y1 = norm(h1) w1         z = y1 W^T + s (y1 A_a^T) B_a     (adapter a of each row)
    h2 = h1 + z        y2 = norm(h2) w2         loss = cross entropy of y2 V^T    (V: the vocabulary)

W (inputs x inputs) and V (words x inputs) are kept in 4 bits, both ways, and do not change; A, B, w1
and w2 are trained.  Prints the loss.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2106_06601_amd as costa  # noqa: E402

EPS = 1e-5


def kept(w):
    """w in 4 bits, and its transpose: for the product and for its input's gradient."""
    q, qt = costa.MxMatrix.empty(4, *w.shape), costa.MxMatrix.empty(4, *w.shape[::-1])
    costa.costa_mx_quantize(1.0, w, q, qt)
    return q, qt


class Model:
    def __init__(self, inputs, words, requests, rank, dtype, gen):
        new = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
        self.w, self.wt = kept(new(inputs, inputs) / inputs**0.5)
        self.v, self.vt = kept(new(words, inputs) / inputs**0.5)
        self.A = (new(requests, rank, inputs) / inputs**0.5).to(dtype)
        self.B = (0.1 * new(requests, rank, inputs)).to(dtype)
        self.w1, self.w2 = torch.ones(inputs, device="cuda"), torch.ones(inputs, device="cuda")
        self.adapters = costa.MxAdapters(self.A, self.B, scales=torch.full((requests,), 0.5, device="cuda"))

    def step(self, x, index, target):
        """(mean loss, gradients of x, A, B, w1 and w2); index: each row's adapter, target: its word."""
        like, floats = (lambda: torch.empty_like(x)), (lambda *s: torch.empty(*s, device="cuda"))  # noqa: E731
        m, rank = x.shape[0], self.adapters.rank
        y1, z, h2, y2, s1, s2 = like(), like(), like(), like(), floats(m), floats(m)
        V, loss, lse = floats(m, rank), floats(m), floats(m)
        costa.costa_mx_norm(EPS, x, self.w1, Y=y1, rstd=s1)
        costa.costa_mx_product_adapted(1.0, y1, self.w, self.adapters, index, 0.0, z, V=V)
        costa.costa_mx_norm(EPS, z, self.w2, R=x, H=h2, Y=y2, rstd=s2)
        costa.costa_mx_loss(1.0, y2, self.v, target, loss, lse)
        # back
        dloss = torch.full((m,), 1.0 / m, device="cuda")
        dy, dh, dx, dV = like(), like(), like(), floats(m, rank)
        dw1, dw2, dA, dB = torch.empty_like(self.w1), torch.empty_like(self.w2), floats(*self.A.shape), floats(*self.B.shape)
        costa.costa_mx_loss_backward(1.0, y2, self.v, target, lse, dloss, WT=self.vt, dX=dy)
        costa.costa_mx_norm_backward(dy, h2, self.w2, s2, dh, dW=dw2)  # of h2: of z and of x
        costa.costa_mx_adapter_gradient(self.adapters, index, V, dh, 0.0, dB)
        costa.costa_mx_product_adapted(1.0, dh, self.wt, self.adapters.turned(), index, 0.0, dy, V=dV)
        costa.costa_mx_adapter_gradient(self.adapters, index, dV, y1, 0.0, dA)
        costa.costa_mx_norm_backward(dy, x, self.w1, s1, dx, dH=dh, dW=dw1)
        return loss.mean(), {"x": dx, "A": dA, "B": dB, "w1": dw1, "w2": dw2}


def train(tokens=512, inputs=256, words=1000, requests=4, rank=16, steps=8, rate=4.0, dtype=torch.bfloat16, seed=0):
    """Runs the steps on one batch; returns the losses."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    model = Model(inputs, words, requests, rank, dtype, gen)
    x = torch.randn(tokens, inputs, generator=gen, device="cuda").to(dtype)
    index = torch.randint(-1, requests, (tokens,), generator=gen, device="cuda").to(torch.int32)
    target = torch.randint(0, words, (tokens,), generator=gen, device="cuda")
    losses = []
    for _ in range(steps):
        loss, grads = model.step(x, index, target)
        losses.append(float(loss))
        for name in ("A", "B", "w1", "w2"):
            p = getattr(model, name)
            p.sub_(rate * grads[name].to(p.dtype))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--inputs", type=int, default=256)
    ap.add_argument("--words", type=int, default=1000)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    for k, loss in enumerate(train(a.tokens, a.inputs, a.words, a.requests, steps=a.steps)):
        print(f"step {k}: loss {loss:.4f}")
