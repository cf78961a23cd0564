"""The operators around products together: a training step of adapters beside frozen 4-bit
weights up to the loss, against the chain rule in 64 bits, as calls and as a replayed graph; a
served step that goes through 8 bits."""
import os
import sys

import numpy as np
import pytest
import torch

import mx_formula as F

C = pytest.importorskip("paper_2106_06601_amd")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def wide(t):
    return t.detach().to(torch.float64).cpu().numpy()


def values(q):
    d, s = C.costa_mx_sizes(q.bits, q.rows, q.cols)
    return F.decode(q.data[:d].cpu().numpy().reshape(q.rows, -1), q.scales[:s].cpu().numpy().reshape(q.rows, -1), q.bits, q.cols)


def norm(h, w):
    s = 1 / np.sqrt((h * h).mean(1, keepdims=True) + float(np.float32(1e-5)))
    return h * s * w, s


def norm_back(dy, h, w, s):
    g, u = dy * w, h * s
    return s * (g - u * (g * u).mean(1, keepdims=True)), (dy * u).sum(0)


def chain(M, x, index, target):
    """Loss and gradients in 64 bits, with the weights as they are stored both ways."""
    x, A, B, w1, w2 = (wide(t) for t in (x, M.A, M.B, M.w1, M.w2))
    w, wt, v, vt = (values(q) for q in (M.w, M.wt, M.v, M.vt))
    m, s = len(x), 0.5
    y1, s1 = norm(x, w1)
    z, V = y1 @ w.T, np.zeros((m, A.shape[1]))
    own = [np.flatnonzero(index == a) for a in range(len(A))]
    for a, i in enumerate(own):
        V[i] = y1[i] @ A[a].T
        z[i] += s * V[i] @ B[a]
    h2 = x + z
    y2, s2 = norm(h2, w2)
    L = y2 @ v.T
    lse = np.log(np.exp(L - L.max(1, keepdims=True)).sum(1)) + L.max(1)
    G = np.exp(L - lse[:, None])
    loss = (lse - L[np.arange(m), target]).mean()
    G[np.arange(m), target] -= 1
    dh, dw2 = norm_back(G @ vt.T / m, h2, w2, s2)
    dy, dA, dB = dh @ wt.T, np.zeros_like(A), np.zeros_like(B)
    for a, i in enumerate(own):
        dV = dh[i] @ B[a].T
        dy[i] += s * dV @ A[a]
        dA[a], dB[a] = s * dV.T @ y1[i], s * V[i].T @ dh[i]
    dx, dw1 = norm_back(dy, x, w1, s1)
    return loss, {"x": dx + dh, "A": dA, "B": dB, "w1": dw1, "w2": dw2}


def off(got, want):
    return np.linalg.norm(wide(got) - want) / np.linalg.norm(want)


# Relative to the whole gradient: about eight results of the types' roundings follow one another, each
# off by at most half a step of its elements (2^-24, 2^-11, 2^-8) and independent of one
# another; their sums amplify none of them by more than the norms' two or three.
TOLERANCE = {torch.float32: 32 * 2.0**-24 * 8, torch.float16: 32 * 2.0**-11, torch.bfloat16: 32 * 2.0**-8}


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("tokens,inputs,words,requests,rank", [(5, 96, 70, 2, 4), (130, 200, 1003, 3, 20), (1100, 512, 2500, 4, 16)])
def test_a_training_step(dtype, tokens, inputs, words, requests, rank):
    import adapted_layer as E
    gen = torch.Generator(device="cuda")
    gen.manual_seed(tokens)
    M = E.Model(inputs, words, requests, rank, dtype, gen)
    x = torch.randn(tokens, inputs, generator=gen, device="cuda").to(dtype)
    index = torch.randint(-1, requests, (tokens,), generator=gen, device="cuda").to(torch.int32)
    target = torch.randint(0, words, (tokens,), generator=gen, device="cuda")
    loss, grads = M.step(x, index, target)
    want, wants = chain(M, x, index.cpu().numpy(), target.cpu().numpy())
    tol = TOLERANCE[dtype]
    assert abs(float(loss) - want) <= tol * want
    for name in wants:
        assert off(grads[name], wants[name]) <= tol, name


def test_a_step_in_a_graph():
    """Captured with torch's allocations of its own pool, replayed on other inputs, with eager steps between."""
    import adapted_layer as E
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    M = E.Model(256, 1000, 3, 16, torch.bfloat16, gen)
    x = torch.randn(300, 256, generator=gen, device="cuda").bfloat16()
    index = torch.randint(-1, 3, (300,), generator=gen, device="cuda").to(torch.int32)
    target = torch.randint(0, 1000, (300,), generator=gen, device="cuda")
    M.step(x, index, target)
    M.adapters.turned()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, kept = M.step(x, index, target)
    for _ in range(3):
        x.normal_(generator=gen)
        index.random_(-1, 3, generator=gen)
        target.random_(0, 1000, generator=gen)
        g.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in kept.items()}
        _, eager = M.step(x, index, target)
        torch.cuda.synchronize()
        for k in got:
            assert torch.equal(got[k], eager[k]), k


def test_the_example_runs():
    import adapted_layer as E
    losses = E.train(tokens=200, inputs=128, words=300, requests=3, steps=3)
    assert len(losses) == 3 and all(np.isfinite(losses))


@pytest.mark.parametrize("m", [1, 7, 64])
def test_a_served_step_through_8_bits(m):
    """norm with the residual to 8 bits, the product of 8 by 4 bits, adapters beside the next one: each call's
    operand is the one before's result."""
    k, n, count, rank = 512, 768, 3, 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, r, w1 = new(m, k).bfloat16(), new(m, k).bfloat16(), 1 + 0.1 * new(k)
    W, U = C.MxMatrix.empty(4, n, k), C.MxMatrix.empty(4, k, n)
    C.costa_mx_quantize(1.0, new(n, k) / k**0.5, W)
    C.costa_mx_quantize(1.0, new(k, n) / n**0.5, U)
    ad = C.MxAdapters((new(count, rank, n) / n**0.5).bfloat16(), new(count, rank, k).bfloat16())
    index = torch.randint(-1, count, (m,), generator=gen, device="cuda").to(torch.int32)
    q, h, y, z = C.MxMatrix.empty(8, m, k), torch.empty_like(x), torch.empty(m, n, device="cuda").bfloat16(), torch.empty_like(x)
    C.costa_mx_norm(1e-5, x, w1, R=r, H=h, Q=q)
    C.costa_mx_product(1.0, q, W, 0.0, y)
    C.costa_mx_product_adapted(1.0, y, U, ad, index, 0.0, z)
    want, _ = norm(wide(x) + wide(r), wide(w1))
    # 8 bits: half a step is 2^-4 of an element at most (and less below the block's largest values)
    assert off_by(values(q), want) <= 2.0**-4
    yy = values(q) @ values(W).T
    assert off_by(wide(y), yy) <= 2.0**-8 + k * 2.0**-24
    zz = wide(y) @ values(U).T
    for a in range(count):
        i = np.flatnonzero(index.cpu().numpy() == a)
        zz[i] += (wide(y)[i] @ wide(ad.A)[a].T) @ wide(ad.B)[a]
    assert off_by(wide(z), zz) <= 2.0**-8 + n * 2.0**-24


def off_by(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)
