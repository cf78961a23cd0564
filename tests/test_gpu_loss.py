"""Softmax cross entropy over a few-bit vocabulary on the GPU against the formulas in 64 bits.

Bounds.  A logit is off by E = (2 (k / 32 + 12) + 4) * 2^-24 of |alpha| |x| |W|; lse by the largest E of
its row (the log sum is a mean's shift at most), by 2 (n / 256 + 40) * 2^-24 for the sum of exponentials (chains of at most
n / 256, joins, the exponential's and the logarithm's last places) and by 2^-24 of |lse|; loss by E of the target's logit and as much.
The gradient G = d (exp(L - lse) - 1_t): the exponent off by e = E + (lse's) + 4 * 2^-24 (1 + |L - lse|), so |d| p e more, and 2 * 2^-24 |G|;
an exponential below 2^-126 is 0 (the instruction has no subnormal results), and of a float G what is below 2^-133 does not
enter a product: 2^-126 |d| + 2^-133 (with 40 times the usual logits, probabilities of 8e-43 came out as 0); in bfloat16 (as a part of the largest |d|, D) half a step, 2^-8 |G| and 2^-133 D.  dX, dW: G's bound times |W'|, |X'|, sums in 32 bits with
(2 (length / 32 + 12) + 8) * 2^-24 (a piece more or less is an addition more: the pieces' number on top), and the type's half step.
"""
import numpy as np
import pytest
import torch

import mx_formula as F

C = pytest.importorskip("paper_2106_06601_amd")
pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0**-24, "bf16": 2.0**-8, "f16": 2.0**-11}  # half of torch.finfo(t).eps
TINY = {"f32": 2.0**-149, "bf16": 2.0**-133, "f16": 2.0**-25}
U = 2.0**-24


def wide(t):
    return t.detach().to(torch.float64).cpu().numpy()


def keep(x, bits):
    """(the values that the stored form stands for, the matrix)"""
    data, scales = F.encode(x, bits)
    q = C.MxMatrix(bits, *x.shape, torch.from_numpy(data).cuda().reshape(-1), torch.from_numpy(scales).cuda().reshape(-1))
    return F.decode(data, scales, bits, x.shape[1]), q


def strided(x, dtype, ld):
    rows, cols = x.shape
    t = torch.full((rows, max(ld, 1)), 77.0, dtype=TORCH[dtype]).cuda()[:, :cols]
    t.copy_(torch.as_tensor(x))
    return t


class Case:
    def __init__(self, m, n, k, dtype, bits, alpha=1.0, gain=4.0, seed=0):
        rng = np.random.default_rng(seed + m * 7 + n * 11 + k * 13)
        w = (rng.standard_normal((n, k)) * (gain / max(k, 1)**0.5)).astype(np.float32)
        x = torch.from_numpy(rng.standard_normal((m, k))).to(TORCH[dtype])
        self.m, self.n, self.k, self.dtype, self.alpha = m, n, k, dtype, alpha
        self.w, self.wq = keep(w, bits)
        self.wt, self.wtq = keep(np.ascontiguousarray(w.T), bits)
        self.xt, self.xtq = keep(np.ascontiguousarray(x.float().numpy().T), 8)
        self.x = x
        t = rng.integers(0, n, m) if n else np.zeros(m, np.int64)
        t[rng.random(m) < 0.2] = -1
        t[rng.random(m) < 0.05] = n
        t[rng.random(m) < 0.05] = 2**62
        self.target = torch.from_numpy(t)
        self.d = torch.from_numpy((rng.standard_normal(m)).astype(np.float32))
        self.L = alpha * (wide(x) @ self.w.T)
        self.E = abs(alpha) * (2 * (k / 32 + 12) + 4) * U * (np.abs(wide(x)) @ np.abs(self.w).T)
        top = self.L.max(1)
        self.lse = top + np.log(np.exp(self.L - top[:, None]).sum(1))
        self.counts = (t >= 0) & (t < n)
        self.at = np.where(self.counts, t, 0)
        i = np.arange(m)
        self.loss = np.where(self.counts, self.lse - self.L[i, self.at], 0)
        own = 2 * (n / 256 + 40) * U + U * np.abs(self.lse)
        self.lse_off = self.E.max(1) + own
        self.loss_off = np.where(self.counts, self.E[i, self.at] + self.lse_off + 2 * U * np.abs(self.loss), 0)

    def gradients(self, bf16, beta_dw, d=None):
        d = np.where(self.counts, wide(self.d) if d is None else d, 0)[:, None]
        p = np.exp(self.L - self.lse[:, None])
        g = p.copy()
        g[np.arange(self.m), self.at] -= 1
        g, p = g * d, p * np.abs(d)
        off = p * (self.E + self.lse_off[:, None] + 4 * U * (1 + np.abs(self.L - self.lse[:, None]))) + 4 * U * (np.abs(g) + np.abs(d) * (np.abs(g) > p)) + 2.0**-126 * np.abs(d) + 2.0**-133
        off[~self.counts] = 0
        if bf16:
            off += (HALF["bf16"] + 2 * U) * (np.abs(g) + off) + TINY["bf16"] * max(1, np.abs(d).max())
        a, pieces = abs(self.alpha), 2 + self.n / 256
        dx, dw = self.alpha * (g @ self.wt.T), self.alpha * (g.T @ self.xt.T) + beta_dw
        ex = a * (off @ np.abs(self.wt).T + (2 * (self.n / 32 + 12) + 8 + pieces) * U * (np.abs(g) @ np.abs(self.wt).T))
        ew = a * (off.T @ np.abs(self.xt).T + (2 * (self.m / 32 + 12) + 8) * U * (np.abs(g).T @ np.abs(self.xt).T)) + 4 * U * np.abs(beta_dw)
        return dx, ex, dw, ew


SHAPES = [(1, 1, 1), (1, 40, 300), (3, 7, 5), (5, 2049, 8), (17, 130, 2500), (64, 5150, 127), (61, 2501, 520), (65, 1, 9), (66, 5, 3),
          (70, 129, 1030), (200, 2500, 257), (333, 1999, 40), (300, 4200, 64), (257, 513, 1029), (513, 1030, 130)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype,bits", [("f32", 8), ("bf16", 4), ("f16", 4), ("bf16", 8)])
def test_loss_and_gradients(shape, dtype, bits):
    m, n, k = shape
    for alpha, out in ((1.0, dtype), (-0.25, "f32" if dtype == "bf16" else "bf16")):
        c = Case(m, n, k, dtype, bits, alpha)
        x, target = strided(c.x, dtype, k + 3 * (alpha < 0)), c.target.cuda()
        for size in (None, *C.costa_mx_loss_workspace(m, n, k, False)):
            ws = None if size is None else torch.full((size,), 0xFF, dtype=torch.uint8).cuda()
            loss, lse = torch.full((m,), 7.0).cuda(), torch.full((m,), 7.0).cuda()
            C.costa_mx_loss(alpha, x, c.wq, target, loss, lse, workspace=ws)
            assert (np.abs(wide(lse) - c.lse) <= c.lse_off).all()
            assert (np.abs(wide(loss) - c.loss) <= c.loss_off).all()
        lse = torch.from_numpy(c.lse.astype(np.float32)).cuda()
        for wx, ww, d in ((True, True, True), (True, False, False), (False, True, True)):
            beta = 0.5 if ww and wx else 0.0
            dw0 = torch.randn(n, k).to(TORCH[out])
            bf16 = out == "bf16"  # (at most so coarse)
            dx, ex, dw, ew = c.gradients(bf16, beta * wide(dw0), None if d else np.ones(m))
            for size in (None, *C.costa_mx_loss_workspace(m, n, k, True)):
                ws = None if size is None else torch.full((size,), 0xFF, dtype=torch.uint8).cuda()
                DX = strided(np.full((m, k), np.nan), out, k + 1) if wx else None
                DW = strided(dw0 if beta else dw0 * np.nan, out, k + 2) if ww else None
                C.costa_mx_loss_backward(alpha, x, c.wq, target, lse, c.d.cuda() if d else None, WT=c.wtq if wx else None,
                                         dX=DX, XT=c.xtq if ww else None, dW=DW, beta=beta, workspace=ws)
                if wx:
                    assert (np.abs(wide(DX) - dx) <= ex + HALF[out] * np.abs(dx) + TINY[out]).all()
                if ww:
                    assert (np.abs(wide(DW) - dw) <= ew + HALF[out] * np.abs(dw) + TINY[out]).all()


# logits enough for the products' own tiles to keep them to themselves: tiles of 256 columns and of 128, the last
# ones cut in both directions
TILED = [(130, 33000, 40), (2047, 4101, 36), (1000, 9002, 24), (700, 16385, 8)]
# and, in bfloat16, for those of the weights' gradient (rows in fours and odd, tiles of 256 and of 128)
WEIGHTS = [(512, 8200, 1030), (300, 8201, 1024), (260, 2500, 520)]


@pytest.mark.parametrize("shape,dtype,bits", [
    *[(s, *t) for s in TILED for t in (("f32", 4), ("f32", 8), ("bf16", 4), ("bf16", 8), ("f16", 4), ("f16", 8))],
    *[(s, "bf16", 4) for s in WEIGHTS]], ids=str)
def test_loss_of_many_logits(shape, dtype, bits):
    m, n, k = shape
    out = "bf16" if dtype == "bf16" else "f32"
    c = Case(m, n, k, dtype, bits, -0.5)
    c.target[-1], c.target[0], c.target[1] = n - 1, 0, n // 256 * 256  # (a tile's corners)
    t = c.target.numpy()
    c.counts = (t >= 0) & (t < n)
    c.at = np.where(c.counts, t, 0)
    i = np.arange(m)
    c.loss = np.where(c.counts, c.lse - c.L[i, c.at], 0)
    c.loss_off = np.where(c.counts, c.E[i, c.at] + c.lse_off + 2 * U * np.abs(c.loss), 0)
    x, target = strided(c.x, dtype, k + 1), c.target.cuda()
    least, most = C.costa_mx_loss_workspace(m, n, k, False)
    got = []
    for size in (least, most):
        loss, lse = torch.full((m,), 7.0).cuda(), torch.full((m,), 7.0).cuda()
        C.costa_mx_loss(-0.5, x, c.wq, target, loss, lse, workspace=torch.full((size,), 0xFF, dtype=torch.uint8).cuda())
        assert (np.abs(wide(lse) - c.lse) <= c.lse_off).all()
        assert (np.abs(wide(loss) - c.loss) <= c.loss_off).all()
    dx, ex, dw, ew = c.gradients(out == "bf16", np.zeros((n, k)))
    least, most = C.costa_mx_loss_workspace(m, n, k, True)
    for size in (least, least + (most - least) // 20, most):
        DX, DW = strided(np.full((m, k), np.nan), out, k + 1), strided(np.full((n, k), np.nan), out, k + 2)
        C.costa_mx_loss_backward(-0.5, x, c.wq, target, lse, c.d.cuda(), WT=c.wtq, dX=DX, XT=c.xtq, dW=DW,
                                 workspace=torch.full((size,), 0xFF, dtype=torch.uint8).cuda())
        assert (np.abs(wide(DX) - dx) <= ex + HALF[out] * np.abs(dx) + TINY[out]).all()
        assert (np.abs(wide(DW) - dw) <= ew + HALF[out] * np.abs(dw) + TINY[out]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_of_a_larger_vocabulary(dtype):
    """Some thousand columns in pieces of every size that a workspace allows."""
    m, n, k = 90, 9000, 72
    c = Case(m, n, k, dtype, 4)
    x, target = c.x.cuda(), c.target.cuda()
    bf16 = dtype == "bf16"
    dx, ex, dw, ew = c.gradients(bf16, np.zeros((n, k)))
    least, most = C.costa_mx_loss_workspace(m, n, k, True)
    few, lots = C.costa_mx_loss_workspace(m, n, k, False)
    for f in (0.0, 0.03, 0.1, 0.3, 0.6):
        loss, lse = torch.zeros(m).cuda(), torch.zeros(m).cuda()
        ws = torch.full((int(few + f * (lots - few)),), 0xFF, dtype=torch.uint8).cuda()
        C.costa_mx_loss(1.0, x, c.wq, target, loss, lse, workspace=ws)
        assert (np.abs(wide(lse) - c.lse) <= c.lse_off).all() and (np.abs(wide(loss) - c.loss) <= c.loss_off).all()
        DX, DW = torch.zeros(m, k, dtype=TORCH[dtype]).cuda(), torch.zeros(n, k, dtype=TORCH[dtype]).cuda()
        ws = torch.full((int(least + f * (most - least)),), 0xFF, dtype=torch.uint8).cuda()
        C.costa_mx_loss_backward(1.0, x, c.wq, target, torch.from_numpy(c.lse.astype(np.float32)).cuda(), c.d.cuda(),
                                 WT=c.wtq, dX=DX, XT=c.xtq, dW=DW, workspace=ws)
        assert (np.abs(wide(DX) - dx) <= ex + HALF[dtype] * np.abs(dx) + TINY[dtype]).all()
        assert (np.abs(wide(DW) - dw) <= ew + HALF[dtype] * np.abs(dw) + TINY[dtype]).all()


@pytest.mark.parametrize("m", [5, 100])
@pytest.mark.parametrize("spread", [0.0, 1.0, 40.0, 1000.0])
def test_even_and_sure_rows(m, spread):
    """Logits all equal, and so far apart that one takes everything: nothing overflows, and the loss of a
    row that is nearly sure keeps its digits (the target's logit against the largest one)."""
    n, k = 3000, 32
    c = Case(m, n, k, "f32", 8, gain=spread)
    c.target[:] = torch.from_numpy(np.where(np.arange(m) % 3, c.L.argmax(1), np.arange(m) % n))
    c.__dict__.update(counts=np.ones(m, bool), at=c.target.numpy())
    i = np.arange(m)
    loss_want = c.lse - c.L[i, c.at]
    loss, lse = torch.zeros(m).cuda(), torch.zeros(m).cuda()
    C.costa_mx_loss(1.0, c.x.cuda(), c.wq, c.target.cuda(), loss, lse)
    assert (np.abs(wide(lse) - c.lse) <= c.lse_off).all()
    # of the target and of the row's largest, errors; then those of the log sum alone
    assert (np.abs(wide(loss) - loss_want) <= c.E[i, c.at] + c.E.max(1) + 2 * (n / 256 + 40) * U + 2 * U * np.abs(loss_want)).all()
    if spread == 0:
        assert (np.abs(wide(loss) - np.log(n)) <= 1e-6 * np.log(n)).all()
    dx, ex, dw, ew = c.gradients(False, np.zeros((n, k)))
    DX, DW = torch.zeros(m, k).cuda(), torch.zeros(n, k).cuda()
    C.costa_mx_loss_backward(1.0, c.x.cuda(), c.wq, c.target.cuda(), torch.from_numpy(c.lse.astype(np.float32)).cuda(), c.d.cuda(),
                             WT=c.wtq, dX=DX, XT=c.xtq, dW=DW)
    assert (np.abs(wide(DX) - dx) <= ex + HALF["f32"] * np.abs(dx) + TINY["f32"]).all()
    assert (np.abs(wide(DW) - dw) <= ew + HALF["f32"] * np.abs(dw) + TINY["f32"]).all()


@pytest.mark.parametrize("m", [6, 80])
def test_gradients_are_the_loss_s_differences(m):
    """In float with W restored from its few bits, so that dX's weights are the forward's: central
    differences of sum(d loss) at 2^-5; their third-order term and roundings are below 2e-2."""
    n, k = 50, 24
    c = Case(m, n, k, "f32", 8, gain=1.0)
    x, target, d = c.x.cuda(), c.target.cuda(), c.d.cuda()
    # a vocabulary whose two roundings are the same: powers of two
    w = np.exp2(np.random.default_rng(1).integers(-2, 1, (n, k))).astype(np.float32) * np.random.default_rng(2).choice([-1, 1], (n, k)).astype(np.float32)
    wv, wq = keep(w, 8)
    tv, wtq = keep(np.ascontiguousarray(w.T), 8)
    assert (wv == w).all() and (tv == w.T).all()

    def f(x):
        loss, lse = torch.zeros(m).cuda(), torch.zeros(m).cuda()
        C.costa_mx_loss(0.5, x, wq, target, loss, lse)
        return float((loss.double() * d.double()).sum()), lse

    DX = torch.zeros(m, k).cuda()
    C.costa_mx_loss_backward(0.5, x, wq, target, f(x)[1], d, WT=wtq, dX=DX)
    for at in range(0, m * k, 17):
        step = torch.zeros(m * k).cuda()
        step[at] = 2.0**-5
        step = step.view(m, k)
        assert abs((f(x + step)[0] - f(x - step)[0]) * 16 - float(DX.view(-1)[at])) < 2e-2


def test_rows_that_do_not_count_see_nothing():
    """NaN in a row without a target: its loss and gradient are 0; infinities and NaN in other rows stay there."""
    for m, n, k in ((8, 300, 64), (100, 300, 64)):
        for dtype in ("f32", "bf16"):
            c = Case(m, n, k, dtype, 8)
            c.target[:] = torch.arange(m) % n
            c.target[3] = -100
            x = c.x.clone()
            x[3], x[5] = float("nan"), float("nan")
            loss, lse = torch.zeros(m).cuda(), torch.zeros(m).cuda()
            C.costa_mx_loss(1.0, x.cuda(), c.wq, c.target.cuda(), loss, lse)
            assert loss[3] == 0 and torch.isnan(loss[5]) and torch.isnan(lse[5]) and torch.isnan(lse[3])
            fine = np.ones(m, bool)
            fine[[3, 5]] = False
            assert (np.abs(wide(lse) - c.lse)[fine] <= c.lse_off[fine]).all()
            DX = torch.full((m, k), 7.0).cuda()
            C.costa_mx_loss_backward(1.0, x.cuda(), c.wq, c.target.cuda(), lse, None, WT=c.wtq, dX=DX)
            assert not wide(DX)[3].any() and np.isnan(wide(DX)[5]).all() and np.isfinite(wide(DX)[fine]).all()


@pytest.mark.parametrize("m,n", [(20, 300), (200, 9000)])
def test_factors_of_rows_that_do_not_count(m, n):
    """In bfloat16 G is held as a part of the largest factor: NaN, infinities and huge ones of rows that do not
    count have no part in that, nor factors that are all 0."""
    k = 64
    c = Case(m, n, k, "bf16", 8)
    x, target = c.x.cuda(), c.target.cuda()
    lse = torch.from_numpy(c.lse.astype(np.float32)).cuda()
    kept = c.d.clone()
    for odd in (float("nan"), float("inf"), 3e38):
        c.d = torch.where(torch.from_numpy(c.counts), kept, torch.tensor(odd))
        dx, ex, _, _ = c.gradients(True, np.zeros((n, k)), np.where(c.counts, wide(kept), 0))
        DX = torch.full((m, k), 7.0).bfloat16().cuda()
        C.costa_mx_loss_backward(1.0, x, c.wq, target, lse, c.d.cuda(), WT=c.wtq, dX=DX)
        assert (np.abs(wide(DX) - dx) <= ex + HALF["bf16"] * np.abs(dx) + TINY["bf16"]).all()
    DX = torch.full((m, k), 7.0).bfloat16().cuda()
    C.costa_mx_loss_backward(1.0, x, c.wq, target, lse, torch.zeros(m).cuda(), WT=c.wtq, dX=DX)
    assert not DX.any()


def test_nothing_to_do():
    for m, n, k in ((0, 5, 6), (5, 0, 6), (5, 4, 0), (100, 0, 6), (100, 4, 0)):
        x, (w, wq), (_, wtq), (_, xtq) = torch.ones(m, k).cuda(), keep(np.ones((n, k), np.float32), 8), keep(np.ones((k, n), np.float32), 8), keep(np.ones((k, m), np.float32), 8)
        target = torch.zeros(m, dtype=torch.int64).cuda()
        loss, lse = torch.full((m,), 7.0).cuda(), torch.full((m,), 7.0).cuda()
        C.costa_mx_loss(1.0, x, wq, target, loss, lse)
        want = np.log(n) if n else -np.inf
        assert (np.abs(wide(lse) - want) <= 1e-6).all() if n else (wide(lse) == want).all()
        assert (np.abs(wide(loss) - (want if n else 0)) <= 1e-6).all()
        DX, DW = torch.full((m, k), 7.0).cuda(), torch.full((n, k), 8.0).cuda()
        C.costa_mx_loss_backward(1.0, x, wq, target, lse, None, WT=wtq, dX=DX, XT=xtq, dW=DW, beta=0.5)
        assert not DX.any() and (DW == 4).all()


@pytest.mark.parametrize("m", [30, 300])
def test_on_another_stream_and_in_a_graph(m):
    n, k = 2600, 520
    c = Case(m, n, k, "bf16", 4)
    x, target = c.x.cuda(), c.target.cuda()
    loss, lse, DX, DW = torch.zeros(m).cuda(), torch.zeros(m).cuda(), torch.zeros(m, k).bfloat16().cuda(), torch.zeros(n, k).bfloat16().cuda()
    ws = torch.empty(max(C.costa_mx_loss_workspace(m, n, k, b)[1] for b in (False, True)), dtype=torch.uint8, device="cuda")

    def both(stream=None):
        C.costa_mx_loss(1.0, x, c.wq, target, loss, lse, workspace=ws, stream=stream)
        C.costa_mx_loss_backward(1.0, x, c.wq, target, lse, None, WT=c.wtq, dX=DX, XT=c.xtq, dW=DW, workspace=ws, stream=stream)

    both()
    out = (loss, lse, DX, DW)
    want = [t.clone() for t in out]
    side = torch.cuda.Stream()
    for t in out:
        t.zero_()
    torch.cuda.synchronize()
    both(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, out))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        x.normal_()
        target.random_(-1, n)
        for t in out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out))
