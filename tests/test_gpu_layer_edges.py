"""The operators around products on the GPU, at the edges of what they say."""
import numpy as np
import pytest
import torch

import test_gpu_adapters as AD
import test_gpu_loss as L

C = pytest.importorskip("paper_2106_06601_amd")
pytestmark = pytest.mark.gpu
U = L.U


def bf16(x):
    return torch.from_numpy(x).to(torch.float32).to(torch.bfloat16)


@pytest.mark.parametrize("m,n,k", [(20, 4097, 40), (64, 1025, 256), (90, 4097, 7), (300, 8193, 136), (1000, 4097, 520)])
@pytest.mark.parametrize("dtype,bits", [("f32", 8), ("bf16", 4), ("f16", 8)])
@pytest.mark.parametrize("factors", [True, False])
def test_the_target_s_part_of_a_gradient_in_bfloat16_is_whole(m, n, k, dtype, bits, factors):
    """Rows of zeros over 2^a + 1 words: every word has 1 / n, and as a part of d (1 - 1 / n) the target's element
    is -1 and each other one 2^-a, which bfloat16 holds (the logits' and lse's roundings, some 2^-20, round
    off).  So dX is off by its sums in 32 bits alone, and is the rounded one of the formula in 64 bits
    wherever those do not reach another rounding."""
    c = L.Case(m, n, k, dtype, bits)
    c.x.zero_()
    t = np.arange(m) * 7 % n
    t[::5] = -1
    d = c.d.numpy().astype(np.float64) if factors else np.ones(m)
    x, target = c.x.cuda(), torch.from_numpy(t).cuda()
    loss, lse = torch.zeros(m).cuda(), torch.zeros(m).cuda()
    C.costa_mx_loss(1.0, x, c.wq, target, loss, lse)
    DX = torch.full((m, k), 7.0).bfloat16().cuda()
    C.costa_mx_loss_backward(0.75, x, c.wq, target, lse, c.d.cuda() if factors else None, WT=c.wtq, dX=DX)
    g = np.full((m, n), 1.0 / n)
    g[np.arange(m), np.maximum(t, 0)] -= 1
    g *= np.where(t >= 0, d, 0)[:, None]
    want = 0.75 * (g @ c.wt.T)
    # a factor off by 2^-20 / n of itself and 8 * 2^-24; sums of n, and the pieces'
    off = (2 * (n / 32 + 12) + 8 + 8 + n / 256) * U * 0.75 * (np.abs(g) @ np.abs(c.wt).T)
    low, high = bf16(want - off), bf16(want + off)
    known = (low == high).numpy()
    assert known.mean() > 0.8
    assert (DX.cpu() == low).numpy()[known].all()


@pytest.mark.parametrize("m", [9, 100, 300])
@pytest.mark.parametrize("spread", [8.0, 40.0, 1000.0])
@pytest.mark.parametrize("size", [1.0, 1e-30, 1e-40, 1e30])
def test_sure_rows_and_odd_factors_in_bfloat16(m, spread, size):
    """Rows from unsure to sure of their target and of another word; factors of all sizes, 0 and subnormal
    ones among them."""
    n, k = 3000, 32
    c = L.Case(m, n, k, "bf16", 8, gain=spread)
    t = np.where(np.arange(m) % 3, c.L.argmax(1), np.arange(m) % n)
    c.target[:] = torch.from_numpy(t)
    c.__dict__.update(counts=np.ones(m, bool), at=t)
    c.d *= size
    c.d[::4] = 0
    dx, ex, _, _ = c.gradients(True, np.zeros((n, k)))
    DX = torch.full((m, k), 7.0).bfloat16().cuda()
    C.costa_mx_loss_backward(1.0, c.x.cuda(), c.wq, c.target.cuda(), torch.from_numpy(c.lse.astype(np.float32)).cuda(), c.d.cuda(),
                             WT=c.wtq, dX=DX)
    # (sums of the smallest factors end below the floats' own steps: 2^-149 a term, 2^-133 the result's)
    least = n * 2.0**-149 * (1 + np.abs(c.wt).max()) + L.TINY["bf16"]
    assert (np.abs(L.wide(DX) - dx) <= ex + L.HALF["bf16"] * np.abs(dx) + least).all()


def test_a_factor_that_is_not_finite_stays_in_its_row():
    m, n, k = 100, 3000, 64
    c = L.Case(m, n, k, "bf16", 4)
    c.target[:] = torch.arange(m) * 11 % n
    c.__dict__.update(counts=np.ones(m, bool), at=c.target.numpy())
    dx, ex, _, _ = c.gradients(True, np.zeros((n, k)))
    d = c.d.clone()
    d[7], d[8] = float("inf"), float("nan")
    DX = torch.full((m, k), 7.0).bfloat16().cuda()
    C.costa_mx_loss_backward(1.0, c.x.cuda(), c.wq, c.target.cuda(), torch.from_numpy(c.lse.astype(np.float32)).cuda(), d.cuda(),
                             WT=c.wtq, dX=DX)
    fine = np.ones(m, bool)
    fine[[7, 8]] = False
    assert (np.abs(L.wide(DX) - dx) <= ex + L.HALF["bf16"] * np.abs(dx) + L.TINY["bf16"])[fine].all()
    assert np.isnan(L.wide(DX)[8]).all() and not np.isfinite(L.wide(DX)[7]).any()


@pytest.mark.parametrize("m,k", [(1, 64), (64, 64), (65, 8), (100, 64), (100, 128), (100, 129), (4096, 128), (300, 3000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_a_loss_over_no_words(m, k, dtype):
    """lse = log 0, no row counts; dX is a sum over nothing."""
    x, target = torch.ones(m, k).to(L.TORCH[dtype]).cuda(), torch.zeros(m, dtype=torch.int64).cuda()
    (_, w), (_, wt) = L.keep(np.ones((0, k), np.float32), 8), L.keep(np.ones((k, 0), np.float32), 8)
    for size in (None, C.costa_mx_loss_workspace(m, 0, k, False)[0]):
        loss, lse = torch.full((m,), 7.0).cuda(), torch.full((m,), 7.0).cuda()
        ws = None if size is None else torch.empty(size, dtype=torch.uint8).cuda()
        C.costa_mx_loss(1.0, x, w, target, loss, lse, workspace=ws)
        assert (lse == -float("inf")).all() and not loss.any()
        DX = torch.full((m, k), 7.0).to(L.TORCH[dtype]).cuda()
        C.costa_mx_loss_backward(1.0, x, w, target, lse, None, WT=wt, dX=DX)
        assert not DX.any()


@pytest.mark.parametrize("m,n,k,bits", [(512, 8200, 1030, 4), (300, 8201, 1024, 8), (260, 2500, 520, 4), (600, 20001, 264, 4)])
def test_gradients_have_the_same_precision_in_every_workspace(m, n, k, bits):
    """dX and dW in bfloat16 of rows of zeros, so that G has the same bits however it is made: in another workspace
    the sums in 32 bits come in another order, 2 (2 (n / 32 + 12) + 8) 2^-24 apart (1.4e-4 at most here, and mostly a
    tenth of that), which moves one result of a hundred or so across the border of a step of 2^-8.  (G in 32 bits in
    one of them and in bfloat16 in another one moves a quarter of them.)"""
    c = L.Case(m, n, k, "bf16", bits)
    x, target, lse = torch.zeros(m, k).bfloat16().cuda(), c.target.cuda(), torch.full((m,), float(np.log(n))).cuda()
    least, most = C.costa_mx_loss_workspace(m, n, k, True)
    got = []
    for size in (most, least, least + (most - least) // 30, least + (most - least) // 3):
        DX, DW = torch.zeros(m, k).bfloat16().cuda(), torch.zeros(n, k).bfloat16().cuda()
        C.costa_mx_loss_backward(1.0, x, c.wq, target, lse, c.d.cuda(), WT=c.wtq, dX=DX, XT=c.xtq, dW=DW,
                                 workspace=torch.full((size,), 0xFF, dtype=torch.uint8).cuda())
        got.append((DX, DW))
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert float((a != b).float().mean()) <= 0.05
            a, b = a.float(), b.float()
            assert ((a - b).abs() <= 2.0**-7 * torch.maximum(a.abs(), b.abs()) + 1e-3 * a.abs().mean()).all()


@pytest.mark.parametrize("m,how", [(40, "few"), (40, "none"), (3000, "few"), (3000, "none")])
@pytest.mark.parametrize("odd", [float("inf"), float("nan")])
def test_scales_that_are_not_finite_stay_with_their_rows(m, how, odd):
    """An adapter without rows has a gradient of beta G whatever its scale; one whose rows are all in one part of a
    split sum gets that part's; one of rank 0 adds nothing to its rows."""
    n, k, count, rank = 130, 256, 4, 8
    rng = np.random.default_rng(m)
    index = rng.integers(0, 2, m)
    index[index == 1] = 3
    if how == "few":
        index[:5] = 1
    index[5:8] = 2
    scales, ranks = torch.tensor([1.0, odd, odd, 0.5]), torch.tensor([8, 8, 0, 3], dtype=torch.int32)
    new = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    A, B, x, v = new(count, rank, k), new(count, rank, n), new(m, k), new(m, rank)
    ad = C.MxAdapters(A, B, ranks.cuda(), scales.cuda())
    at = torch.from_numpy(index.astype(np.int32)).cuda()
    for beta in (0.0, 2.0):
        for size in C.costa_mx_adapter_gradient_workspace(m, k, count, rank):
            G = torch.full((count, rank, k), 3.0 if beta else float("nan")).cuda()
            C.costa_mx_adapter_gradient(ad, at, v, x, beta, G, workspace=torch.full((size,), 0xFF, dtype=torch.uint8).cuda())
            assert (G[2] == 3 * beta).all() and (G[3, 3:] == 3 * beta).all() and torch.isfinite(G[0]).all() and torch.isfinite(G[3]).all()
            if how == "none":
                assert (G[1] == 3 * beta).all()
            else:
                assert (torch.isnan(G[1]) if odd != odd else torch.isinf(G[1])).all()
    w = C.MxMatrix.empty(8, n, k)
    C.costa_mx_quantize(1.0, new(n, k), w)
    y, plain = torch.zeros(m, n).cuda(), torch.zeros(m, n).cuda()
    C.costa_mx_product_adapted(1.0, x, w, ad, at, 0.0, y)
    C.costa_mx_product_adapted(1.0, x, w, ad, torch.full_like(at, -1), 0.0, plain)
    assert torch.equal(y[5:8], plain[5:8]) and torch.isfinite(y[8:]).all()


def guarded(size):
    """A workspace of so many bytes, with more behind it that a call has no part in."""
    room = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    return room, room[:size]


@pytest.mark.parametrize("m,n,k,count,rank", [(1, 40, 300, 3, 4), (61, 702, 1030, 6, 16), (333, 199, 1250, 5, 100), (900, 2000, 64, 3, 4),
                                              (1023, 260, 520, 7, 64), (1024, 4096, 64, 2, 32), (1300, 1999, 40, 1, 100),
                                              (2101, 10, 4161, 5, 70)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_no_call_writes_past_its_workspace(m, n, k, count, rank, dtype):
    c = AD.Case(m, n, k, count, rank, dtype, 4, "mixed")
    l = L.Case(m, n, k, dtype, 4)
    x, index, target = c.x.cuda(), c.index.cuda(), l.target.cuda()
    t = L.TORCH[dtype]

    def check(sizes, call):
        least, most = sizes
        for size in (least, (least + (most - least) // 3) // 16 * 16 if most > least else least, most):
            if size < least:
                continue
            room, ws = guarded(size)
            call(ws)
            assert (room[size:] == 0xA5).all()

    v, ev, want, off = c.forward(1.0, 0.0, dtype)
    for V in (None, torch.zeros(m, rank).cuda()):
        y = torch.zeros(m, n, dtype=t).cuda()

        def product(ws):
            y.fill_(float("nan"))
            C.costa_mx_product_adapted(1.0, x, c.wq, c.adapters, index, 0.0, y, V=V, workspace=ws)
            assert (np.abs(L.wide(y) - want) <= off).all()

        check(C.costa_mx_adapted_workspace(m, n, k, rank), product)
    G, V = torch.zeros(count, rank, k).cuda(), torch.zeros(m, rank).cuda()
    check(C.costa_mx_adapter_gradient_workspace(m, k, count, rank),
          lambda ws: C.costa_mx_adapter_gradient(c.adapters, index, V, x, 0.0, G, workspace=ws))
    loss, lse = torch.zeros(m).cuda(), torch.zeros(m).cuda()
    check(C.costa_mx_loss_workspace(m, n, k, False), lambda ws: C.costa_mx_loss(1.0, l.x.cuda(), l.wq, target, loss, lse, workspace=ws))
    DX, DW = torch.zeros(m, k, dtype=t).cuda(), torch.zeros(n, k, dtype=t).cuda()
    for dx, dw in ((DX, None), (DX, DW), (None, DW)):
        check(C.costa_mx_loss_workspace(m, n, k, True),
              lambda ws: C.costa_mx_loss_backward(1.0, l.x.cuda(), l.wq, target, lse, None, WT=l.wtq, dX=dx, XT=l.xtq, dW=dw, workspace=ws))
    H, D, dw, s = torch.ones(m, n, dtype=t).cuda(), torch.zeros(m, n, dtype=t).cuda(), torch.zeros(n).cuda(), torch.ones(m).cuda()
    check(C.costa_mx_norm_workspace(m, n), lambda ws: C.costa_mx_norm_backward(H, H, None, s, D, dW=dw, workspace=ws))


@pytest.mark.parametrize("shape", [(900, 2000, 64, 3, 4), (1000, 4099, 300, 5, 4), (700, 3001, 129, 4, 33), (521, 2501, 1030, 2, 100)], ids=str)
@pytest.mark.parametrize("dtype,bits", [("f32", 4), ("bf16", 8), ("f16", 4)])
@pytest.mark.parametrize("how", ["runs", "mixed"])
def test_sums_that_go_by_slices_of_rows(shape, dtype, bits, how):
    """Fewer rows than the products' own tiles take, and a workspace that does not hold their sums: X, the index, V and C
    are each at the slice's first row, and the sums' room is used again.  Within the bounds of the whole, which
    count any order of the sums (a slice may be split otherwise than the whole)."""
    m, n, k, count, rank = shape
    c = AD.Case(m, n, k, count, rank, dtype, bits, how)
    out = "f32" if how == "mixed" else dtype
    v, ev, want, off = c.forward(-0.5, 0.25, out)
    X, index = AD.strided(c.x, dtype, k + 3), c.index.cuda()
    least, most = C.costa_mx_adapted_workspace(m, n, k, rank)
    sums, kept = 4 * n, -(-4 * m * rank // 16) * 16  # a row's; v's
    slices = []
    for size in (least, least + 100 * sums, least + 300 * sums, most):
        for V in (None, AD.strided(np.full((m, rank), np.nan), "f32", rank + 2)):
            room = size - (kept if V is None else 0)
            slices.append(-(-m // (room // sums)))
            y, ws = AD.strided(c.c0, out, n + 5), torch.full((size,), 0xFF, dtype=torch.uint8).cuda()
            C.costa_mx_product_adapted(-0.5, X, c.wq, c.adapters, index, 0.25, y, V=V, workspace=ws)
            assert (np.abs(L.wide(y) - want) <= off).all()
            assert (y._base[:, n:] == 77).all()
            if V is not None:
                assert (np.abs(L.wide(V) - v) <= ev).all()
    assert slices[0] > 1 and slices[1] > 1 and slices[-1] == 1


# Relative to the whole gradient.  Eight results follow one another (y1, z, h2, y2 and, back, those of y2, h2, y1 and x), each
# rounded by at most half a step h of its elements: 2^-8, 2^-11, spread evenly over it at the worst, so h / sqrt(3) of its
# norm; independent of one another, sqrt(8 / 3) h together, and the norms and the softmax between them
# pass on no more than some 2.5 times as much: 4 h.
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("tokens,inputs,words,requests,rank", [(130, 200, 1003, 3, 20), (1100, 512, 2500, 4, 16), (300, 256, 9000, 2, 32)])
def test_a_training_step_is_off_by_its_roundings(dtype, tokens, inputs, words, requests, rank):
    import test_gpu_layer_step as T
    import adapted_layer as E
    gen = torch.Generator(device="cuda")
    gen.manual_seed(tokens + 1)
    M = E.Model(inputs, words, requests, rank, dtype, gen)
    x = torch.randn(tokens, inputs, generator=gen, device="cuda").to(dtype)
    index = torch.randint(-1, requests, (tokens,), generator=gen, device="cuda").to(torch.int32)
    target = torch.randint(0, words, (tokens,), generator=gen, device="cuda")
    loss, grads = M.step(x, index, target)
    want, wants = T.chain(M, x, index.cpu().numpy(), target.cpu().numpy())
    half = torch.finfo(dtype).eps / 2
    assert abs(float(loss) - want) <= 4 * half * want
    off = {name: T.off(grads[name], wants[name]) / half for name in wants}
    assert max(off.values()) <= 4, off


@pytest.mark.parametrize("m,n", [(5, 1023), (9, 2501), (3, 8191), (2, 16400), (700, 33)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bits", [4, 8])
def test_a_norm_s_few_bits_alone_are_the_same(m, n, dtype, bits):
    """Codes, scales and what pads them, with H, Y and rstd beside them and without."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m * n)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(L.TORCH[dtype])  # noqa: E731
    x, r, w = new(m, n), new(m, n), new(n)
    kept = []
    for more in (dict(), dict(H=torch.empty_like(x), Y=torch.empty_like(x), rstd=torch.empty(m, device="cuda"))):
        q = C.MxMatrix(bits, m, n, *(torch.full((k,), 0xA5, dtype=torch.uint8, device="cuda") for k in C.costa_mx_sizes(bits, m, n)))
        C.costa_mx_norm(1e-5, x, w, R=r, Q=q, **more)
        kept.append(q)
    assert torch.equal(kept[0].data, kept[1].data) and torch.equal(kept[0].scales, kept[1].scales)
    pad = -(-n // 32)
    assert not kept[0].scales.view(m, -1)[:, pad:].any()


@pytest.mark.parametrize("m", [3, 100])
@pytest.mark.parametrize("top,gap", [(112.0, 14.0), (96.0, 6.0), (-96.0, 12.0), (448.0, 14.0)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_what_lse_s_rounding_costs_a_sure_row(m, top, gap, out):
    """Logits that are whole numbers, `gap` below the target's, and weights behind that pick one word each, so that dX is
    G: a probability is off by 2^-24 |lse| of itself, the target's element by as much, and some 8 * 2^-24 (1 + gap) of
    the exponential's; the loss by its own last places alone."""
    n, k = 40, 40
    w, x = np.zeros((n, k), np.float32), np.zeros((m, k), np.float32)
    x[:, 0], x[:, 32] = top, gap
    w[:, 0], w[1:, 32] = 1.0, -1.0  # (two blocks of a stored row)
    values, wq = L.keep(w, 8)
    assert (values == w).all()
    one, wtq = L.keep(np.eye(k, n, dtype=np.float32), 8)
    assert (one == np.eye(k, n)).all()
    logits = x.astype(np.float64) @ values.T
    assert (logits[:, 0] == top).all() and (logits[:, 1:] == top - gap).all()
    rest = (n - 1) * np.exp(-gap)
    loss, lse, target = torch.zeros(m).cuda(), torch.zeros(m).cuda(), torch.zeros(m, dtype=torch.int64).cuda()
    X = torch.from_numpy(x).cuda()
    C.costa_mx_loss(1.0, X, wq, target, loss, lse)
    want = np.log1p(rest)
    # The sum 1 + rest, below 2, is of 40 exponentials: up to 15 additions in a lane, 6 between lanes and 3 between waves, each
    # off by 2^-24 at most; the exponentials by 8 * 2^-24 (1 + gap) of themselves; the logarithm by two steps of its
    # result, below 1.
    assert (np.abs(L.wide(loss) - want) <= (24 + 8 * (1 + gap) * rest + 2) * U).all()
    DX = torch.zeros(m, k).to(L.TORCH[out]).cuda()
    C.costa_mx_loss_backward(1.0, X, wq, target, lse, None, WT=wtq, dX=DX)
    g = np.full(n, np.exp(-gap) / (1 + rest))
    g[0] = -rest / (1 + rest)
    off = U * abs(top + want) + 8 * U * (1 + gap)
    p = np.where(np.arange(n) == 0, 1.0, np.abs(g))
    # (in bfloat16: G's half step of words that are not the target, and dX's)
    halves = 0 if out == "f32" else 2 * L.HALF[out]
    assert (np.abs(L.wide(DX) - g) <= p * off * (1 + halves) + (halves + L.HALF[out]) * np.abs(g)).all()


def apart(t, ld):
    """A copy of t with rows `ld` elements apart (what lies between is not set)."""
    far = torch.empty(t.shape[0], ld, dtype=t.dtype, device="cuda")[:, :t.shape[1]]
    far.copy_(t)
    return far


@pytest.mark.parametrize("m,n,k,rank", [(70, 130, 264, 16), (2100, 100, 4161, 20), (1100, 2051, 300, 5)])
def test_rows_whose_offsets_pass_32_bits(m, n, k, rank):
    """Elements past the 2^32nd of a buffer, in each operand: the same bits as next to one another."""
    ld, count = (2**32 // m + 4096) // 8 * 8 + 3, 3
    c, l = AD.Case(m, n, k, count, rank, "bf16", 4, "mixed"), L.Case(m, n, k, "bf16", 4)
    x, dy, index, target = c.x.cuda(), c.dy.cuda(), c.index.cuda(), l.target.cuda()
    X = apart(x, ld)

    y, V = torch.zeros(m, n).bfloat16().cuda(), torch.zeros(m, rank).cuda()
    C.costa_mx_product_adapted(1.0, x, c.wq, c.adapters, index, 0.0, y, V=V)
    Y = apart(y * 0, ld)
    C.costa_mx_product_adapted(1.0, X, c.wq, c.adapters, index, 0.0, Y)
    assert torch.equal(Y, y)
    del Y
    G, H = torch.zeros(count, rank, k).cuda(), torch.zeros(count, rank, k).cuda()
    C.costa_mx_adapter_gradient(c.adapters, index, V, x, 0.0, G)
    C.costa_mx_adapter_gradient(c.adapters, index, V, X, 0.0, H)
    assert torch.equal(G, H)
    FV = apart(V, ld)
    H.zero_()
    C.costa_mx_adapter_gradient(c.adapters, index, FV, x, 0.0, H)
    assert torch.equal(G, H)
    FV.zero_()
    C.costa_mx_product_adapted(1.0, x, c.wq, c.adapters, index, 0.0, y, V=FV)
    assert torch.equal(FV, V)
    del FV

    one, far = [(torch.zeros(m).cuda(), torch.zeros(m).cuda()) for _ in range(2)]
    C.costa_mx_loss(1.0, x, l.wq, target, *one)
    C.costa_mx_loss(1.0, X, l.wq, target, *far)
    assert torch.equal(one[0], far[0]) and torch.equal(one[1], far[1])
    DX = torch.zeros(m, k).bfloat16().cuda()
    FX = apart(DX, ld)
    C.costa_mx_loss_backward(1.0, x, l.wq, target, one[1], l.d.cuda(), WT=l.wtq, dX=DX)
    C.costa_mx_loss_backward(1.0, X, l.wq, target, one[1], l.d.cuda(), WT=l.wtq, dX=FX)
    assert torch.equal(DX, FX)

    w, s, t = torch.rand(k).cuda(), torch.zeros(m).cuda(), torch.zeros(m).cuda()
    want, got = torch.zeros_like(x), FX
    C.costa_mx_norm(1e-5, x, w, R=DX, Y=want, rstd=s)
    kept = DX.clone()
    C.costa_mx_norm(1e-5, X, w, R=kept, Y=got, rstd=t)
    assert torch.equal(want, got) and torch.equal(s, t)
    a, b = [torch.zeros(k).cuda() for _ in range(2)]
    C.costa_mx_norm_backward(want, x, w, s, kept, dW=a)
    C.costa_mx_norm_backward(got, X, w, s, got, dW=b)
    assert torch.equal(kept, got) and torch.equal(a, b)
