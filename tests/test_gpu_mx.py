"""Microscaled matrices on the GPU: quantisation bit for bit against the
formula in 64 bits, products and gradients against 64-bit sums of the values
that the stored matrices stand for.

Bounds.  Quantisation and its inverse are exact or rounded once: compared for
equality.  Products: each is a sum of exact products in 32 bits, so an element
is off by at most about (k / 32 + 8) roundings (each matrix instruction adds 32
or more products and rounds once or a few times) of 2^-24 of the sum of
magnitudes S = sum |a b|, and by the rounding of the result: 2^-24, 2^-9 or
2^-11 of it.
"""
import numpy as np
import pytest
import torch

import mx_formula as F

C = pytest.importorskip("paper_2106_06601_amd")
pytestmark = pytest.mark.gpu

TORCH = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": 2.0**-24, "bf16": 2.0**-9, "f16": 2.0**-11}


def gpu(x, dtype="f32"):
    return torch.as_tensor(x).to(TORCH[dtype]).cuda()


def filled(bits, rows, cols):
    """A matrix whose buffers hold garbage before the call, with guard bytes behind them."""
    d, s = C.costa_mx_sizes(bits, rows, cols)
    data = torch.full((d + 64,), 0xA5, dtype=torch.uint8).cuda()
    scales = torch.full((s + 64,), 0xA5, dtype=torch.uint8).cuda()
    return C.MxMatrix(bits, rows, cols, data, scales)


def stored(q):
    """(data, scales) as numpy, after a look at the guards."""
    d, s = C.costa_mx_sizes(q.bits, q.rows, q.cols)
    data, scales = q.data.cpu().numpy(), q.scales.cpu().numpy()
    assert (data[d:] == 0xA5).all() and (scales[s:] == 0xA5).all(), "written past the end"
    return data[:d].reshape(q.rows, -1), scales[:s].reshape(q.rows, -1)


def check_stored(q, x):
    data, scales = stored(q)
    want_data, want_scales = F.encode(x, q.bits)
    np.testing.assert_array_equal(scales, want_scales)
    np.testing.assert_array_equal(data, want_data)


def keep(x, bits):
    """The stored form of a numpy matrix, made by the formula."""
    data, scales = F.encode(x, bits)
    return C.MxMatrix(bits, *x.shape, torch.from_numpy(data).cuda().reshape(-1), torch.from_numpy(scales).cuda().reshape(-1))


def values(rng, rows, cols, dtype="f32"):
    """Normal values over a few orders of magnitude, blocks of zeros, ties."""
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-8, 8, (rows, cols)))
    x[rng.random((rows, cols)) < 0.1] = 0.0
    x[rng.random((rows, cols)) < 0.1] = 2.5
    if cols >= 64:
        x[:, 32:64] = 0.0
    return torch.from_numpy(x).to(TORCH[dtype]).to(torch.float64).numpy()


SHAPES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 127), (33, 128), (129, 130), (64, 256), (31, 257), (257, 1),
          (200, 515), (130, 1000)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["f64", "f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["row", "col"])
def test_quantize_both_ways(shape, bits, dtype, order):
    rng = np.random.default_rng(hash((shape, bits)) % 2**32)
    x = values(rng, *shape, dtype)
    t = gpu(x, dtype)
    if order == "col":
        t = t.t().contiguous().t()
    x = x.astype(np.float32)
    for which in ("q", "qt", "both"):
        q = filled(bits, *shape) if which != "qt" else None
        qt = filled(bits, *shape[::-1]) if which != "q" else None
        C.costa_mx_quantize(1.0, t, q, qt)
        if q is not None:
            check_stored(q, x)
        if qt is not None:
            check_stored(qt, x.T)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("ld,offset", [(130, 0), (131, 1), (136, 8), (128, 3)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_strided_source(bits, ld, offset, dtype):
    rng = np.random.default_rng(7)
    flat = gpu(rng.standard_normal(40 * ld + offset + 200), dtype)
    t = torch.as_strided(flat, (40, 127), (ld, 1), offset)
    x = t.to(torch.float32).cpu().numpy()
    for src, want in ((t, x), (t.t(), x.T)):
        q, qt = filled(bits, *want.shape), filled(12 - bits, *want.shape[::-1])  # the other format across
        C.costa_mx_quantize(1.0, src, q, qt)
        check_stored(q, want)
        check_stored(qt, want.T)
        q = filled(bits, *want.shape)
        C.costa_mx_quantize(1.0, src, q)
        check_stored(q, want)


@pytest.mark.parametrize("bits", [4, 8])
def test_every_rounding(bits):
    """Values on, just beside and between every two neighbours of the format, in
    blocks whose largest magnitude is the format's or the largest that rounds down to it."""
    grid = F.GRID[bits]
    mid = (grid[1:] + grid[:-1]) / 2
    v = np.concatenate([grid, mid, np.nextafter(mid.astype(np.float32), 0), np.nextafter(mid.astype(np.float32), 1e9)])
    v = np.concatenate([v, -v]).astype(np.float32)
    v = np.resize(v, (-(-v.size // 31), 31))
    for top in (grid[-1], np.nextafter(np.float32(2 * 2.0 ** F.EMAX[bits]), 0)):
        for scale in (1.0, 2.0**-126, 2.0**-120, 2.0**100):
            x = np.concatenate([v, np.full((v.shape[0], 1), top, np.float32)], 1) * np.float32(scale)
            for alpha in (1.0, -2.0):
                q, qt = filled(bits, *x.shape), filled(bits, *x.shape[::-1])
                C.costa_mx_quantize(alpha, gpu(x), q, qt)
                check_stored(q, x * np.float32(alpha))
                check_stored(qt, (x * np.float32(alpha)).T)
                back = torch.full(x.shape, 7.0).cuda()
                C.costa_mx_dequantize(1.0, q, 0.0, back)
                np.testing.assert_array_equal(back.cpu().numpy().astype(np.float64), F.decode(*F.encode(x * np.float32(alpha), bits), bits, x.shape[1]))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("alpha", [-1.0, 0.0, float("inf"), float("nan")])
def test_scalars_leave_what_pads_a_row_alone(bits, alpha):
    x = np.abs(np.random.default_rng(9).standard_normal((37, 45))).astype(np.float32) + 1
    with np.errstate(invalid="ignore"):
        want = x * np.float32(alpha)
    for dtype in ("f32", "bf16"):
        w = want if dtype == "f32" else torch.from_numpy(x).bfloat16().float().numpy() * np.float32(alpha)
        q, qt = filled(bits, 37, 45), filled(bits, 45, 37)
        C.costa_mx_quantize(alpha, gpu(x, dtype), q, qt)
        check_stored(q, w)
        check_stored(qt, w.T)
        q = filled(bits, 37, 45)
        C.costa_mx_quantize(alpha, gpu(x, dtype), q)
        check_stored(q, w)


@pytest.mark.parametrize("bits", [4, 8])
def test_extremes_and_what_is_no_number(bits):
    big = np.finfo(np.float32).max
    x = np.random.default_rng(3).standard_normal((16, 96)).astype(np.float32)
    x[0, 5] = np.inf
    x[1, 40] = -np.inf
    x[2, 95] = np.nan
    x[3] = big
    x[4] = 1e-40  # subnormals
    x[5, :32] = 0.0
    x[6, :32] = -0.0
    x[7, 0] = big
    x[8, :32] = 2.0**-149
    x[9, 0] = np.frombuffer(np.uint32(0x7F800001).tobytes(), np.float32)[0]  # a NaN whose upper half reads as infinity
    q, qt = filled(bits, *x.shape), filled(bits, *x.shape[::-1])
    C.costa_mx_quantize(1.0, gpu(x), q, qt)
    check_stored(q, x)
    check_stored(qt, x.T)
    back = torch.empty(16, 96).cuda()
    C.costa_mx_dequantize(1.0, q, 0.0, back)
    b = back.cpu().numpy()
    assert np.isnan(b[0, :32]).all() and np.isnan(b[1, 32:64]).all() and np.isnan(b[2, 64:]).all()
    assert np.isnan(b[9, :32]).all() and np.isfinite(b[[0, 2, 3, 4, 5, 6, 7, 8, 9], 32:64]).all()
    # a double past the floats' range is an infinity
    q = filled(bits, 1, 32)
    C.costa_mx_quantize(1.0, gpu(np.full((1, 32), 1e300), "f64"), q)
    assert (stored(q)[1][0, 0] == 255).all()


@pytest.mark.parametrize("spec", [
    ("bc", 70, 90, 16, 8, 3, 2, "row", "col"), ("bc", 300, 257, 32, 64, 2, 2, "col", "row"),
    ("bc", 129, 1000, 100, 77, 2, 3, "row", "row"), ("bc", 1, 200, 5, 3, 2, 2, "row", "col"),
    ("bc", 500, 1, 64, 1, 4, 1, "row", "row"), ("bc", 130, 140, 1, 1, 2, 3, "row", "col"), ("gen", 131, 260, "row"),
    ("gen", 131, 260, "col"), ("gen1", 64, 100, "col"), ("window", 201, 140)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
def test_quantize_out_of_layouts(spec, dtype):
    import synth
    rng = np.random.default_rng(11)
    kind, m, n = spec[:3]
    if kind == "bc":
        L = C.Layout.block_cyclic(*spec[1:])
    elif kind == "gen":
        rs = [0] + sorted(rng.choice(np.arange(1, m), 7, replace=False).tolist()) + [m]
        cs = [0] + sorted(rng.choice(np.arange(1, n), 9, replace=False).tolist()) + [n]
        L = C.Layout.general(m, n, rs, cs, rng.integers(0, 5, 80).tolist(), 6, spec[3])
    elif kind == "gen1":
        L = C.Layout.general(m, n, [0, m], [0, n], [1], 3, spec[3], [5], [m + 2])
    else:
        big = C.Layout.scalapack([1, 0, 400, 300, 37, 20, 1, 2, 250], 2, 3)
        L = big.submatrix(17, 45, m, n)
    bufs = [torch.zeros(L.local_elems(r), dtype=TORCH[dtype]).cuda() if L.local_elems(r) else None
            for r in range(L.nranks)]
    x = values(rng, m, n, dtype)
    host = [None if b is None else b.cpu().to(torch.float64).numpy() for b in bufs]
    rs, cs = _splits(L, spec, rng)
    for bi in range(L.nbr):
        for bj in range(L.nbc):
            o, off, ld = C.costa_layout_block(L.handle, bi, bj)
            for i in range(rs[bi], rs[bi + 1]):
                j = np.arange(cs[bj], cs[bj + 1])
                at = off + (i - rs[bi]) + (j - cs[bj]) * ld if L.block_order == "col" else \
                    off + (i - rs[bi]) * ld + (j - cs[bj])
                host[o][at] = x[i, j]
    bufs = [None if h is None else gpu(h, dtype) for h in host]
    x = x.astype(np.float32)
    for bits in (4, 8):
        q, qt = filled(bits, m, n), filled(12 - bits, n, m)
        C.costa_mx_quantize_layout(dtype, 1.0, L, bufs, q, qt)
        check_stored(q, x)
        check_stored(qt, x.T)
        qt = filled(bits, n, m)
        C.costa_mx_quantize_layout(dtype, 0.5, L, bufs, None, qt)
        check_stored(qt, x.T * np.float32(0.5))


def test_quantize_window_far_into_a_matrix():
    """Rows past 2^32 of a block-cyclic matrix; the ranks' buffers are addressed as
    if the whole of their local matrices were there, and only the window's part is read."""
    nb, np_, r0, m, n = 1 << 31, 2, (1 << 32) + 77, 100, 70
    whole = C.Layout.block_cyclic(1 << 33, n, nb, 32, np_, 1, "row", "row")
    L = whole.submatrix(r0, 0, m, n)
    x = np.random.default_rng(8).standard_normal((m, n)).astype(np.float32)
    t = gpu(x)
    # row r0 + i is in block 2, process 0's second: its local row nb + 77 + i
    at = t.data_ptr() - (nb + 77) * n * 4
    q, qt = filled(8, m, n), filled(4, n, m)
    C.costa_mx_quantize_layout("f32", 1.0, L, [at, 16], q, qt)
    check_stored(q, x)
    check_stored(qt, x.T)


def _splits(L, spec, rng):
    """The splits of a test's layout, from its recipe."""
    kind, m, n = spec[:3]
    if kind == "bc":
        mb, nb = spec[3:5]
        return list(range(0, m, mb)) + [m], list(range(0, n, nb)) + [n]
    if kind == "gen1":
        return [0, m], [0, n]
    if kind == "window":
        cut = lambda o, n, b: [0] + [c - o for c in range((o // b + 1) * b, o + n, b)] + [n]  # noqa: E731
        return cut(17, m, 37), cut(45, n, 20)
    rng = np.random.default_rng(11)  # the generator as it was
    return ([0] + sorted(rng.choice(np.arange(1, m), 7, replace=False).tolist()) + [m],
            [0] + sorted(rng.choice(np.arange(1, n), 9, replace=False).tolist()) + [n])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["f64", "f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["row", "col"])
@pytest.mark.parametrize("alpha,beta", [(1.0, 0.0), (0.375, 0.0), (-1.0, 1.0), (0.75, -2.5)])
def test_dequantize(bits, dtype, order, alpha, beta):
    rng = np.random.default_rng(5)
    for rows, cols in ((1, 1), (3, 7), (65, 250), (40, 264)):
        x = rng.standard_normal((rows, cols)).astype(np.float32)
        q = keep(x, bits)
        a = rng.standard_normal((rows, cols))
        if beta == 0.0:
            a[:] = np.nan  # not read
        a = gpu(a, dtype)
        if order == "col":
            a = a.t().contiguous().t()
        W = torch.float64 if dtype == "f64" else torch.float32
        v = torch.from_numpy(F.decode(*F.encode(x, bits), bits, cols)).to(W)
        want = v * alpha
        if beta:
            want = want + a.cpu().to(W) * beta
        C.costa_mx_dequantize(alpha, q, beta, a)
        np.testing.assert_array_equal(a.cpu().to(torch.float64).numpy(), want.to(TORCH[dtype]).to(torch.float64).numpy())


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def check_product(got, a, b, alpha, beta, c0, out):
    """got against alpha a b^T + beta c0 in 64 bits."""
    got = got.cpu().to(torch.float64).numpy()
    k = a.shape[1]
    want = alpha * (a @ b.T)
    size = abs(alpha) * (np.abs(a) @ np.abs(b).T)
    if beta:
        want = want + beta * c0
        size = size + np.abs(beta * c0)
    bound = (k / 32 + 8) * 2.0**-24 * size + 2 * UNIT[out] * np.abs(want) + (2.0**-24 if out == "f16" else 0.0)
    off = np.abs(got - want)
    assert (off <= bound + 1e-300).all(), (off / (bound + 1e-300)).max()


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 130, 500), (3, 17, 33), (16, 16, 128), (17, 100, 257), (40, 300, 129),
            (64, 64, 4096), (65, 33, 2000), (128, 128, 256), (130, 260, 384), (257, 255, 640), (300, 513, 1000),
            (513, 300, 96), (7, 1024, 8192), (260, 20, 5000), (70, 40, 5), (5, 300, 7), (130, 70, 8)]


@pytest.mark.parametrize("m,n,k", PRODUCTS, ids=str)
@pytest.mark.parametrize("abits,bbits", [(4, 4), (8, 4), (4, 8), (8, 8)])
@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
def test_product(m, n, k, abits, bbits, out):
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    a, b = rng.standard_normal((m, k)), rng.standard_normal((n, k)) * 0.25
    a[:, :: 17] *= 20
    qa, qb = keep(a, abits), keep(b, bbits)
    va, vb = F.decode(*F.encode(a, abits), abits, k), F.decode(*F.encode(b, bbits), bbits, k)
    c = torch.full((m, n), float("nan"), dtype=TORCH[out]).cuda()
    C.costa_mx_product(0.125, qa, qb, 0.0, c)
    check_product(c, va, vb, 0.125, 0.0, None, out)
    # by columns, with padding around it, added to what is there
    flat = torch.randn((m + 3) * n + 8).to(TORCH[out]).cuda()
    before = flat.clone()
    c = torch.as_strided(flat, (m, n), (1, m + 3), 5)
    c0 = c.cpu().to(torch.float64).numpy()
    C.costa_mx_product(-0.5, qa, qb, 0.75, c)
    check_product(c, va, vb, -0.5, 0.75, c0, out)
    mask = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(mask, (m, n), (1, m + 3), 5).fill_(False)
    assert torch.equal(flat[mask], before[mask]), "written outside C"


@pytest.mark.parametrize("m,n,k", PRODUCTS, ids=str)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("op", ["N", "T"])
@pytest.mark.parametrize("order", ["row", "col"])
def test_product_real(m, n, k, bits, dtype, op, order):
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    a, b = rng.standard_normal((m, k)), rng.standard_normal((n, k)) * 0.25
    a[:, :: 17] *= 20
    t = gpu(a, dtype)
    a = t.cpu().to(torch.float64).numpy()
    if op == "T":
        t = t.t()
    rows, cols = t.shape
    pad = {"f32": 1, "bf16": 8, "f16": 0}[dtype]  # odd and even strides
    if order == "row":
        held = torch.full((rows, cols + pad), float("nan"), dtype=TORCH[dtype]).cuda()
        held[:, :cols] = t
        t = held[:, :cols]
    else:
        held = torch.full((cols, rows + pad), float("nan"), dtype=TORCH[dtype]).cuda()
        held[:, :rows] = t.t()
        t = held[:, :rows].t()
    q = keep(b, bits)
    vb = F.decode(*F.encode(b, bits), bits, k)
    for out in ("f32", dtype):
        c = torch.full((m, n), float("nan"), dtype=TORCH[out]).cuda()
        C.costa_mx_product_real(1.0, op, t, q, 0.0, c)
        check_product(c, a, vb, 1.0, 0.0, None, out)
        c = torch.randn(n, m + 1).to(TORCH[out]).cuda().t()[:m]
        c0 = c.cpu().to(torch.float64).numpy()
        C.costa_mx_product_real(-0.25, op, t, q, 1.0, c)
        check_product(c, a, vb, -0.25, 1.0, c0, out)


@pytest.mark.parametrize("m", [1, 5, 40, 300])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_what_is_no_number_stays_where_it_is(m, dtype):
    """An infinity or a NaN of one row, and a block of NaN of one column, reach
    that row or column and no other element."""
    n, k = 200, 700
    rng = np.random.default_rng(1)
    a, b = rng.standard_normal((m, k)), np.abs(rng.standard_normal((n, k))) + 0.5
    b[3, 600] = np.nan
    a[m - 1, 650] = np.inf
    if m > 1:
        a[0, 699] = np.nan
    q = keep(b, 8)
    for op in ("N", "T"):
        t = gpu(a, dtype)
        c = torch.zeros(m, n).cuda()
        C.costa_mx_product_real(1.0, op, t if op == "N" else t.t().contiguous(), q, 0.0, c)
        c = c.cpu().numpy()
        want = np.full((m, n), 0.0)
        want[m - 1] = np.inf
        if m > 1:
            want[0] = np.nan
        want[:, 3] = np.nan
        np.testing.assert_array_equal(np.isnan(c), np.isnan(want))
        np.testing.assert_array_equal(np.isinf(c), np.isinf(want))
    for abits in (4, 8):
        for bbits in (4, 8):
            for out in ("f32", "bf16"):
                c = torch.zeros(m, n, dtype=TORCH[out]).cuda()
                C.costa_mx_product(1.0, keep(np.where(np.isinf(a), 1.0, a), abits), keep(b, bbits), 0.0, c)
                nan = np.isnan(c.float().cpu().numpy())
                assert nan[:, 3].all() and (m == 1 or nan[0].all())
                nan[:, 3] = False
                nan[0] = nan[0] & (m == 1)
                assert not nan.any()


def test_tiny_and_huge_magnitudes():
    """Scales at both ends of their range: products whose factors a 32-bit sum holds."""
    rng = np.random.default_rng(2)
    for m in (2, 40, 200):
        for ea, eb in ((100, -112), (-100, 90), (60, -110)):
            a, b = rng.standard_normal((m, 256)) * 2.0**ea, rng.standard_normal((130, 256)) * 2.0**eb
            for bits in (4, 8):
                q = keep(b, bits)
                vb = F.decode(*F.encode(b, bits), bits, 256)
                t = gpu(a)
                c = torch.empty(m, 130).cuda()
                C.costa_mx_product_real(1.0, "N", t, q, 0.0, c)
                check_product(c, t.cpu().to(torch.float64).numpy(), vb, 1.0, 0.0, None, "f32")
                for abits in (4, 8):
                    va = F.decode(*F.encode(a, abits), abits, 256)
                    C.costa_mx_product(1.0, keep(a, abits), q, 0.0, c)
                    check_product(c, va, vb, 1.0, 0.0, None, "f32")


def test_empty_products():
    q = keep(np.ones((5, 32)), 4)
    for m, n, k in ((0, 5, 32), (4, 0, 32), (4, 5, 0)):
        qa = C.MxMatrix.empty(8, m, k)
        qb = C.MxMatrix.empty(4, n, k) if (n, k) != (5, 32) else q
        c = torch.full((m, n), 3.0).cuda()
        C.costa_mx_product(1.0, qa, qb, 0.5, c)
        assert (c == 1.5).all()
        C.costa_mx_product_real(1.0, "N", torch.empty(m, k).cuda(), qb, 0.0, c)
        assert (c == 0.0).all()
    for shape in ((0, 5), (5, 0)):
        q, qt = C.MxMatrix.empty(4, *shape), C.MxMatrix.empty(8, *shape[::-1])
        C.costa_mx_quantize(1.0, torch.empty(shape).cuda(), q, qt)
        C.costa_mx_dequantize(1.0, q, 0.0, torch.empty(shape).cuda())


def test_same_bits_every_time_and_on_any_stream():
    """Repeated calls, calls with a workspace of the caller's, and calls on another
    stream give the same bits (no atomics in any sum)."""
    rng = np.random.default_rng(4)
    a, b = rng.standard_normal((60, 40000)), rng.standard_normal((70, 40000))
    q, t = keep(b, 8), gpu(a)
    first = torch.empty(60, 70).cuda()
    C.costa_mx_product_real(1.0, "N", t, q, 0.0, first)
    space = torch.empty(max(16, C.costa_mx_workspace(60, 70, 40000)), dtype=torch.uint8).cuda()
    side = torch.cuda.Stream()
    for k in range(4):
        c = torch.empty(60, 70).cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(side if k == 3 else torch.cuda.current_stream()):
            C.costa_mx_product_real(1.0, "N", t, q, 0.0, c, workspace=space if k == 1 else None,
                                    stream=side if k == 2 else None)
        torch.cuda.synchronize()
        assert torch.equal(c, first)
    # without a workspace the sum is not split over workgroups
    none = torch.empty(60, 70).cuda()
    C.costa_mx_product_real(1.0, "N", t, q, 0.0, none, workspace=torch.empty(0, dtype=torch.uint8).cuda())
    check_product(none, t.cpu().to(torch.float64).numpy(), F.decode(*F.encode(b, 8), 8, 40000), 1.0, 0.0, None, "f32")


def test_captured_calls():
    """One graph of a store out of a layout and the products that read it, replayed on new inputs."""
    L = C.Layout.block_cyclic(192, 320, 32, 64, 2, 2)
    bufs = [torch.randn(L.local_elems(r)).cuda() for r in range(4)]
    x = torch.randn(20, 320).cuda()
    q, qt, c, d = C.MxMatrix.empty(4, 192, 320), C.MxMatrix.empty(8, 320, 192), torch.empty(20, 192).cuda(), torch.empty(20, 320).cuda()

    def step():
        C.costa_mx_quantize_layout("f32", 1.0, L, bufs, q, qt)
        C.costa_mx_product_real(1.0, "N", x, q, 0.0, c)
        C.costa_mx_product_real(1.0, "N", c, qt, 0.0, d)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()  # uploads the layout's tables
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for k in range(4):
        x.copy_(torch.randn(20, 320))
        for b in bufs:
            b.mul_(1.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = c.clone(), d.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], c) and torch.equal(got[1], d)
    fresh = C.Layout.block_cyclic(64, 64, 32, 32, 2, 2)
    fb, fq = [torch.randn(1024).cuda() for _ in range(4)], C.MxMatrix.empty(4, 64, 64)
    back, other = torch.empty(192, 320).cuda(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(other, stream=side):
        with pytest.raises(C.CostaError) as e:
            C.costa_mx_quantize_layout("f32", 1.0, fresh, fb, fq)
        C.costa_mx_dequantize(1.0, q, 0.0, back)
    assert e.value.status == C.NOT_SUPPORTED


def test_tables_of_many_layouts():
    """More layouts than the library keeps tables of; a captured call's stay for its replays."""
    L = C.Layout.block_cyclic(100, 90, 16, 32, 2, 2)
    bufs = [torch.randn(L.local_elems(r)).cuda() for r in range(4)]
    q, want = C.MxMatrix.empty(8, 100, 90), C.MxMatrix.empty(8, 100, 90)
    C.costa_mx_quantize_layout("f32", 1.0, L, bufs, want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        C.costa_mx_quantize_layout("f32", 1.0, L, bufs, q)
    x = torch.randn(60, 70)
    for k in range(150):
        M = C.Layout.general(60, 70, [0, 1 + k % 59, 60], [0, 1 + k % 69, 70], [0, 1, 2, 0], 3, "row")
        parts = [torch.zeros(max(1, M.local_elems(r))).cuda() for r in range(3)]
        for bi, (r0, r1) in enumerate(((0, 1 + k % 59), (1 + k % 59, 60))):
            for bj, (c0, c1) in enumerate(((0, 1 + k % 69), (1 + k % 69, 70))):
                o, off, ld = C.costa_layout_block(M.handle, bi, bj)
                torch.as_strided(parts[o], (r1 - r0, c1 - c0), (ld, 1), off).copy_(x[r0:r1, c0:c1])
        m = filled(4, 60, 70)
        C.costa_mx_quantize_layout("f32", 1.0, M, parts, m)
        check_stored(m, x.numpy())
    for _ in range(3):
        q.data.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q.data, want.data) and torch.equal(q.scales, want.scales)


# ---------------------------------------------------------------------------
# gradients
# ---------------------------------------------------------------------------
def test_layer_gradients_against_formula_and_differences():
    """dX = dY W^ and dW = dY^T X^ of Y = X W^^T with X kept in 8 bits: against the
    formula, and against differences of the layer's own output (linear in X
    and W^, so a difference quotient of any step is exact up to rounding)."""
    T, K, N = 70, 130, 90
    rng = np.random.default_rng(6)
    x, w, dy = rng.standard_normal((T, K)), rng.standard_normal((N, K)) * 0.2, rng.standard_normal((T, N))
    X, W, DY = gpu(x), gpu(w), gpu(dy)
    wq, wqt, xt = C.MxMatrix.empty(4, N, K), C.MxMatrix.empty(4, K, N), C.MxMatrix.empty(8, K, T)
    C.costa_mx_quantize(1.0, W, wq, wqt)
    C.costa_mx_quantize(1.0, X, None, xt)
    dX, dW = torch.empty(T, K).cuda(), torch.ones(N, K).cuda()
    C.costa_mx_product_real(1.0, "N", DY, wqt, 0.0, dX)
    C.costa_mx_product_real(1.0, "T", DY, xt, 1.0, dW)
    f32 = lambda v: v.astype(np.float32).astype(np.float64)  # noqa: E731
    vwt = F.decode(*F.encode(w.astype(np.float32).T, 4), 4, N)  # K x N
    vxt = F.decode(*F.encode(x.astype(np.float32).T, 8), 8, T)  # K x T
    check_product(dX, f32(dy), vwt, 1.0, 0.0, None, "f32")
    check_product(dW, f32(dy).T, vxt, 1.0, 1.0, np.ones((N, K)), "f32")
    # differences: of L = <dY, X W^^T> with the same W^ (the transposed store decoded), along a random direction
    step = rng.standard_normal((T, K))
    L = lambda xx: float(np.sum(f32(dy) * (xx @ vwt)))  # noqa: E731
    slope = (L(f32(x) + step) - L(f32(x) - step)) / 2
    got = float(np.sum(dX.cpu().to(torch.float64).numpy() * step))
    assert abs(got - slope) <= 1e-5 * np.sum(np.abs(dX.cpu().numpy() * step))
    stepw = rng.standard_normal((N, K))
    Lw = lambda ww: float(np.sum(f32(dy) * (vxt.T @ ww.T)))  # noqa: E731
    slope = (Lw(w + stepw) - Lw(w - stepw)) / 2
    got = float(np.sum((dW.cpu().to(torch.float64).numpy() - 1.0) * stepw))
    assert abs(got - slope) <= 1e-5 * np.sum(np.abs(dW.cpu().numpy() * stepw))


def test_offsets_past_32_bits():
    """A stored matrix and a plain one of more than 2^32 bytes: the last rows are read and written at their own place."""
    rows, cols = 70000, 65536  # 4.6e9 bytes in 8 bits
    q = C.MxMatrix.empty(8, rows, cols)
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(3, cols, dtype=torch.bfloat16)
    x[-3:] = tail.cuda()
    C.costa_mx_quantize(1.0, x, q)
    del x
    want = F.encode(tail.float().numpy(), 8)
    np.testing.assert_array_equal(q.data[-3 * cols:].cpu().numpy().reshape(3, -1), want[0])
    np.testing.assert_array_equal(q.scales[-3 * cols // 32:].cpu().numpy().reshape(3, -1), want[1])
    one = torch.randn(2, cols, dtype=torch.bfloat16).cuda()
    c = torch.empty(2, rows, device="cuda")
    C.costa_mx_product_real(1.0, "N", one, q, 0.0, c)
    assert (c[:, :-3] == 0).all()
    check_product(c[:, -3:], one.cpu().double().numpy(), F.decode(*want, 8, cols), 1.0, 0.0, None, "f32")
    big = one.repeat(40, 1)
    c = torch.empty(80, rows, device="cuda")
    C.costa_mx_product_real(1.0, "N", big, q, 0.0, c)
    check_product(c[:, -3:], big.cpu().double().numpy(), F.decode(*want, 8, cols), 1.0, 0.0, None, "f32")


def test_example_trains():
    """The example's loss falls to what 4-bit weights leave: their rounding error is up to a
    quarter of a value (1 to 1.5 of a step of 0.5 .. and so on), so under a tenth of the first loss."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "few_bit_layer.py")
    spec = importlib.util.spec_from_file_location("few_bit_layer", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    losses = mod.train(tokens=2048, inputs=384, outputs=250, steps=8)
    assert losses[-1] < losses[0] / 10, losses
