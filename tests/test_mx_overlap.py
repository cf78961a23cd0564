"""Which operands of a call overlap, against the sets of their bytes; on the CPU,
over the stand-in of the HIP runtime."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.spawns  # builds the stand-in

ref = ctypes.byref
COL, ROW = 0, 1
SIZE = {1: 4, 2: 2, 3: 2}  # float, bfloat16, float16
BASE = 1 << 40             # memory that nothing reads
FAR = 1 << 44


@pytest.fixture(scope="module")
def standin():
    import standin
    return standin.load()


def bytes_of(m):
    """Addresses of a matrix's bytes."""
    lines, line = (m.cols, m.rows) if m.order == COL else (m.rows, m.cols)
    es = SIZE[m.type]
    at = m.data + es * (np.arange(lines)[:, None] * m.ld + np.arange(line)[None, :])
    return (at[..., None] + np.arange(es)).reshape(-1)


def status_of(S, a, c, b=None, workspace=(None, 0)):
    b = b or S.C.CostaMx(0, c.cols, a.cols, FAR, 2 * FAR)
    st = S.C._lib.costa_mx_product_real(1.0, 0, ref(a), ref(b), 0.0, ref(c), *workspace, None)
    S.faults()  # (kernels that the stand-in does not run)
    S.lib.standin_tile_launches(None, 0)
    return st


def test_slices_of_one_buffer_side_by_side(standin):
    """Columns of a row-major buffer are read, others are written."""
    S = standin
    M = S.C.CostaMatrix
    a = M(1, ROW, 100, 128, 256, BASE)
    for at in (128, 160, 192):
        assert status_of(S, a, M(1, ROW, 100, 64, 256, BASE + 4 * at)) == S.C.SUCCESS, S.C.costa_last_error()
    assert status_of(S, a, M(1, ROW, 100, 64, 256, BASE + 4 * 127)) == S.C.INVALID_VALUE
    # the columns past the row's end are the next row's first
    assert status_of(S, a, M(1, ROW, 99, 64, 256, BASE + 4 * 193)) == S.C.SHAPE_MISMATCH
    assert status_of(S, M(1, ROW, 99, 128, 256, BASE), M(1, ROW, 99, 64, 256, BASE + 4 * 193)) == S.C.INVALID_VALUE
    assert status_of(S, M(1, ROW, 1, 128, 256, BASE), M(1, ROW, 1, 64, 256, BASE + 4 * 193)) == S.C.SUCCESS
    # a stored matrix, and a workspace, between the rows of C
    c = M(1, ROW, 5, 3, 1024, BASE)
    few = M(1, ROW, 5, 64, 64, 3 * FAR)
    for gap, want in ((16, S.C.SUCCESS), (0, S.C.INVALID_VALUE), (4096 - 384, S.C.SUCCESS), (4096 - 368, S.C.INVALID_VALUE)):
        assert status_of(S, few, c, S.C.CostaMx(0, 3, 64, BASE + 4096 + gap, FAR)) == want
        assert status_of(S, few, c, workspace=(BASE + 8192 + gap, 384)) == want


def test_random_strides_and_places(standin):
    S, rng, seen = standin, np.random.default_rng(21), {False: 0, True: 0}
    for _ in range(3000):
        rows, k, n = (int(rng.integers(1, 12)) for _ in range(3))
        ms = []
        for cols in (k, n):
            t, order = int(rng.choice([1, 2, 3])), int(rng.choice([COL, ROW]))
            ld = (rows if order == COL else cols) + int(rng.choice([0, 1, 5, 17, 40]))
            ms.append(S.C.CostaMatrix(t, order, rows, cols, ld, BASE + SIZE[t] * int(rng.integers(0, 80))))
        a, c = ms
        meet = np.intersect1d(bytes_of(a), bytes_of(c)).size > 0
        seen[meet] += 1
        assert status_of(S, a, c) == (S.C.INVALID_VALUE if meet else S.C.SUCCESS), \
            [(m.type, m.order, m.rows, m.cols, m.ld, m.data - BASE) for m in ms]
    assert min(seen.values()) > 300


def test_long_lines_far_apart(standin):
    """Strides and numbers of lines whose products pass 64 bits on the way."""
    S = standin
    M, m = S.C.CostaMatrix, 2**31 - 1
    p, q = 2**25 + 9, 2**25 + 8  # (a's lines move against c's by one element a line)
    a = M(1, ROW, 1 << 20, 8, p, BASE)
    for j in (0, 5, 1000, (1 << 20) - 2):
        c = M(1, ROW, 1 << 20, 8, q, BASE + 4 * (8 + j))  # side by side at first; line j + 1 of a meets line j + 1 of c
        assert status_of(S, a, c) == S.C.INVALID_VALUE
    c = M(1, ROW, 1 << 20, 8, q, BASE + 4 * (8 + (1 << 20) - 1))
    assert status_of(S, a, c) == S.C.SUCCESS
    big = 2**58 // m // 8 * 8
    a, b = M(1, ROW, m, 8, big, BASE), S.C.CostaMx(0, 4, 8, FAR + 4096, 2 * FAR + 4096)  # (between two rows)
    assert status_of(S, a, M(1, ROW, m, 4, big, BASE + 32), b) == S.C.SUCCESS, S.C.costa_last_error()
    assert status_of(S, a, M(1, ROW, m, 4, big, BASE + 28), b) == S.C.INVALID_VALUE
    assert S.C.costa_last_error() == "C overlaps A"
    b.data = FAR  # where a row of C begins
    assert status_of(S, a, M(1, ROW, m, 4, big, BASE + 32), b) == S.C.INVALID_VALUE
    assert S.C.costa_last_error() == "C overlaps B"


def test_every_pair_of_operands_is_checked(standin):
    """Each buffer of a call laid over each other one that the call may not share it with."""
    S = standin
    C, M, bad = S.C, S.C.CostaMatrix, S.C.INVALID_VALUE

    def mx(fmt, rows, cols, at):
        return C.CostaMx(fmt, rows, cols, at, at + (1 << 20))

    def message(what, status):
        S.faults()
        S.lib.standin_tile_launches(None, 0)
        assert status == bad and "overlap" in C.costa_last_error(), (what, status, C.costa_last_error())

    # quantise: B, Q and QT, each with two buffers of the few-bit ones
    for what in ("B Q.data", "B Q.scales", "B QT.data", "B QT.scales", "Q.data QT.data", "Q.data QT.scales",
                 "Q.scales QT.data", "Q.scales QT.scales", "Q.data Q.scales", "QT.data QT.scales"):
        held = {"B": M(1, ROW, 40, 70, 70, BASE), "Q": mx(0, 40, 70, 2 * BASE), "QT": mx(1, 70, 40, 3 * BASE)}
        assert C._lib.costa_mx_quantize(1.0, *map(ref, held.values()), None) == C.SUCCESS
        one, two = what.split()
        at = held["B"].data if one == "B" else getattr(held[one.split(".")[0]], one.split(".")[1])
        name, field = two.split(".")
        setattr(held[name], field, at + 16)
        message(what, C._lib.costa_mx_quantize(1.0, *map(ref, held.values()), None))
    for field in ("data", "scales"):
        q = mx(1, 40, 70, 2 * BASE)
        assert C._lib.costa_mx_dequantize(1.0, ref(q), 0.0, ref(M(1, ROW, 40, 70, 70, BASE)), None) == C.SUCCESS
        message(field, C._lib.costa_mx_dequantize(1.0, ref(q), 0.0, ref(M(1, ROW, 40, 70, 70, getattr(q, field))), None))
    # products: the workspace
    a, b, few, c = M(1, ROW, 5, 64, 64, BASE), mx(0, 9, 64, 2 * BASE), mx(1, 5, 64, 3 * BASE), M(1, ROW, 5, 9, 9, 4 * BASE)
    for at in (5 * BASE, a.data, b.data, b.scales, c.data):
        st = C._lib.costa_mx_product_real(1.0, 0, ref(a), ref(b), 0.0, ref(c), at, 64, None)
        if at == 5 * BASE:
            assert st == C.SUCCESS
        else:
            message(at, st)
    for at in (few.data, few.scales):
        message(at, C._lib.costa_mx_product(1.0, ref(few), ref(b), 0.0, ref(c), at, 64, None))
    S.faults()


def test_a_row_of_a_store_in_the_gaps_of_a_matrix(standin):
    """What lies between a strided matrix's lines is not the matrix's."""
    S = standin
    C = S.C
    b = C.CostaMatrix(1, ROW, 1, 40, 4096, BASE)
    for rows, at, want in ((1, 160, C.SUCCESS), (1, 144, C.INVALID_VALUE), (2, 160, C.SUCCESS), (2, 16384 - 112, C.INVALID_VALUE)):
        b.rows = rows
        q = C.CostaMx(0, rows, 40, BASE + at, FAR)
        assert C._lib.costa_mx_quantize(1.0, ref(b), ref(q), None, None) == want, (rows, at)
    S.faults()
