"""The launches of a product's tiles, on the CPU: the library's host code over the
stand-in of the HIP runtime."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.spawns  # builds the stand-in

ROW, COL, F32, BF16 = 1, 0, 1, 2
A, B, SCALES, OUT = (k << 48 for k in (1, 4, 6, 8))  # addresses that nothing reads


@pytest.fixture(scope="module")
def standin():
    import standin
    S = standin.load()
    S.lib.standin_tile_launches.argtypes = [ctypes.c_void_p, ctypes.c_int]
    return S


def launches(S):
    out = np.zeros((1024, 10), np.int64)
    return out[:S.lib.standin_tile_launches(out.ctypes.data, len(out))].tolist()


def product(S, m, n, k, kind, order=ROW):
    """The status of a product with no workspace of an m x k matrix by n x k in 4 bits, and the
    bytes between rows of A and of C, and between columns of C."""
    C, ref = S.C, ctypes.byref
    b = C.CostaMx(0, n, k, B, SCALES)
    c = C.CostaMatrix(F32, order, m, n, n if order == ROW else m, OUT)
    rs, cs = (4 * n, 4) if order == ROW else (4, 4 * m)
    if kind == "few_bit":
        a = C.CostaMx(0, m, k, A, A + (1 << 47))
        return C._lib.costa_mx_product(1.0, ref(a), ref(b), 0.0, ref(c), None, 0, None), -(-k // 256) * 128, rs, cs
    turned = kind == "turned"
    a = C.CostaMatrix(BF16, ROW, *((k, m, m) if turned else (m, k, k)), A)
    st = C._lib.costa_mx_product_real(1.0, int(turned), ref(a), ref(b), 0.0, ref(c), None, 0, None)
    return st, 2 if turned else 2 * k, rs, cs


@pytest.mark.parametrize("kind", ["real", "turned", "few_bit"])
@pytest.mark.parametrize("m,n,k", [(600_000_000, 1, 16), (600_000_000, 65, 256), (2**31 - 1, 3, 8), (65, 600_000_000, 256),
                                   (2**31 - 1, 129, 64), (1 << 29, 64, 8), ((1 << 29) + 1, 64, 8), (300, 300, 300)])
@pytest.mark.parametrize("order", [ROW, COL], ids=["row", "col"])
def test_thin_products_of_every_length_are_launched(standin, m, n, k, kind, order):
    """Every element of C is one launch's, whose operands begin where its rows and columns do,
    and a launch holds no more than a grid does."""
    S = standin
    launches(S)
    status, a_row, rs, cs = product(S, m, n, k, kind, order)
    assert status == S.C.SUCCESS, S.C.costa_last_error()
    S.check()
    got = launches(S)
    assert got
    b_row, b_scales, i, j = -(-k // 256) * 128, -(-k // 256) * 8, 0, 0
    tiles = {(256, 256), (128, 256), (128, 128), (128, 64)}
    for gm, gn, nm, nn, count, splits, a, b, s, c in got:
        assert splits == 1 and count == nm * nn and 0 < count * 512 < 2**32
        tiles = {(bm, bn) for bm, bn in tiles if -(-gm // bm) == nm and -(-gn // bn) == nn}
        assert (a, b, s, c) == (A + i * a_row, B + j * b_row, SCALES + j * b_scales, OUT + i * rs + j * cs)
        j += gn  # (columns first)
        if j == n:
            i, j = i + gm, 0
        else:
            assert gn % 256 == 0
        assert i == m or j or gm % 256 == 0
    assert (i, j) == (m, 0) and tiles


def test_products_past_all_memory_are_not_supported(standin):
    S = standin
    launches(S)
    assert product(S, 2**31 - 1, 2**31 - 1, 8, "real")[0] == S.C.NOT_SUPPORTED
    assert not launches(S)
