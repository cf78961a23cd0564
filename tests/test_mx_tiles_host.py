"""The launches of a product's tiles, on the CPU: the library's host code over the
stand-in of the HIP runtime, and the kernels' order of tiles."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.spawns  # builds the stand-in

ROW, F32, BF16 = 1, 1, 2
AT = 1 << 50  # an address that nothing reads


@pytest.fixture(scope="module")
def standin():
    import standin
    S = standin.load()
    u32 = ctypes.c_uint32
    S.lib.standin_tile_launches.argtypes = [ctypes.c_void_p, ctypes.c_int]
    S.lib.standin_xcd_tiles.argtypes = [u32] * 6 + [ctypes.c_void_p] * 2
    S.lib.standin_xcd_tiles.restype = None
    return S


def launches(S):
    out = np.zeros((64, 5), np.uint32)
    return out[:S.lib.standin_tile_launches(out.ctypes.data, 64)].tolist()


def product(S, m, n, k, few_bit=None):
    """The status of a product with no workspace of m x k bfloat16 (or 4-bit) by n x k in 4 bits."""
    C, ref = S.C, ctypes.byref
    b = C.CostaMx(0, n, k, AT + (1 << 47), AT + (1 << 48))
    c = C.CostaMatrix(F32, ROW, m, n, n, AT + (1 << 49))
    if few_bit:
        a = C.CostaMx(0, m, k, AT, AT + (1 << 46))
        return C._lib.costa_mx_product(1.0, ref(a), ref(b), 0.0, ref(c), None, 0, None)
    a = C.CostaMatrix(BF16, ROW, m, k, k, AT)
    return C._lib.costa_mx_product_real(1.0, 0, ref(a), ref(b), 0.0, ref(c), None, 0, None)


@pytest.mark.parametrize("few_bit", [False, True], ids=["real", "few_bit"])
@pytest.mark.parametrize("m,n,k", [(600_000_000, 1, 16), (600_000_000, 65, 256), (2**31 - 1, 3, 8), (65, 600_000_000, 256),
                                   (2**31 - 1, 129, 64), (1 << 29, 64, 8), ((1 << 29) + 1, 64, 8), (300, 300, 300)])
def test_thin_products_of_every_length_are_launched(standin, m, n, k, few_bit):
    """Every tile of C is in one launch, and a launch holds no more than a grid does."""
    S = standin
    launches(S)
    assert product(S, m, n, k, few_bit) == S.C.SUCCESS, S.C.costa_last_error()
    S.check()
    got, at = launches(S), 0
    assert got
    for nm, nn, first, tiles, splits in got:
        assert (nm, nn) == tuple(got[0][:2]) and splits == 1
        assert first == at and 0 < tiles * 512 < 2**32
        at += tiles
    assert at == nm * nn
    assert any(-(-m // bm) == nm and -(-n // bn) == nn for bm, bn in ((256, 256), (128, 256), (128, 128), (128, 64)))


def test_products_past_all_memory_are_not_supported(standin):
    S = standin
    assert product(S, 2**31 - 1, 2**31 - 1, 8) == S.C.NOT_SUPPORTED
    assert not launches(S)


@pytest.mark.parametrize("nm,nn", [(1, 1), (3, 2), (8, 8), (9, 5), (17, 33), (1, 100), (100, 1), (31, 7)])
@pytest.mark.parametrize("slices", [1, 3])
def test_every_tile_is_one_workgroups(standin, nm, nn, slices):
    seen, size = np.zeros((nm, nn), int), max(8, -(-nm * nn // slices) // 8 * 8)
    for first in range(0, nm * nn, size):
        n = min(size, nm * nn - first)
        tm, tn = np.zeros(n, np.uint32), np.zeros(n, np.uint32)
        standin.lib.standin_xcd_tiles(nm, nn, first, n, 0, n, tm.ctypes.data, tn.ctypes.data)
        np.add.at(seen, (tm, tn), 1)
    assert (seen == 1).all()


@pytest.mark.parametrize("nm,nn", [(2**24, 1), (2**24, 3), (1, 2**25), (5, 2**25), (2**24, 127), (2**12, 2**19 - 1)])
def test_tiles_far_into_a_long_matrix(standin, nm, nn):
    """32-bit positions do not wrap: the last slice's workgroups have the tiles that 64 bits give."""
    total, size, seen = nm * nn, 1 << 22, set()
    assert total < 2**31
    first = (total - 1) // size * size
    n = total - first
    for b0 in (0, max(0, n - 5000)):
        count = min(5000, n)
        tm, tn = np.zeros(count, np.uint32), np.zeros(count, np.uint32)
        standin.lib.standin_xcd_tiles(nm, nn, first, n, b0, count, tm.ctypes.data, tn.ctypes.data)
        b = np.arange(b0, b0 + count, dtype=object)
        t = [first + (x % 8) * (n // 8) + min(x % 8, n % 8) + x // 8 for x in b]
        group = [x // (8 * nn) for x in t]
        rows = [min(8, nm - 8 * g) for g in group]
        rest = [x - 8 * nn * g for x, g in zip(t, group)]
        assert tm.tolist() == [8 * g + r % w for g, r, w in zip(group, rest, rows)]
        assert tn.tolist() == [r // w for r, w in zip(rest, rows)]
        assert (tm < nm).all() and (tn < nn).all()
