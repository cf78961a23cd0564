"""The rule that picks a product's kernel, on the CPU."""
import ctypes
import itertools

import numpy as np
import pytest

import mx_wide as W

pytestmark = pytest.mark.spawns  # builds the stand-in

FEW_ROWS, TILES_BF16, TILES_SCALED, THIN = range(4)


@pytest.fixture(scope="module")
def plan():
    import standin
    f = standin.load().lib.standin_plan
    i64 = ctypes.c_int64
    f.argtypes, f.restype = [ctypes.c_int] * 3 + [i64] * 3 + [ctypes.c_void_p], None

    def call(src, op, bbits, m, n, k):
        out = np.zeros(4, np.int32)
        f(W.SOURCES[src], int(op == "N"), bbits, m, n, k, out.ctypes.data)
        return tuple(out.tolist())

    return call


def test_the_wide_sizes_reach_every_wide_kernel(plan):
    """Those that the large products run on: each type, either direction, with and without
    a last lane that lacks rows, split and not."""
    seen = set()
    for (m, n, k), (src, op), bbits in itertools.product(
            W.SHAPES, [("mx4", "N"), ("mx8", "N")] + [(s, o) for s in ("bf16", "f16", "f32") for o in "NT"], (4, 8)):
        seen.add(W.kernel(src, op, bbits, m, plan(src, op, bbits, m, n, k)))
    want = set()
    for split, bbits in itertools.product((False, True), (4, 8)):
        want.add(("mx4", bbits, TILES_SCALED if bbits == 4 else TILES_BF16, 256, 256, False, False, split))
        want.add(("mx8", bbits, TILES_BF16, 256, 256, False, False, split))
        for src in ("bf16", "f16", "f32"):
            bm = 256 if W.PARTS[src] == 1 else 128
            want |= {(src, bbits, TILES_BF16, bm, 256, turned, lacks, split)
                     for turned, lacks in ((False, False), (True, False), (True, True))}
    assert want <= seen, sorted(want - seen)


SIZES = [1, 2, 7, 8, 31, 64, 65, 100, 128, 129, 257, 1000, 4096, 70000, 2**24, 2**24 + 1, 2**31 - 1]


@pytest.mark.parametrize("src", list(W.SOURCES))
def test_plans_are_of_tiles_that_the_kernels_have(plan, src):
    for m, n, k, op, bbits in itertools.product(SIZES, SIZES, SIZES, "NT", (4, 8)):
        if op == "T" and src in ("mx4", "mx8"):
            continue
        variant, bm, bn, splits = p = plan(src, op, bbits, m, n, k)
        at = (src, op, bbits, m, n, k, p)
        assert 1 <= splits <= 256, at
        assert splits == 1 or splits * m * n * 4 <= 256 << 20, at
        if variant == THIN:
            assert k < 8 and splits == 1 and W.SOURCES[src] >= 2, at
        elif variant == FEW_ROWS:
            assert m <= 64 and m <= bm and bm in (16, 32, 64) and bn in (16, 32) and op == "N", at
            assert splits <= max(1, k * bbits // 1024), at  # a piece for every wave at least
        elif variant == TILES_SCALED:
            assert src == "mx4" and bbits == 4 and (bm, bn) in ((256, 256), (128, 128)) and k <= 2**24, at
            assert splits <= -(-k // 256), at
        else:
            assert (bm, bn) in ((256 if W.PARTS[src] == 1 else 128, 256), (128, 128), (128, 64)), at
            assert splits <= -(-k // 64), at
