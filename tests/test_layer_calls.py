"""The calls around products on the CPU, as far as their launches: the library's host code over the
stand-in of the HIP runtime (kernels are named and not run)."""
import ctypes
import itertools

import pytest

pytestmark = pytest.mark.spawns  # builds the stand-in

F32, BF16, F16 = 1, 2, 3
ROW = 1
ROOM = 1 << 40  # bytes of workspace
ref = lambda a: None if a is None else ctypes.byref(a)  # noqa: E731
at = lambda k: k << 56  # noqa: E731  (addresses that nothing reads)


@pytest.fixture(scope="module")
def S():
    import standin
    S = standin.load()
    S.lib.standin_tile_launches.argtypes = [ctypes.c_void_p, ctypes.c_int]
    S.faults(), S.lib.standin_tile_launches(None, 0)
    return S


class Calls:
    """Each call with operands of given sizes; `seen` has what the last one launched."""

    def __init__(self, S, bits=8):
        self.S, self.C, self.fmt = S, S.C, S.C.MX_FORMATS[bits]

    def M(self, rows, cols, where, type):
        return self.C.CostaMatrix(type, ROW, rows, cols, max(cols, 1), at(where))

    def Q(self, rows, cols, where, fmt=None):
        return self.C.CostaMx(self.fmt if fmt is None else fmt, rows, cols, at(where), at(where) + (1 << 55))

    def done(self, status):
        said = self.S.faults().decode()
        tiles = self.S.lib.standin_tile_launches(None, 0)
        self.empty = [s for s in said.splitlines() if "no workgroups" in s]
        self.seen = [s.split(": ")[1] for s in said.splitlines() if "does not run" in s] + ["tiles_bf16"] * tiles
        return status

    def loss(self, m, n, k, type, room=ROOM):
        return self.done(self.C._lib.costa_mx_loss(1.0, ref(self.M(m, k, 1, type)), ref(self.Q(n, k, 2)), at(3), at(4), at(5),
                                                   at(20), room, None))

    def loss_backward(self, m, n, k, type, out, x=True, w=True, room=ROOM):
        return self.done(self.C._lib.costa_mx_loss_backward(
            1.0, ref(self.M(m, k, 1, type)), ref(self.Q(n, k, 2)), at(3), at(5), None, ref(self.Q(k, n, 6) if x else None),
            ref(self.M(m, k, 7, out) if x else None), ref(self.Q(k, m, 8, 1) if w else None), 0.5,
            ref(self.M(n, k, 9, out) if w else None), at(20), room, None))

    def adapted(self, m, n, k, count, rank, type, room=ROOM, V=True):
        A, B = self.M(count * rank, k, 3, type), self.M(count * rank, n, 4, type)
        a = self.C.CostaMxAdapters(count, rank, ctypes.pointer(A), ctypes.pointer(B), None, None)
        return self.done(self.C._lib.costa_mx_product_adapted(
            1.0, ref(self.M(m, k, 1, type)), ref(self.Q(n, k, 2)), ref(a), at(5), 0.5, ref(self.M(m, n, 6, type)),
            ref(self.M(m, rank, 7, F32) if V else None), at(20), room, None))

    def gradient(self, m, n, count, rank, type, room=ROOM):
        a = self.C.CostaMxAdapters(count, rank, None, None, None, None)
        return self.done(self.C._lib.costa_mx_adapter_gradient(
            ref(a), at(5), ref(self.M(m, rank, 1, F32)), ref(self.M(m, n, 2, type)), 0.5, ref(self.M(count * rank, n, 6, type)),
            at(20), room, None))

    def norm(self, m, n, type):
        return self.done(self.C._lib.costa_mx_norm(1e-5, ref(self.M(m, n, 1, type)), None, None, None, ref(self.M(m, n, 2, type)),
                                                   ref(self.Q(m, n, 3)), at(4), None))

    def norm_backward(self, m, n, type, room=ROOM):
        return self.done(self.C._lib.costa_mx_norm_backward(
            ref(self.M(m, n, 1, type)), ref(self.M(m, n, 2, type)), None, at(3), None, ref(self.M(m, n, 4, type)),
            ref(self.M(1, n, 5, F32)), at(20), room, None))


SIZES = [0, 1, 5, 8, 17, 64, 65, 128, 1000, 4096, 70000]


@pytest.mark.parametrize("type", [F32, BF16, F16])
def test_no_launch_is_empty(S, type):
    """Sizes of nothing among others: a call succeeds and launches no grid without workgroups, which HIP refuses."""
    c = Calls(S)

    def fine(status):
        assert status == c.C.SUCCESS, c.C.costa_last_error()
        assert not c.empty

    for m, n, k in itertools.product(SIZES, SIZES, SIZES):
        if m * n * k > 1 << 36:
            continue
        fine(c.loss(m, n, k, type))
        for out, x, w in ((type, True, True), (BF16, True, False), (F32, False, True)):
            fine(c.loss_backward(m, n, k, type, out, x, w))
        for count, rank in ((0, 3), (3, 0), (2, 20)):
            fine(c.adapted(m, n, k, count, rank, type))
    for m, n in itertools.product(SIZES, SIZES):
        fine(c.norm(m, n, type))
        fine(c.norm_backward(m, n, type))
        for count, rank in ((0, 3), (3, 0), (2, 20), (40, 130)):
            fine(c.gradient(m, n, count, rank, type))
            fine(c.gradient(m, n, count, rank, type, room=0))


def test_a_loss_over_no_words(S):
    """Nothing but the join of no statistics, for products of every kind."""
    for m, k, type in itertools.product((1, 64, 65, 100, 4096), (1, 8, 64, 128, 129, 5000), (F32, BF16, F16)):
        c = Calls(S)
        assert c.loss(m, 0, k, type) == c.C.SUCCESS
        assert len(c.seen) == 1 and "loss_join" in c.seen[0], (m, k, type, c.seen)


@pytest.mark.parametrize("m,n,k", [(512, 8200, 1030), (260, 2500, 520), (4096, 65536, 4096), (2048, 20000, 2048), (300, 8201, 1024),
                                   (70, 500, 100), (64, 8200, 1030)])
def test_the_workspace_does_not_choose_the_precision(S, m, n, k):
    """Whether G is in bfloat16 (with dW: its products' factor is in device memory) is the same for every room."""
    c = Calls(S, 4)
    least, most = c.C.costa_mx_loss_workspace(m, n, k, True)
    for x in (True, False):
        kinds = set()
        for room in (least, least + (most - least) // 30, (least + most) // 2, most, ROOM):
            assert c.loss_backward(m, n, k, BF16, BF16, x, True, room) == c.C.SUCCESS, c.C.costa_last_error()
            kinds.add(any("tiles_loss_dw" in s for s in c.seen))
        assert len(kinds) == 1


@pytest.mark.parametrize("bits", [4, 8])
def test_an_adapted_product_asks_for_what_it_uses(S, bits):
    """The least workspace holds v and either 256 rows of sums or v spread, and calls of every type get by with it: v is
    spread by products of 1024 rows and more alone."""
    c, up16 = Calls(S, bits), lambda x: -(-x // 16) * 16
    spreads = 0
    for m, n, k, rank in itertools.product((1, 17, 300, 1000, 1023, 1024, 4096, 20000), (1, 130, 1999, 8192), (1, 64, 2501, 8192), (1, 16, 33, 256)):
        least, most = c.C.costa_mx_adapted_workspace(m, n, k, rank)
        v, sums, spread = up16(4 * m * rank), 4 * min(m, 256) * n, -(-m // 16) * -(-rank // 32) * 3 * 1024
        assert least in ((v + sums,) if m < 1024 else (v + sums, v + spread, v + max(sums, spread))) and least <= most
        for type in (F32, BF16, F16):
            assert c.adapted(m, n, k, 3, rank, type, room=least, V=False) == c.C.SUCCESS, c.C.costa_last_error()
            spreads += any("adapter_spread" in s for s in c.seen)
            assert least >= v + (spread if any("adapter_spread" in s for s in c.seen) else sums)
            assert c.adapted(m, n, k, 3, rank, type, room=least - 1, V=False) == c.C.INVALID_VALUE
    assert spreads


@pytest.mark.parametrize("m,n,k,rank", [(900, 2000, 64, 4), (1000, 4099, 300, 4), (700, 3001, 129, 33), (521, 2501, 1030, 100)])
def test_slices_of_rows_are_products_of_their_own(S, m, n, k, rank):
    """Each with operands that begin at its first row, one after another over all of them."""
    import numpy as np
    c, out = Calls(S, 4), np.zeros((64, 10), np.int64)
    least, most = c.C.costa_mx_adapted_workspace(m, n, k, rank)
    for type in (F32, BF16, F16):
        for room in (least, least + 400 * n, most):
            A, B = c.M(3 * rank, k, 3, type), c.M(3 * rank, n, 4, type)
            a = c.C.CostaMxAdapters(3, rank, ctypes.pointer(A), ctypes.pointer(B), None, None)
            st = c.C._lib.costa_mx_product_adapted(1.0, ref(c.M(m, k, 1, type)), ref(c.Q(n, k, 2)), ref(a), at(5), 0.0,
                                                   ref(c.M(m, n, 6, type)), None, at(20), room, None)
            assert st == c.C.SUCCESS
            S.faults()
            got = out[:S.lib.standin_tile_launches(out.ctypes.data, len(out))].tolist()
            per, row, es = (room - -(-4 * m * rank // 16) * 16) // (4 * n), 0, 4 if type == F32 else 2
            for rows, cols, _, _, _, _, x, _, _, to in got:
                assert (cols, x, to) == (n, at(1) + row * k * es, at(20) + -(-4 * m * rank // 16) * 16)
                assert rows == min(per, m - row)
                row += rows
            # (up to 64 rows at the end are no tiles' but the kernels' for few rows)
            assert row == m or (row == m // per * per and m - row <= 64)
            assert (row < m or len(got) > 1) == (per < m)


LONG = [(2**31 - 1, 1, 8), (2**31 - 1, 40, 64), (1, 2**31 - 1, 64), (64, 2**28, 300), (300, 2**28, 64), (5000, 2**30, 8), (2**30, 3, 256),
        (100, 100, 2**31 - 1), (2**28, 1000, 100), (4096, 2**28, 4096), (2**24, 2**24, 8)]


@pytest.mark.parametrize("m,n,k", LONG)
@pytest.mark.parametrize("type", [F32, BF16])
def test_launches_of_long_operands_hold_in_a_grid(S, m, n, k, type):
    """(Workspaces of whole TiB for row sums and statistics: of what the calls ask for.)"""
    c = Calls(S)

    def fine(status):
        assert status == c.C.SUCCESS, c.C.costa_last_error()

    need = lambda name, *sizes: c.C._two_sizes(name, *sizes)[0]  # noqa: E731
    if m * k < 1 << 42 and m * n < 1 << 46:  # (a backward pass goes by pieces of the vocabulary, some million of them for the longest)
        fine(c.loss(m, n, k, type, need("costa_mx_loss_workspace", m, n, k, 0)))
    for count, rank in ((2, 20), (3000, 256)):
        if count * rank * max(n, k) < 1 << 46 and m * n < 1 << 42:
            fine(c.adapted(m, n, k, count, rank, type, need("costa_mx_adapted_workspace", m, n, k, rank)))
            fine(c.adapted(m, n, k, count, rank, type, c.C._two_sizes("costa_mx_adapted_workspace", m, n, k, rank)[1]))
            fine(c.gradient(m, n, count, rank, type))
    fine(c.norm(m, n, type))
    fine(c.norm_backward(m, n, type))
