"""The device tables of layouts that the quantise calls keep, on the CPU: the
library's host code over the stand-in of the HIP runtime."""
import ctypes
import threading

import numpy as np
import pytest

pytestmark = pytest.mark.spawns  # builds the stand-in

KEPT = 64  # layouts whose tables the library keeps


@pytest.fixture(scope="module")
def standin():
    import standin
    S = standin.load()
    S.lib.standin_before_launch.argtypes = [ctypes.c_void_p]
    return S


class Store:
    """Quantise calls of one layout in 2 x 2 blocks over three ranks."""

    def __init__(self, S, k):
        self.S, C = S, S.C
        self.L = C.Layout.general(60, 70, [0, 1 + k % 59, 60], [0, 1 + k % 69, 70], [0, 1, 2, 0], 3, "row")
        self.bufs = [np.zeros(max(1, self.L.local_elems(r)), np.float32) for r in range(3)]
        size = [(n + 15) // 16 * 16 + 16 for n in C.costa_mx_sizes(4, 60, 70)]
        self.out = [np.zeros(n, np.uint8) for n in size]
        up = [(a.ctypes.data + 15) // 16 * 16 for a in self.out]
        self.q = C.CostaMx(0, 60, 70, *up)

    def run(self, stream=None):
        at = (ctypes.c_void_p * 3)(*[b.ctypes.data for b in self.bufs])
        status = self.S.C._lib.costa_mx_quantize_layout(1, 1.0, self.L.handle, at, ctypes.byref(self.q), None, stream)
        assert status == 0, self.S.C.costa_last_error()


def test_tables_stay_until_the_call_that_looked_them_up_is_enqueued(standin):
    """Just before one thread's call launches its kernel, another thread makes calls of
    as many new layouts as start the tables over."""
    S = standin
    S.C.costa_finalize()
    stores = [Store(S, k) for k in range(KEPT)]
    for s in stores:
        s.run()
    S.run(None)
    S.check()
    others = [Store(S, k) for k in range(100, 103)]
    failed = []

    def many():
        try:
            for s in others:
                s.run()
        except BaseException as e:  # noqa: BLE001
            failed.append(e)

    t = threading.Thread(target=many)

    @ctypes.CFUNCTYPE(None)
    def meanwhile():
        t.start()
        t.join(1.0)  # (a call that waits for this one goes on afterwards)

    S.lib.standin_before_launch(ctypes.cast(meanwhile, ctypes.c_void_p))
    stores[0].run()
    t.join()
    assert not failed
    S.run(None)
    S.check()


def test_tables_start_over_past_their_number(standin):
    S = standin
    S.C.costa_finalize()
    for k in range(3 * KEPT):
        s = Store(S, k)
        s.run()
        s.run()
    S.run(None)
    S.check()
    S.C.costa_finalize()
