"""The binding of the microscaled matrices without a GPU: whose memory a call
takes, and on which stream."""
import contextlib

import pytest

torch = pytest.importorskip("torch")
C = pytest.importorskip("paper_2106_06601_amd")


class Pools:
    """torch's streams and allocations as the binding asks for them: every
    allocation is noted with the stream that is current there."""

    def __init__(self, current):
        self.handle, self.taken = current, []

    def empty(self, n, dtype=None, device=None):
        self.taken.append((n, self.handle))
        return torch.zeros(n, dtype=dtype)

    @contextlib.contextmanager
    def stream(self, s):
        was, self.handle = self.handle, s
        yield
        self.handle = was


@pytest.fixture
def pools(monkeypatch):
    p = Pools(current=0x1000)
    monkeypatch.setattr(torch, "empty", p.empty)
    monkeypatch.setattr(torch.cuda, "stream", p.stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda at, **kw: at)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: type("S", (), {"cuda_stream": p.handle}))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    monkeypatch.setattr(C, "_stream", lambda s: p.handle if s is None else s)
    return p


@pytest.mark.parametrize("stream,want", [(None, 0x1000), (0x1000, 0x1000), (0x2000, 0x2000), (0, 0)])
def test_a_workspace_belongs_to_the_stream_that_uses_it(pools, stream, want):
    """A block of another stream's pool may still be read and written by work that is
    queued there; only its own stream's order makes taking it safe."""
    m, n, k = 60, 70, 40000
    need = C.costa_mx_workspace(m, n, k)
    assert need > 0
    at, size, keep = C._product_workspace(m, n, k, None, "cuda", stream)
    assert pools.taken == [(need, want)]
    assert size == need and at == keep.data_ptr()
    assert pools.handle == 0x1000


def test_a_product_without_split_takes_nothing(pools):
    assert C.costa_mx_workspace(5, 7, 1) == 0
    assert C._product_workspace(5, 7, 1, None, "cuda", 0x2000) == (None, 0, None)
    assert pools.taken == []


def test_a_buffer_for_every_rank_is_asked_for():
    """The library reads an address for each rank of the layout."""
    L = C.Layout.block_cyclic(8, 6, 2, 2, 2, 2)
    for layout in (L, L.handle):
        for bufs in ([], [1 << 20], [1 << 20] * 3):
            with pytest.raises(ValueError, match="buffers"):
                C.costa_mx_quantize_layout("f32", 1.0, layout, bufs)
        with pytest.raises(C.CostaError):  # neither Q nor QT
            C.costa_mx_quantize_layout("f32", 1.0, layout, [1 << 20] * 4)
