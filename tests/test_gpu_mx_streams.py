"""Products on a stream of the caller's that is not torch's current one."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2106_06601_amd as C  # noqa: E402

pytestmark = pytest.mark.gpu


def keep(x, bits):
    q = C.MxMatrix.empty(bits, *x.shape)
    C.costa_mx_quantize(1.0, x, q)
    return q


def test_a_split_product_beside_work_of_the_current_stream():
    """The current stream has work queued on a block that its owner has given back;
    a product on another stream takes its parts' memory elsewhere."""
    m, n, k = 60, 70, 40000
    need = C.costa_mx_workspace(m, n, k)
    assert need > 0
    a, q = torch.randn(m, k, device="cuda"), keep(torch.randn(n, k, device="cuda"), 8)
    want, c = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    C.costa_mx_product_real(1.0, "N", a, q, 0.0, want)
    side = torch.cuda.Stream()
    for _ in range(4):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        busy, block = torch.zeros(1 << 26, device="cuda"), torch.empty(need, dtype=torch.uint8, device="cuda")
        at, total = block.data_ptr(), torch.zeros((), device="cuda")
        c.zero_()
        side.wait_stream(torch.cuda.current_stream())
        for r in range(20):
            busy.add_(1.0)
        block.fill_(1)
        total += block.sum(dtype=torch.float32)
        del block  # (free for the current stream, whose kernels still use it)
        C.costa_mx_product_real(1.0, "N", a, q, 0.0, c, stream=side)
        again = torch.empty(need, dtype=torch.uint8, device="cuda")
        assert again.data_ptr() == at  # the product has not taken it
        torch.cuda.synchronize()
        assert torch.equal(c, want)
        assert int(total) == need
