"""Products of microscaled matrices past a launch's size."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2106_06601_amd as C  # noqa: E402
import mx_formula as F  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("left", ["bf16", "mx4"])
def test_more_tiles_than_a_launch_has(left):
    """2^22 tiles of 128 rows, and some rows more: those on either side of the slices'
    edge and the last ones are where they belong, all others zero."""
    m, n, k = (1 << 29) + 300, 3, 16
    rng = np.random.default_rng(12)
    rows = np.array([0, 1, (1 << 29) - 1, 1 << 29, (1 << 29) + 1, m - 2, m - 1])
    a = torch.from_numpy(rng.standard_normal((len(rows), k))).to(torch.bfloat16)
    b = rng.standard_normal((n, k)).astype(np.float32)
    q = C.MxMatrix.empty(4, n, k)
    C.costa_mx_quantize(1.0, torch.from_numpy(b).cuda(), q)
    vb = F.decode(*F.encode(b, 4), 4, k)
    c = torch.full((m, n), 3.0, dtype=torch.bfloat16, device="cuda")
    if left == "bf16":
        va = a.double().numpy()
        x = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
        x[torch.from_numpy(rows).cuda()] = a.cuda()
        C.costa_mx_product_real(1.0, "N", x, q, 0.0, c)
    else:
        codes, scales = F.encode(a.float().numpy(), 4)
        va = F.decode(codes, scales, 4, k)
        x = C.MxMatrix(4, m, k, torch.zeros(m, codes.shape[1], dtype=torch.uint8, device="cuda"),
                       torch.zeros(m, scales.shape[1], dtype=torch.uint8, device="cuda"))
        at = torch.from_numpy(rows).cuda()
        x.data[at], x.scales[at] = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
        C.costa_mx_product(1.0, x, q, 0.0, c)
    want = va @ vb.T
    got = c[torch.from_numpy(rows).cuda()].double().cpu().numpy()
    # rounded once to 8 bits, of sums of 16 exact products in 24
    assert (np.abs(got - want) <= 2.0**-8 * np.abs(want) + 2.0**-20 * (np.abs(va) @ np.abs(vb).T)).all()
    c[torch.from_numpy(rows).cuda()] = 0
    assert int(torch.count_nonzero(c)) == 0
