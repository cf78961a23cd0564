"""Products in the widest tiles, against 64 bits.  The few-bit operands are random codes with
random scales."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2106_06601_amd as C  # noqa: E402
import mx_formula as F  # noqa: E402
import mx_wide as W  # noqa: E402

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": 2.0**-24, "bf16": 2.0**-9, "f16": 2.0**-12}


def stored(gen, rows, cols, bits):
    """A few-bit matrix and the values that it stands for, in 64 bits."""
    pc = -(-cols // F.PAD[bits]) * F.PAD[bits]
    rand = lambda hi, *shape: torch.randint(hi, shape, generator=gen, device="cuda", dtype=torch.int64)  # noqa: E731
    half = 1 << bits - 1
    grid = torch.from_numpy(F.GRID[bits]).cuda()
    code, sign = rand(len(grid), rows, pc), rand(2, rows, pc)
    code[:, cols:] = 0
    sign[:, cols:] = 0
    scale = 123 + rand(8, rows, pc // 32) - (2 if bits == 4 else 8)
    scale[:, -(-cols // 32):] = 0
    value = torch.where(sign > 0, -grid[code], grid[code]) * torch.repeat_interleave(
        torch.exp2((scale - 127).to(torch.float64)), 32, dim=1)
    data = (code + sign * half).to(torch.uint8)
    if bits == 4:
        data = data[:, 0::2] | data[:, 1::2] << 4
    return C.MxMatrix(bits, rows, cols, data.contiguous(), scale.to(torch.uint8)), value[:, :cols].contiguous()


def check(got, va, vb, alpha, beta, c0, out, parts=1):
    """The bound: sums of k exact products (`parts` of each) in 32 bits, eight at a time at
    least; the result rounded."""
    k = va.shape[1]
    want = alpha * (va @ vb.t())
    size = abs(alpha) * (va.abs() @ vb.abs().t())
    if beta:
        want += beta * c0
        size += (beta * c0).abs()
    bound = (parts * k / 8 + 8) * 2.0**-24 * size + 2 * UNIT[out] * want.abs() + (2.0**-24 if out == "f16" else 0.0)
    worst = ((got.to(torch.float64) - want).abs() / (bound + 1e-300)).max()
    assert float(worst) <= 1.0, float(worst)


def run(call, m, n, outs, va, vb, parts=1):
    """Into rows with beta 0 over NaN; into columns of a padded buffer with beta 0.5."""
    for out in outs:
        c = torch.full((m, n), float("nan"), dtype=TORCH[out], device="cuda")
        call(1.0, 0.0, c)
        check(c, va, vb, 1.0, 0.0, None, out, parts)
        flat = torch.randn(n, m + 3, device="cuda").to(TORCH[out])
        before, c = flat.clone(), flat[:, 2:m + 2].t()
        c0 = c.to(torch.float64)
        call(-0.25, 0.5, c)
        check(c, va, vb, -0.25, 0.5, c0, out, parts)
        assert torch.equal(flat[:, :2], before[:, :2]) and torch.equal(flat[:, m + 2:], before[:, m + 2:])


@pytest.mark.parametrize("shape", W.SHAPES, ids=str)
@pytest.mark.parametrize("bbits", [4, 8])
@pytest.mark.parametrize("abits", [4, 8])
def test_product_in_wide_tiles(shape, abits, bbits):
    m, n, k = shape
    gen = torch.Generator(device="cuda").manual_seed(m + 10 * abits + bbits)
    (a, va), (b, vb) = stored(gen, m, k, abits), stored(gen, n, k, bbits)
    run(lambda alpha, beta, c: C.costa_mx_product(alpha, a, b, beta, c), m, n, ("bf16",), va, vb)


@pytest.mark.parametrize("shape", W.SHAPES, ids=str)
@pytest.mark.parametrize("bbits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("op", ["N", "T"])
def test_product_real_in_wide_tiles(shape, bbits, dtype, op):
    m, n, k = shape
    gen = torch.Generator(device="cuda").manual_seed(m + bbits)
    b, vb = stored(gen, n, k, bbits)
    rows, cols = (m, k) if op == "N" else (k, m)
    held = torch.full((rows, cols + 5), float("nan"), dtype=TORCH[dtype], device="cuda")
    held[:, 3:cols + 3] = torch.randn(rows, cols, generator=gen, device="cuda")
    held[:, 3:cols + 3:17] *= 20
    a = held[:, 3:cols + 3]
    va = a.to(torch.float64)
    va = va if op == "N" else va.t().contiguous()
    run(lambda alpha, beta, c: C.costa_mx_product_real(alpha, op, a, b, beta, c), m, n, (dtype,), va, vb,
        W.PARTS[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("op", ["N", "T"])
def test_what_is_no_number_in_wide_tiles(dtype, op):
    """An infinity and a NaN of rows, and a block of NaN of a column, reach no other element."""
    m, n, k = W.SHAPES[0]
    gen = torch.Generator(device="cuda").manual_seed(3)
    b, vb = stored(gen, n, k, 8)
    b.scales.view(n, -1)[300, 3] = 255
    a = torch.rand(m, k, generator=gen, device="cuda").to(TORCH[dtype])
    a[5, 99], a[m - 1, 64] = float("inf"), float("nan")
    c = torch.empty(m, n, device="cuda")
    C.costa_mx_product_real(1.0, op, a if op == "N" else a.t().contiguous(), b, 0.0, c)
    want = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    want[:, 300] = want[m - 1] = True
    zero = vb[:, 99] == 0
    want[5, zero] = True
    assert torch.equal(torch.isnan(c), want)
    inf = torch.zeros_like(want)
    inf[5] = ~zero
    inf[5, 300] = False
    assert torch.equal(torch.isinf(c), inf)


def test_small_scales():
    """Stored values down to 2^-133, below the normal bfloat16 ones, enter products whole."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    for m in (3, 50, 200):
        for bits in (4, 8):
            b, vb = stored(gen, 140, 256, bits)
            b.scales.fill_(4 if bits == 4 else 6)  # 2^-123, 2^-121: elements from 2^-124, 2^-130 on
            vb = vb * 0 + torch.from_numpy(F.decode(b.data.view(140, -1).cpu().numpy(), b.scales.view(140, -1).cpu().numpy(),
                                                    bits, 256)).cuda()
            a = torch.randn(m, 256, generator=gen, device="cuda") * 2.0**100
            c = torch.empty(m, 140, device="cuda")
            C.costa_mx_product_real(1.0, "N", a, b, 0.0, c)
            check(c, a.to(torch.float64), vb, 1.0, 0.0, None, "f32", 3)
