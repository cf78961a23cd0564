"""A layer's gradients against differences of its own forward product."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2106_06601_amd as C  # noqa: E402
import mx_formula as F  # noqa: E402

pytestmark = pytest.mark.gpu


def f64(t):
    return t.cpu().to(torch.float64).numpy()


@pytest.mark.parametrize("tokens,inputs,outputs", [(70, 130, 90), (300, 257, 200)])
def test_gradients_against_differences_of_the_forward_product(tokens, inputs, outputs):
    """The forward product is linear in X and in the stored weights, so that a difference quotient of
    any step is its derivative.  The gradients read other roundings of the same matrices (W^T in
    blocks along the outputs; X^T in 8 bits): they are off the derivative by what those roundings
    differ by, and by nothing else."""
    rng = np.random.default_rng(tokens)
    f32 = lambda v: v.astype(np.float32)  # noqa: E731
    x, w, dy = (f32(rng.standard_normal(s)) for s in ((tokens, inputs), (outputs, inputs), (tokens, outputs)))
    gpu = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    empty = C.MxMatrix.empty
    wq, wqt, xt = empty(4, outputs, inputs), empty(4, inputs, outputs), empty(8, inputs, tokens)
    C.costa_mx_quantize(1.0, gpu(w), wq, wqt)
    C.costa_mx_quantize(1.0, gpu(x), None, xt)
    dx, dw = torch.empty(tokens, inputs).cuda(), torch.empty(outputs, inputs).cuda()
    C.costa_mx_product_real(1.0, "N", gpu(dy), wqt, 0.0, dx)
    C.costa_mx_product_real(1.0, "T", gpu(dy), xt, 0.0, dw)

    def forward(xx, q):
        y = torch.full((tokens, outputs), float("nan")).cuda()
        C.costa_mx_product_real(1.0, "N", gpu(xx), q, 0.0, y)
        return f64(y)

    # a sum of n products of three parts each, 32 at a time, in 32 bits
    unit = lambda n: (3 * n / 32 + 8) * 2.0**-24  # noqa: E731
    W = F.decode(*F.encode(w, 4), 4, inputs)
    WT = F.decode(*F.encode(w.T, 4), 4, outputs).T
    XT = F.decode(*F.encode(x.T, 8), 8, tokens).T
    size = np.abs(x).astype(np.float64) @ np.abs(W).T
    assert (np.abs(forward(x, wq) - x.astype(np.float64) @ W.T) <= unit(inputs) * size).all()

    # the input: of <dY, Y(X)> along a step, which the two ends take in 32 bits
    step = f32(rng.standard_normal(x.shape))
    up, down = x + step, x - step
    slope = np.sum(dy * (forward(up, wq) - forward(down, wq))) / 2
    along = (up.astype(np.float64) - down) / 2
    off = np.sum((dy.astype(np.float64) @ (WT - W)) * along)
    rounding = unit(inputs) * np.sum((np.abs(dy) @ np.abs(W)) * (np.abs(up) + np.abs(down))) / 2 + \
        unit(outputs) * np.sum((np.abs(dy) @ np.abs(WT)) * np.abs(along))
    assert abs(np.sum(f64(dx) * along) - slope - off) <= rounding
    assert abs(off) > 2 * rounding  # (another rounding of the weights would be seen)

    # the weights: Y is linear in what is stored; a step of values that 4 bits hold
    d = F.decode(*F.encode(f32(rng.standard_normal(w.shape)), 4), 4, inputs)
    dq = empty(4, outputs, inputs)
    C.costa_mx_quantize(1.0, gpu(f32(d)), dq)
    slope = np.sum(dy * forward(x, dq))
    off = np.sum((dy.T.astype(np.float64) @ (XT - x)) * d)
    rounding = unit(inputs) * np.sum((np.abs(dy).T @ np.abs(x)) * np.abs(d)) + \
        unit(tokens) * np.sum((np.abs(dy).T @ np.abs(XT)) * np.abs(d))
    assert abs(np.sum(f64(dw) * d) - slope - off) <= rounding
    assert abs(off) > 2 * rounding
