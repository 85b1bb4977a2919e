"""fp16 adapters' weight gradients where one rank is not finite, against 64 bits: the other ranks keep their digits.

h (or dh) enters as two fp16 numbers after a power of two that brings the largest finite one to 512 or more: off by 2^-22 of itself and 2^-33 of the largest.  It is a sum
of I (or O) products in fp32, the gradient a sum over M tokens: 2^-24 of the products' absolute values for each of them, and 8 for the sums of parts.
"""
import pytest
import torch

from paper_2407_12637_b200 import lm

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("size", [1e-4, 1.0, 3e3])   # of x and dy: h and dh from below 2^-20 to above 65504
@pytest.mark.parametrize("r", [4, 16, 40])
def test_one_rank_is_not_finite(r, size, value):
    g = torch.Generator(device="cuda").manual_seed(r)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    M, I, O = 200, 64, 48
    factor = 10.0 if size > 1 else 1e-3 if size < 1 else 1.0
    a, b, x, dy = ((randn(*s) * f).half() for s, f in (((1, r, I), factor), ((1, r, O), factor), ((M, I), size), ((M, O), size)))
    a[0, 2, 5] = b[0, 1, 7] = value
    adapters = lm.Adapters(a, b)
    adapters.forward(x, torch.zeros(M, O, dtype=torch.half, device="cuda"), keep=True)
    grads = adapters.backward(dy)
    A, B, X, D = (t.double() for t in (a[0], b[0], x, dy))
    for got, weights, source, other, bad in ((grads["db"][0], A, X, D, 2), (grads["da"][0], B, D, X, 1)):
        fine = [k for k in range(r) if k != bad]
        f, width = source @ weights[fine].T, weights.shape[1]
        tol = ((width + M + 8) * U * (source.abs() @ weights[fine].abs().T) + 2.0 ** -22 * f.abs() + 2.0 ** -33 * f.abs().max()).T @ other.abs()
        err = (got[fine].double() - f.T @ other).abs()
        assert (err <= tol).all(), float((err / tol).max())
        assert not torch.isfinite(got[bad]).any()
