"""Group norm's statistics where a thread takes many pixels and the first of them lies far off, against 64 bits.

u = 2^-24, D: the distance of the first pixel from the others.  A thread moves the value around which it sums to the mean of its pixels after 4, 8, 16, 32, 64, 96, ..
of them (kept on chip: after a quarter of them, q, or, by eights, not at all, q being all of them; then 3 q u of q D^2 are lost).  The first four: three sums of four terms of at most D^2 (of squares, of differences twice) lose 3 x 4 u of 4 D^2 together, 48 u of D^2, of which the image's own
sum of squares holds at least 1 - 1/P; the next ones, whose differences are D / 4 at most, 8 u more.  Then each of a thread's n pixels may cost u of the sum: the variance
is off by (n + 64) u of itself, where sums by lanes, shares and channels add u for each of their at most 200 numbers, and a mean that is off by e adds 2 e / sigma (a
share's mean times its distance from the whole).  A mean is off by u of the largest value for each time that it moves, n / 32 + 5 of them, and for each of 200 numbers
joined.  rstd is off by half of the variance's error and 4 u of the root.
"""
import pytest
import torch

from paper_2407_12637_b200 import cnn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _stats(x, C, G):
    norm = cnn.GroupNorm(C, G, eps=1e-5)
    norm.forward(x, keep=True)
    return norm.kept[1]


def _check(x, G, n, q=0):
    """n: the pixels of a thread, at most; q: those that it sums around its first one (0: four)."""
    N, P, C = x.shape
    got = _stats(x, C, G).double()
    for g0 in range(0, G, 1024):   # (64-bit copies stay small)
        g1 = min(G, g0 + 1024)
        part = x[:, :, g0 * C // G:g1 * C // G].double().reshape(N, P, g1 - g0, C // G)
        mean = part.mean((1, 3))
        var = ((part - mean[:, None, :, None]) ** 2).mean((1, 3))
        rstd = 1 / torch.sqrt(var + 1e-5)
        off = (n / 32 + 205) * U * part.abs().amax((1, 3))
        assert ((got[:, g0:g1, 0] - mean).abs() <= off).all()
        tol = 0.5 * ((n + 264 + 3 * q * q) * U + 2 * off * rstd) + 6 * U
        err = (got[:, g0:g1, 1] / rstd - 1).abs()
        assert (err <= tol).all(), (float(err.max()), float((err / tol).max()))


def _image(N, P, C, dtype, first, mean, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(P)
    x = torch.empty(N, P, C, dtype=dtype, device="cuda")
    for image in x:
        image.copy_(torch.randn(P, C, generator=g, device="cuda") * std + mean)
    x[:, 0] = first
    return x


FAR = [(0.0, 300.0), (3e4, 0.0)]


@pytest.mark.parametrize("first,mean", FAR)
@pytest.mark.parametrize("shape,G,dtype", [((1, 2500, 76803), 25601, torch.float32), ((40, 2001, 2049), 683, torch.bfloat16)])
def test_images_read_twice(shape, G, dtype, first, mean):
    """One share for each image and block of channels, one pixel lane: a thread takes all of an image's pixels."""
    _check(_image(*shape, dtype, first, mean), G, shape[1])


@pytest.mark.parametrize("first,mean", FAR)
@pytest.mark.parametrize("C,G", [(64, 8), (66, 11), (65, 5)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_images_kept_on_chip(dtype, C, G, first, mean):
    """As large as a cluster keeps: 110 KB a CTA, up to 27 pixels a thread by eights, 55 by twos, 110 one by one."""
    _check(_image(3, 10000, C, dtype, first, mean), G, *{64: (27, 27), 66: (55, 14), 65: (110, 28)}[C])


@pytest.mark.parametrize("shape,G,n", [((3, 10000, 64), 8, (27, 27)), ((3, 10000, 66), 11, (55, 14)), ((3, 10000, 65), 5, (110, 28)), ((40, 2001, 2049), 683, (2001, 0))])
@pytest.mark.parametrize("dtype,std", [(torch.bfloat16, 8.0), (torch.float16, 1.0)], ids=str)
def test_a_mean_far_from_zero(dtype, std, shape, G, n):
    """2000 +- 1 (+- 8, a step of bf16): the mean of the squares less the square of the mean, in fp32, is off by 1.7 times the tolerance and more here (sums of
    25 values, then of 400 such), or negative."""
    _check(_image(*shape, dtype, 2000.0, 2000.0, std), G, *n)
