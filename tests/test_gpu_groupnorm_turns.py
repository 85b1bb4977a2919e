"""Group norm where the images take turns on the device (clusters of eight to sixteen CTAs), and 16-bit images whose first values lie far off.

Formulas and tolerances are those of the other group norm tests.  There sums of 64 + P / 8 numbers that follow one another stand for the mean and the
variance; a thread's squares around its first value are fewer (at most 110), and lose 2^-24 of themselves with each, however far off that value lies: it is
one of the image's, so the image's own sum of squares is no smaller.
"""
import math

import pytest
import torch

from paper_2407_12637_b200 import cnn
from test_gpu_groupnorm import _check, _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,G,dtype,act", [((16, 96, 96, 64), 16, torch.float16, "silu"), ((17, 95, 97, 64), 8, torch.bfloat16, "relu"),
                                               ((40, 56, 56, 64), 32, torch.float32, "silu"), ((31, 4001, 66), 11, torch.bfloat16, "none"),
                                               ((37, 3001, 65), 5, torch.float16, "silu"), ((100, 50, 50, 64), 4, torch.bfloat16, "silu")])
def test_images_in_turns(shape, G, dtype, act):
    _run(shape, G, dtype, act, seed=11)


@pytest.mark.parametrize("C", [64, 66, 65])
@pytest.mark.parametrize("first", [0.0, 3e4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_first_values_far_off(dtype, first, C):
    """Values of 300 +- 1 behind a first pixel of 0, or values around 0 behind one of 30000."""
    x, dy, w, b = _inputs((3, 5000, C), dtype, torch.float32, seed=13, mean=300.0 if first == 0.0 else 0.7)
    x[:, 0] = first
    norm = cnn.GroupNorm(C, 1, w, b, act="silu")
    y = norm.forward(x, keep=True)
    _check(x, dy, w, b, 1, "silu", 1e-5, y, norm.backward(dy))


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("pixel", [0, 999])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_what_is_not_finite_stays_in_its_group(dtype, pixel, value):
    """The first value of a thread or another one: its group is not finite, the others keep their bits."""
    x, _, w, b = _inputs((3, 1000, 64), dtype, torch.float32, seed=15)
    norm = cnn.GroupNorm(64, 8, w, b)
    want = norm.forward(x).clone()
    x[1, pixel, 17] = value
    y = norm.forward(x)
    assert not torch.isfinite(y[1, :, 16:24]).any()
    y[1, :, 16:24] = want[1, :, 16:24]
    assert torch.equal(y, want)
