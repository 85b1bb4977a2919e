"""The norm of many gradients, and clipping by it, against 64 bits.

Tolerances.  Eight squares are added in fp32 (at most five roundings, all of them positive terms) and everything else in 64 bits: the
norm is within 2.5 * 2^-24 and its own rounding, 2^-24; so is the factor; a clipped gradient has one rounding more, to its type (half a step: bf16 keeps 8 bits, 2^-8; fp16 values below 2^-14 are multiples of 2^-24).
"""
import math

import pytest
import torch

from guard import Guard
from paper_2407_12637_b200 import lbt, lm

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
TOL = 4 * EPS
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SIZES = [1, 2, 7, 8, 9, 255, 256, 257, 0, 2047, 2048, 2049, 70000, 33]


def _grads(sizes, dtype, seed=0, scale=1e-2, guard=None, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    guard = guard or Guard()
    out = []
    for n in sizes:
        t = guard.alloc((n + shift,), dtype)[shift:]
        t.copy_(torch.randn(n, generator=gen, device="cuda") * scale)
        out.append(t)
    return out


def _norms(grads):
    each = torch.stack([torch.linalg.vector_norm(g.double()) for g in grads])
    return torch.linalg.vector_norm(each), each


def _near(got, want, tol=TOL):
    assert float((got.double() - want).abs().max()) <= tol * float(want.abs().max()), (got, want)


@pytest.mark.parametrize("shift", [0, 1], ids=["aligned", "shifted"])
@pytest.mark.parametrize("dtype", list(HALF_ULP), ids=str)
def test_norm_and_clipping_in_place(dtype, shift):
    guard = Guard()
    grads = _grads(SIZES, dtype, guard=guard, shift=shift)
    total, each = _norms(grads)
    clip = lm.GradClip(grads, float(total) / 3)
    before = [g.clone() for g in grads]
    assert clip.measure() is clip.norm
    _near(clip.norm, total.reshape(1))
    assert ((clip.norms.double() - each).abs() <= TOL * each).all()
    _near(clip.scale, torch.tensor([1 / 3], dtype=torch.float64, device="cuda"), 2 * TOL)
    assert int(clip.skip) == 0 and all(torch.equal(a, b) for a, b in zip(grads, before))   # (measured, not clipped)
    clip.clip()
    for g, b in zip(grads, before):
        want = b.double() * float(clip.scale)
        assert ((g.double() - want).abs() <= (HALF_ULP[dtype] + 2 * EPS) * want.abs() + 2.0 ** -25 * (dtype == torch.float16)).all()
    guard.check()
    clip.measure()
    assert float(clip.norm) <= float(total) / 3 * (1 + 4 * max(HALF_ULP[dtype], EPS))


@pytest.mark.parametrize("dtype,odtype", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16), (torch.float16, torch.float32),
                                          (torch.float16, torch.float16)], ids=str)
@pytest.mark.parametrize("limit", [0.5, 1e9, math.inf])
def test_clipping_into_other_tensors(dtype, odtype, limit):
    guard = Guard()
    grads = _grads(SIZES, dtype, seed=3)
    outs = [guard.alloc((n,), odtype, 7.0) for n in SIZES]
    before = [g.clone() for g in grads]
    clip = lm.GradClip(grads, limit, out=outs)
    clip.clip()
    total, _ = _norms(grads)
    factor = min(1.0, limit / float(total))
    _near(clip.scale, torch.tensor([factor], dtype=torch.float64, device="cuda"))
    if factor == 1.0:
        assert float(clip.scale) == 1.0
    for g, b, o in zip(grads, before, outs):
        assert torch.equal(g, b)
        want = b.double() * factor
        assert ((o.double() - want).abs() <= (HALF_ULP[odtype] + 6 * EPS) * want.abs() + 2.0 ** -25 * (odtype == torch.float16)).all()
    guard.check()


@pytest.mark.parametrize("count", [0, 1, 40, 41, 128, 129, 800, 801, 1700])
def test_many_tensors(count):
    grads = _grads([(13 * i) % 700 for i in range(count)], torch.float32, seed=5)
    clip = lm.GradClip(grads, 1e-3)
    clip.clip()
    if count == 0:
        assert float(clip.norm) == 0 and float(clip.scale) == 1 and int(clip.skip) == 0 and clip.norms.numel() == 0
        return
    before = _grads([(13 * i) % 700 for i in range(count)], torch.float32, seed=5)
    total, each = _norms(before)
    assert abs(float(clip.norm) - float(total)) <= TOL * float(total)
    assert ((clip.norms.double() - each).abs() <= TOL * each).all()
    factor = min(1.0, 1e-3 / float(total)) if float(total) else 1.0
    for g, b in zip(grads, before):
        assert ((g.double() - b.double() * factor).abs() <= 6 * EPS * b.double().abs()).all()


@pytest.mark.parametrize("size", [3e4, 1e19, 3e38, 1e-18, 1e-25, 1e-38, 1e-44, 0.0])
def test_squares_beyond_fp32(size):
    """Squares of these overflow or vanish in fp32: the norm does not, and no gradient is called infinite."""
    grads = [torch.full((1000,), size, device="cuda"), torch.full((3,), -size, device="cuda")]
    grads[0][::3] = 0.0
    clip = lm.GradClip(grads, 1.0)
    clip.measure()
    total, each = _norms(grads)
    want = total.float().double()   # (beyond fp32's range: infinite there too)
    assert int(clip.skip) == 0
    assert float(clip.norm) == float(want) or abs(float(clip.norm) - float(want)) <= TOL * float(want) + 2.0 ** -149
    factor = min(1.0, 1.0 / float(total)) if float(total) else 1.0
    assert abs(float(clip.scale) - factor) <= TOL * factor + 2.0 ** -149
    assert ((clip.norms.double() - each).abs() <= TOL * each + 2.0 ** -149).all() or not torch.isfinite(each.float()).all()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_gradient_that_is_not_finite(bad):
    grads = _grads([100, 5000, 17], torch.bfloat16, seed=7)
    grads[1][4321] = bad
    before = [g.clone() for g in grads]
    clip = lm.GradClip(grads, 1e-3)
    clip.clip()
    assert int(clip.skip) == 1 and float(clip.scale) == 0.0 and not math.isfinite(float(clip.norm))
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(grads, before))
    assert torch.isfinite(clip.norms).tolist() == [True, False, True]
    grads[1][4321] = 0.0   # the next step is whole again
    clip.clip()
    assert int(clip.skip) == 0 and float(clip.scale) > 0.0


def test_grad_scale_is_part_of_norm_and_factor():
    grads = _grads([300, 5000], torch.float32, seed=9)
    total, _ = _norms(grads)
    clip, s = lm.GradClip(grads, 0.25), torch.tensor([-1.0 / 1024], device="cuda")
    clip.measure(grad_scale=s)
    _near(clip.norm, (total / 1024).reshape(1))
    assert abs(float(clip.scale) + min(1.0, 0.25 * 1024 / float(total)) / 1024) <= 2 * TOL / 1024
    clip.measure(grad_scale=torch.tensor([math.inf], device="cuda"))
    assert int(clip.skip) == 1


def test_before_an_optimizer_step():
    """measure + AdamW.step(grad_scale, skip) is clip + AdamW.step, up to the rounding of the clipped gradients; a gradient that is not
    finite holds the step back."""
    sizes = [1000, 257, 3]

    def make():
        ps, gs = _grads(sizes, torch.float32, seed=11), _grads(sizes, torch.float32, seed=12, scale=3.0)
        return ps, gs, lm.GradClip(gs, 1.0), lm.AdamW(ps, gs, lr=1e-2, state_bits=32)
    ps, gs, clip, opt = make()
    clip.measure()
    opt.step(grad_scale=clip.scale, skip=clip.skip)
    qs, hs, clip2, opt2 = make()
    clip2.clip()
    opt2.step()
    for a, b, m, n in zip(ps, qs, opt.m, opt2.m):
        assert ((a - b).abs() <= 1e-2 * 64 * EPS + 4 * EPS * a.abs()).all() and ((m - n).abs() <= 4 * EPS * m.abs()).all()
    before = [p.clone() for p in ps]
    gs[0][5] = math.nan
    clip.measure()
    opt.step(grad_scale=clip.scale, skip=clip.skip)
    assert all(torch.equal(a, b) for a, b in zip(ps, before)) and opt.taken() == 1


def test_the_same_gradients_give_the_same_bits():
    grads = _grads([100000, 3, 70001, 513] * 5, torch.bfloat16, seed=13)
    clip, seen = lm.GradClip(grads, 1.0), set()
    for _ in range(20):
        clip.measure()
        seen.add((float(clip.norm), float(clip.scale), tuple(clip.norms.tolist())))
    assert len(seen) == 1


def test_streams_and_captured_graphs():
    grads = _grads([4096, 999], torch.float32, seed=15)
    clip, side = lm.GradClip(grads, 1e-2), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    clip.measure(stream=side)
    side.synchronize()
    want = float(clip.norm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clip.clip()
    for factor in (1.0, 3.0):
        for g, b in zip(grads, _grads([4096, 999], torch.float32, seed=15)):
            g.copy_(b * factor)
        graph.replay()
        assert abs(float(clip.norm) - factor * want) <= TOL * factor * want
        total, _ = _norms(grads)
        assert abs(float(total) - 1e-2) <= 1e-2 * 8 * EPS
    clip.measure()   # eager again, next to the graph that lives
    assert abs(float(clip.norm) - 1e-2) <= 1e-2 * 8 * EPS
    assert clip._space and lbt.grad_norm_workspace_bytes(clip.table) == clip._bytes
