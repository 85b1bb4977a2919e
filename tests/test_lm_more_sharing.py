"""Adapters, group norm and gradient clipping shared by threads, devices and tensors (no GPU): stand-in tensors and devices, the addresses handed to the
library are never read."""
import ctypes as C
import gc
import threading
import weakref

import pytest
import torch

from paper_2407_12637_b200 import cnn, lbt, lm
from test_lm_more_host import A, _Devices, _objects, _Tensor


def _two_at_once(work):
    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(10)


class _Calls:
    """Library calls of a scratch address each: which of them were under way with the same one.  The first one stays until the second has come in, or for 0.3 s."""

    def __init__(self):
        self.inside, self.overlaps, self.entered = [], [], threading.Event()

    def __call__(self, scratch):
        self.overlaps.extend(s for s in self.inside if s == scratch)
        self.inside.append(scratch)
        if len(self.inside) == 1:
            self.entered.wait(0.3)
        else:
            self.entered.set()
        self.inside.remove(scratch)
        return lbt.OK


def test_threads_that_share_a_group_norm_take_turns(monkeypatch):
    """A pass over large images is two launches that meet in the workspace: between the two no other thread's pass may use it."""
    devices = _Devices(monkeypatch)
    _, norm, half = _objects(0)
    x, y, vec = half(2, 3, 16), half(2, 3, 16), _Tensor((16,), torch.float32)
    calls = _Calls()
    devices.lbt_groupnorm_forward = lambda *a: calls(a[10])
    norm.forward(x, out=y)   # (the workspace is there from now on)
    calls.entered.clear()
    _two_at_once(lambda: norm.forward(x, out=y))
    assert not calls.overlaps
    norm.forward(x, out=y, keep=True)
    calls = _Calls()
    devices.lbt_groupnorm_backward = lambda *a: calls(a[9])
    _two_at_once(lambda: norm.backward(y, dx=x, dw=vec, db=vec))
    assert not calls.overlaps


def test_threads_that_share_adapters_take_turns(monkeypatch):
    """A backward pass leaves dh in the workspace, from which the weight gradients' launch reads it."""
    devices = _Devices(monkeypatch)
    adapters, _, half = _objects(0)
    x, dy, da, db = half(5, 64), half(5, 32), _Tensor((2, 4, 64), torch.float32), _Tensor((2, 4, 32), torch.float32)
    adapters.forward(x, half(5, 32), keep=True)
    calls = _Calls()
    devices.lbt_adapters_backward = lambda *a: calls(a[15])
    adapters.backward(dy, half(5, 64), da=da, db=db)
    calls.entered.clear()
    _two_at_once(lambda: adapters.backward(dy, half(5, 64), da=da, db=db))
    assert not calls.overlaps


def test_norms_without_parameters_keep_scratch_for_each_device(monkeypatch):
    """Such a norm belongs to no device, and the default stream's handle is 0 on every one of them."""
    devices = _Devices(monkeypatch)
    monkeypatch.setattr(lbt, "_current_raw_stream", lambda index: 0)
    seen = {}
    devices.lbt_groupnorm_forward = lambda *a: seen.setdefault("forward", []).append((a[9], a[10])) or lbt.OK     # (statistics, workspace)
    devices.lbt_groupnorm_backward = lambda *a: seen.setdefault("backward", []).append((a[5], a[9])) or lbt.OK
    devices.lbt_resnorm_forward = lambda *a: seen.setdefault("res forward", []).append((a[13],)) or lbt.OK
    devices.lbt_resnorm_backward = lambda *a: seen.setdefault("res backward", []).append((a[9], a[17])) or lbt.OK
    norm, res = cnn.GroupNorm(16, 2), lm.ResNorm(32)
    for index in (0, 1):
        x, y = (_Tensor((2, 3, 16), torch.bfloat16, index, at) for at in (A, 2 * A))
        norm.forward(x, out=y, keep=True)
        norm.backward(y, dx=_Tensor((2, 3, 16), torch.bfloat16, index, 3 * A))
        x, y, z = (_Tensor((5, 32), torch.bfloat16, index, at) for at in (A, 2 * A, 3 * A))
        res.forward(x, y, out=(z, z), keep=True)
        res.backward(z, z, out={"dx": x, "dh": y})
    assert len(seen) == 4
    for calls in seen.values():
        assert len(calls) == 2 and all(a != b for a, b in zip(*calls))


def test_a_descriptor_lives_as_long_as_the_call_that_reads_it(monkeypatch):
    """The library's call lets other threads run; one of them may clear the plans (256 sizes) while this one's descriptor is read."""
    devices = _Devices(monkeypatch)
    adapters, norm, half = _objects(0)
    res, alive, own = lm.ResNorm(32), [], []

    def call(*args):
        (plan,) = own[0]._plans.values()
        descriptor = weakref.ref(plan[0])
        del plan
        own[0]._plans.clear()
        gc.collect()
        alive.append(descriptor() is not None)
        return lbt.OK

    for name in ("adapters", "groupnorm", "resnorm"):
        for way in ("forward", "backward"):
            setattr(devices, f"lbt_{name}_{way}", call)
    x, y, z = half(2, 3, 16), half(5, 32), half(5, 64)
    for obj, passes in ((adapters, (lambda: adapters.forward(z, y, keep=True), lambda: adapters.backward(y, z, da=_Tensor((2, 4, 64), torch.float32), db=_Tensor((2, 4, 32), torch.float32)))),
                        (norm, (lambda: norm.forward(x, out=x), lambda: norm.forward(x, out=half(2, 3, 16, at=2 * A), keep=True),
                                lambda: norm.backward(x, dx=x, dw=_Tensor((16,), torch.float32), db=_Tensor((16,), torch.float32)))),
                        (res, (lambda: res.forward(y, y, out=(y, y), keep=True), lambda: res.backward(y, y, out={"dx": y, "dh": y})))):
        own[:] = [obj]
        for work in passes:
            work()
    assert len(alive) == 7 and all(alive)


def test_adapters_keep_no_x_that_is_overwritten(monkeypatch):
    devices = _Devices(monkeypatch)
    half = lambda *s: _Tensor(s, torch.bfloat16)  # noqa: E731
    adapters = lm.Adapters(half(2, 4, 64), half(2, 4, 64))
    x, base = half(5, 64), half(5, 64)
    for bad in (lambda: adapters.forward(x, base, out=x, keep=True), lambda: adapters.forward(x, x, keep=True)):
        with pytest.raises(ValueError):
            bad()
    assert not devices.calls and adapters.kept is None
    adapters.forward(x, base, out=x)   # (without a backward pass x may go)
    assert len(devices.calls) == 1


def test_a_group_norm_keeps_no_x_that_is_overwritten(monkeypatch):
    devices = _Devices(monkeypatch)
    x, clip = _Tensor((2, 3, 16), torch.float32), _Tensor((1,), torch.float32)
    norm = cnn.GroupNorm(16, 2)
    for bad in (lambda: norm.forward(x, out=x, keep=True), lambda: norm.forward_codes(x, clip, out=x, keep=True)):
        with pytest.raises(ValueError):
            bad()
    assert not devices.calls and norm.kept is None
    norm.forward(x, out=x)   # (without a backward pass x may go)
    assert len(devices.calls) == 1


def test_outputs_of_a_clip_lie_apart():
    """In their own gradient's place or nowhere near another tensor: the order in which tensors are read and written is the device's."""
    def clip(grads, out=None):   # (tensors as first byte, elements, type)
        make = lambda spans: [_Tensor((n,), dtype, 0, A + at) for at, n, dtype in spans]  # noqa: E731
        return lm.GradClip(make(grads), 1.0, make(out) if out is not None else None)

    f, h = torch.float32, torch.bfloat16
    two = [(0, 64, f), (256, 64, f)]
    with pytest.MonkeyPatch.context() as patch:
        _Devices(patch)
        patch.setattr(lbt, "_at", lambda t, device=None: t.data_ptr())   # (an object's own result is on the host here)
        for grads, out in ((two, [(256, 64, f), (0, 64, f)]), (two, [(256, 64, f), (512, 64, f)]), (two, [(1024, 64, f), (1200, 64, f)]), (two, [(0, 64, f), (508, 64, f)]),
                           (two, [(4, 64, f), (512, 64, f)]), (two, [(1024, 64, f), (128, 64, h)]), ([(0, 64, f), (252, 64, f)], None), ([(0, 64, f), (0, 8, h)], None)):
            with pytest.raises(ValueError):
                clip(grads, out)
        for grads, out in ((two, None), (two, two), (two, [(0, 64, f), (512, 64, h)]), (two, [(512, 64, f), (768, 64, f)]), ([two[0]] * 2, [(512, 64, f), (768, 64, f)]),
                           (two + [(0, 0, f)], None), (two, [(768, 64, h), (896, 64, h)]), ([(0, 64, f), (4, 0, f)], None)):
            clip(grads, out)


def test_the_scale_of_no_images():
    """q is then an empty tensor, whose address is 0: the scale is asked for all the same, by the quantizer's rules."""
    d = lbt.GroupnormDesc(0, 10, 24, 3, lbt.F32, lbt.F32, lbt.ACT_RELU, 1e-5)
    call = lambda **k: lbt.lib().lbt_groupnorm_forward(C.addressof(d), *{**dict(x=None, w=A, b=A, y=None, q=None, bits=4, clip=A, scale=A, stats=None, ws=A, ws_bytes=1 << 20), **k}.values(), None)  # noqa: E731
    assert call(bits=9) == call(bits=1) == lbt.ERR_UNSUPPORTED_BITS and call(scale=A + 2) == lbt.ERR_ALIGNMENT
    assert call(clip=None, scale=None) == lbt.OK
