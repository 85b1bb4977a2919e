"""Host side of gradient clipping, adapters and group norm (no GPU): struct mirrors, workspace sizes, every refusal that needs no device, and what
their objects do with devices, streams and scratch.  The addresses handed to the library are never read."""
import contextlib
import ctypes as C

import pytest
import torch

from paper_2407_12637_b200 import build as lib_build
from paper_2407_12637_b200 import cnn, lbt, lm

A = 1 << 20   # an aligned address


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


def test_struct_sizes():
    assert (C.sizeof(lbt.GradTensor), C.sizeof(lbt.AdaptersDesc), C.sizeof(lbt.GroupnormDesc)) == (32, 96, 80)
    assert lbt.AdaptersDesc.ld_x.offset == 48 and lbt.GroupnormDesc.ld_x.offset == 48 and lbt.GradTensor.g_type.offset == 24


# ---------------------------------------------------------------------------------------------- gradient norm
@pytest.mark.parametrize("change,want", [
    ({"count": -1}, lbt.ERR_INVALID_ARG), ({"table": None}, lbt.ERR_INVALID_ARG), ({"g": None}, lbt.ERR_INVALID_ARG), ({"g_type": 3}, lbt.ERR_INVALID_ARG),
    ({"g": A + 2}, lbt.ERR_ALIGNMENT), ({"n": (1 << 40) + 1}, lbt.ERR_UNSUPPORTED), ({"max_norm": 0.0}, lbt.ERR_INVALID_ARG), ({"max_norm": float("nan")}, lbt.ERR_INVALID_ARG),
    ({"result": None}, lbt.ERR_INVALID_ARG), ({"result": A + 2}, lbt.ERR_ALIGNMENT), ({"norms": A + 1}, lbt.ERR_ALIGNMENT), ({"scale": A + 2}, lbt.ERR_ALIGNMENT),
    ({"ws": None}, lbt.ERR_WORKSPACE), ({"ws": A + 4}, lbt.ERR_ALIGNMENT), ({"ws_bytes": 8}, lbt.ERR_WORKSPACE)])
def test_grad_norm(change, want):
    a = {"g": A, "n": 5000, "g_type": lbt.F32, "max_norm": 1.0, "scale": None, "result": A, "norms": A, "ws": A, "ws_bytes": 1 << 20, "count": 1, **change}
    table = (lbt.GradTensor * 1)(lbt.GradTensor(a["g"], A, a["n"], a["g_type"], lbt.F32))
    assert lbt.lib().lbt_grad_norm(a.get("table", table), a["count"], a["max_norm"], a["scale"], a["result"], a["norms"], a["ws"], a["ws_bytes"], None) == want


def test_grad_clip_and_workspace():
    f = lbt.lib().lbt_grad_clip
    t = lambda **k: (lbt.GradTensor * 1)(lbt.GradTensor(*[{"g": A, "out": A, "n": 9, "g_type": lbt.F32, "out_type": lbt.BF16, **k}[n] for n in ("g", "out", "n", "g_type", "out_type")]))  # noqa: E731
    assert f(None, 1, A, None) == lbt.ERR_INVALID_ARG and f(None, 0, A, None) == lbt.OK and f(None, 0, None, None) == lbt.ERR_INVALID_ARG
    assert f(t(out=None), 1, A, None) == lbt.ERR_INVALID_ARG and f(t(out_type=9), 1, A, None) == lbt.ERR_INVALID_ARG and f(t(out=A + 1), 1, A, None) == lbt.ERR_ALIGNMENT
    assert f(t(), 1, A + 2, None) == lbt.ERR_ALIGNMENT and f(t(n=0, g=None, out=None), 1, A, None) == lbt.OK
    assert lbt.grad_norm_workspace_bytes(t(n=1)) >= 16 and lbt.grad_norm_workspace_bytes(t(g_type=7)) == 0
    sizes = [lbt.grad_norm_workspace_bytes(t(n=10 ** k)) for k in range(3, 12)]
    assert sizes == sorted(sizes) and sizes[-1] <= 8 * (148 * 16 + 2)   # the chunks grow with the tensors


# ---------------------------------------------------------------------------------------------- adapters
def _adapters(**change):
    d = lbt.AdaptersDesc(8, 64, 32, 2, 3, 16, lbt.BF16, 0)
    for k, v in change.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,want", [
    ({"M": -1}, lbt.ERR_INVALID_ARG), ({"I": 0}, lbt.ERR_INVALID_ARG), ({"O": 0}, lbt.ERR_INVALID_ARG), ({"runs": -1}, lbt.ERR_INVALID_ARG), ({"adapters": 0}, lbt.ERR_INVALID_ARG),
    ({"rank": 0}, lbt.ERR_INVALID_ARG), ({"rank": 129}, lbt.ERR_UNSUPPORTED), ({"type": 3}, lbt.ERR_INVALID_ARG), ({"ld_x": 63}, lbt.ERR_INVALID_ARG),
    ({"ld_out": 31}, lbt.ERR_INVALID_ARG), ({"M": 1 << 29}, lbt.ERR_UNSUPPORTED), ({"adapters": 65536}, lbt.ERR_UNSUPPORTED), ({"M": 0}, lbt.OK), ({"runs": 0}, lbt.OK)])
def test_adapters_desc(change, want):
    d = _adapters(**change)
    assert lbt.lib().lbt_adapters_forward(C.addressof(d), A, A, A, A, A, A, A, A if want != lbt.OK else None, None, None, None) == want
    assert (lbt.adapters_workspace_bytes(d) > 0) == (want == lbt.OK)


def test_adapters_pointers():
    f, b = lbt.lib().lbt_adapters_forward, lbt.lib().lbt_adapters_backward
    keep = _adapters()
    d = C.addressof(keep)
    args = dict(x=A, a=A, b=A, scale=A, offsets=A, index=A, base=A, out=A, h=A, status=A)
    call = lambda **k: f(d, *{**args, **k}.values(), None)  # noqa: E731
    for name in ("x", "a", "b", "base", "out"):
        assert call(**{name: None}) == lbt.ERR_INVALID_ARG and call(**{name: A + 1}) == lbt.ERR_ALIGNMENT
    for name in ("scale", "offsets", "index", "h", "status"):
        assert call(**{name: A + 2}) == lbt.ERR_ALIGNMENT
    assert call(index=None) == lbt.ERR_INVALID_ARG and call(offsets=None) == lbt.ERR_INVALID_ARG
    assert f(None, *args.values(), None) == lbt.ERR_INVALID_ARG
    more = dict(dy=A, x=A, h=A, a=A, b=A, scale=None, offsets=A, index=A, dbase=A, dx=A, da=A, db=A, grad_type=lbt.F32, status=None, ws=A, ws_bytes=1 << 20)
    call = lambda **k: b(d, *{**more, **k}.values(), None)  # noqa: E731
    for name in ("dy", "x", "h", "a", "b", "dbase", "index"):
        assert call(**{name: None}) == lbt.ERR_INVALID_ARG
    for name in ("dy", "x", "dx", "da", "db", "h", "ws"):
        assert call(**{name: A + 1}) == lbt.ERR_ALIGNMENT
    assert call(dx=None, da=None, db=None) == lbt.ERR_INVALID_ARG and call(grad_type=lbt.F16) == lbt.ERR_INVALID_ARG
    assert call(ws=None) == lbt.ERR_WORKSPACE and call(ws_bytes=8 * 16 * 4 - 1) == lbt.ERR_WORKSPACE


def test_adapters_gradient_in_the_place_of_what_is_read_behind_it():
    """dx is written first: not in the place of x where da is wanted, nor in dy's where db is."""
    d = _adapters()
    B = A + (1 << 20)
    for x, dy, dx, da, db in ((A, B, A, A, None), (A, B, A, A, A), (B, A, A, None, A), (B, A, A, A, A)):
        status = lbt.lib().lbt_adapters_backward(C.addressof(d), dy, x, A, A, A, None, A, A, A, dx, da, db, lbt.F32, None, A, 1 << 20, None)
        assert status == lbt.ERR_INVALID_ARG


# ---------------------------------------------------------------------------------------------- group norm
def _norm(**change):
    d = lbt.GroupnormDesc(2, 10, 24, 3, lbt.BF16, lbt.F32, lbt.ACT_RELU, 1e-5)
    for k, v in change.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,want", [
    ({"N": -1}, lbt.ERR_INVALID_ARG), ({"P": 0}, lbt.ERR_INVALID_ARG), ({"C": 0}, lbt.ERR_INVALID_ARG), ({"G": 0}, lbt.ERR_INVALID_ARG), ({"G": 5}, lbt.ERR_INVALID_ARG),
    ({"type": 3}, lbt.ERR_INVALID_ARG), ({"param_type": -1}, lbt.ERR_INVALID_ARG), ({"act": 3}, lbt.ERR_INVALID_ARG), ({"eps": -1.0}, lbt.ERR_INVALID_ARG),
    ({"eps": float("nan")}, lbt.ERR_INVALID_ARG), ({"ld_x": 23}, lbt.ERR_INVALID_ARG), ({"ld_dx": 5}, lbt.ERR_INVALID_ARG), ({"N": 65535}, lbt.ERR_UNSUPPORTED), ({"N": 0}, lbt.OK)])
def test_groupnorm_desc(change, want):
    d = _norm(**change)
    assert lbt.lib().lbt_groupnorm_forward(C.addressof(d), A, A, A, A, None, 0, None, None, A, A, 1 << 20, None) == want
    assert (lbt.groupnorm_workspace_bytes(d) > 0) == (want == lbt.OK)


def test_groupnorm_pointers():
    f, b = lbt.lib().lbt_groupnorm_forward, lbt.lib().lbt_groupnorm_backward
    keep, odd = _norm(), _norm(C=21, G=3)
    args = dict(x=A, w=A, b=A, y=A, q=None, bits=0, clip=None, scale=None, stats=A, ws=A, ws_bytes=1 << 20)
    call = lambda d=keep, **k: f(C.addressof(d), *{**args, **k}.values(), None)  # noqa: E731
    assert call(x=None) == call(y=None) == call(q=A, bits=4) == call(q=A, bits=4, clip=A) == lbt.ERR_INVALID_ARG
    for name, at in (("x", A + 1), ("y", A + 1), ("w", A + 2), ("b", A + 2), ("stats", A + 4), ("ws", A + 4)):
        assert call(**{name: at}) == lbt.ERR_ALIGNMENT
    codes = dict(q=A, clip=A, scale=A)
    assert call(**codes, bits=1) == call(**codes, bits=9) == lbt.ERR_UNSUPPORTED_BITS and call(**{**codes, "q": A + 4}, bits=4) == lbt.ERR_ALIGNMENT
    assert call(odd, **codes, bits=4) == lbt.ERR_UNSUPPORTED and call(**codes, bits=4, x=A + 2) == lbt.ERR_ALIGNMENT
    assert call(ws=None) == call(ws_bytes=16) == lbt.ERR_WORKSPACE
    more = dict(dy=A, x=A, w=A, b=A, stats=A, dx=A, dw=A, db=A, ws=A, ws_bytes=1 << 20)
    call = lambda **k: b(C.addressof(keep), *{**more, **k}.values(), None)  # noqa: E731
    for name in ("dy", "x", "stats"):
        assert call(**{name: None}) == lbt.ERR_INVALID_ARG
    assert call(dx=None, dw=None, db=None) == lbt.ERR_INVALID_ARG and call(ws_bytes=16) == lbt.ERR_WORKSPACE
    for name in ("dy", "dx", "dw", "db", "stats"):
        assert call(**{name: A + 1}) == lbt.ERR_ALIGNMENT


# ---------------------------------------------------------------------------------------------- devices, streams and scratch, without a device
class _Tensor:
    """A contiguous tensor as the objects see one on a CUDA device: nothing behind its address."""

    def __init__(self, shape, dtype, index=0, at=A, strides=None):
        self.shape, self.dtype, self.index, self.at, self.strides = torch.Size(shape), dtype, index, at, strides
        self.device = torch.device("cpu")   # where an object makes its scratch

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return self.index

    def stride(self):
        steps = [1]
        for n in reversed(self.shape[1:]):
            steps.append(steps[-1] * n)
        return self.strides or tuple(reversed(steps))

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


class _Devices:
    """Two CUDA devices as torch and the library see them: which one is current, and which one each call was made on."""

    def __init__(self, monkeypatch):
        self.current, self.calls = 0, []
        monkeypatch.setattr(lbt, "_device", lambda: self.current)
        monkeypatch.setattr(lbt, "_current_raw_stream", lambda index: 7)
        monkeypatch.setattr(lbt, "lib", lambda: self)
        monkeypatch.setattr(torch.cuda, "device", self.enter)
        monkeypatch.setattr(torch.cuda, "stream", self.enter)
        monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False)
        zeros = torch.zeros   # (what the objects keep of their own is on the host here, and said to be on their tensors' device)
        monkeypatch.setattr(torch, "zeros", lambda *a, **k: zeros(*a, **k) if "index" not in k else None)

    @contextlib.contextmanager
    def enter(self, where):
        before = self.current
        self.current = where if isinstance(where, int) else getattr(where, "device_index", before)
        try:
            yield
        finally:
            self.current = before

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("workspace_bytes"):
                return 256
            self.calls.append((name, self.current))
            return lbt.OK
        return call


def _objects(index):
    half = lambda *s, **k: _Tensor(s, torch.bfloat16, index, **k)  # noqa: E731
    adapters = lm.Adapters(half(2, 4, 64), half(2, 4, 32), _Tensor((2,), torch.float32, index))
    norm = cnn.GroupNorm(16, 2, _Tensor((16,), torch.float32, index), _Tensor((16,), torch.float32, index))
    return adapters, norm, half


def test_calls_launch_on_their_tensors_device(monkeypatch):
    devices = _Devices(monkeypatch)
    adapters, norm, half = _objects(1)
    adapters.forward(half(5, 64), half(5, 32), keep=True)
    adapters.backward(half(5, 32), half(5, 64), da=_Tensor((2, 4, 64), torch.float32, 1), db=_Tensor((2, 4, 32), torch.float32, 1))
    norm.forward(half(2, 3, 16), out=half(2, 3, 16), keep=True)
    norm.backward(half(2, 3, 16), dx=half(2, 3, 16), dw=_Tensor((16,), torch.float32, 1), db=_Tensor((16,), torch.float32, 1))
    assert len(devices.calls) == 4 and {index for _, index in devices.calls} == {1} and devices.current == 0


def test_operands_on_several_devices_are_refused(monkeypatch):
    devices = _Devices(monkeypatch)
    adapters, norm, half = _objects(1)
    other = lambda *s: _Tensor(s, torch.bfloat16, 0)  # noqa: E731
    i32 = lambda n, index: _Tensor((n,), torch.int32, index)  # noqa: E731
    for bad in (lambda: adapters.forward(other(5, 64), other(5, 32)), lambda: adapters.forward(half(5, 64), other(5, 32)),
                lambda: adapters.forward(half(5, 64), half(5, 32), i32(3, 0), i32(2, 1)), lambda: adapters.forward(half(5, 64), half(5, 32), i32(3, 1), i32(2, 0)),
                lambda: norm.forward(other(2, 3, 16), out=other(2, 3, 16)), lambda: norm.forward(half(2, 3, 16), out=other(2, 3, 16)),
                lambda: lm.Adapters(half(1, 4, 8), other(1, 4, 8)), lambda: cnn.GroupNorm(16, 2, _Tensor((16,), torch.float32, 0), _Tensor((16,), torch.float32, 1)),
                lambda: lm.GradClip([half(5), other(5)]), lambda: lm.GradClip([half(5)], out=[other(5)]), lambda: lm.GradClip([_Tensor((5,), torch.float32, -1)])):
        with pytest.raises(ValueError):
            bad()
    assert not devices.calls


def test_a_captured_call_keeps_no_scratch(monkeypatch):
    _Devices(monkeypatch)
    for capturing in (True, False):
        monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: capturing)
        adapters, norm, half = _objects(0)
        adapters.forward(half(5, 64), half(5, 32), keep=True)
        adapters.backward(half(5, 32), half(5, 64), da=_Tensor((2, 4, 64), torch.float32), db=_Tensor((2, 4, 32), torch.float32))
        norm.forward(half(2, 3, 16), out=half(2, 3, 16), keep=True)
        for kept in (adapters._own_kept, adapters._space, norm._stats, norm._space):
            assert bool(kept) != capturing
        assert adapters.kept is not None and norm.kept is not None


def test_what_a_clip_refuses(monkeypatch):
    _Devices(monkeypatch)
    g = lambda n=5, dtype=torch.float32, at=A: _Tensor((n,), dtype, 0, at)  # noqa: E731
    for bad in (lambda: lm.GradClip([g()], max_norm=0.0), lambda: lm.GradClip([g()], max_norm=float("nan")), lambda: lm.GradClip([g()], out=[]),
                lambda: lm.GradClip([g()], out=[g(6, at=2 * A)]), lambda: lm.GradClip([g(dtype=torch.float64)]), lambda: lm.GradClip([g(), g()]),   # the same gradient twice
                lambda: lm.GradClip([g()], out=[g(dtype=torch.bfloat16)])):                                                                         # another type in the same place
        with pytest.raises(ValueError):
            bad()


def test_rows_that_overlap_are_refused(monkeypatch):
    """An expanded tensor's leading dimension is 0, which stands for the row's length in a descriptor: it must not get there."""
    devices = _Devices(monkeypatch)
    adapters, norm, half = _objects(0)
    wide = half(5, 32, strides=(0, 1))
    res = lm.ResNorm(32)
    for bad in (lambda: adapters.forward(half(5, 64), wide), lambda: adapters.forward(half(5, 64), half(5, 32), out=half(5, 32, strides=(31, 1))),
                lambda: norm.forward(half(2, 3, 16, strides=(0, 0, 1)), out=half(2, 3, 16)), lambda: norm.forward(half(2, 3, 16, strides=(45, 15, 1)), out=half(2, 3, 16)),
                lambda: res.forward(wide, half(5, 32), out=(half(5, 32), half(5, 32))), lambda: res.forward(half(5, 32), half(5, 32), out=(wide, half(5, 32)))):
        with pytest.raises(ValueError):
            bad()
    assert not devices.calls
    one = half(1, 32, strides=(0, 1))   # (one row does not overlap)
    res.forward(one, half(1, 32), out=(half(1, 32), half(1, 32)))
    assert len(devices.calls) == 1
