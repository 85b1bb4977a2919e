"""Host side of the transformer operators (no GPU): struct mirrors, workspace sizes, and every refusal that needs no device.

The addresses handed to the library here are never read: each call is refused (or has nothing to do) before a launch.
"""
import contextlib
import ctypes as C
import threading
import types

import pytest
import torch

from paper_2407_12637_b200 import build as lib_build
from paper_2407_12637_b200 import lbt, lm

A = 1 << 20   # an aligned address


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


def test_struct_sizes():
    assert (C.sizeof(lbt.AdamwTensor), C.sizeof(lbt.AdamwHyper), C.sizeof(lbt.ResnormDesc)) == (80, 40, 120)
    assert lbt.ResnormDesc.ld_x.offset == 56 and lbt.ResnormDesc.ld_dh.offset == 112


def test_pitch_of_code_rows():
    assert [lbt.pitch8(n) for n in (1, 15, 16, 17, 4096)] == [16, 16, 16, 32, 4096]
    assert 127 * 127 * lbt.MAX_REDUCTION8 < 2 ** 31 <= 127 * 127 * (lbt.MAX_REDUCTION8 + 1)


@pytest.mark.parametrize("change,want", [
    ({}, lbt.OK), ({"rows": -1}, lbt.ERR_INVALID_ARG), ({"cols": 0}, lbt.ERR_INVALID_ARG), ({"ld": 63}, lbt.ERR_INVALID_ARG),
    ({"type": 3}, lbt.ERR_INVALID_ARG), ({"ldq": 48}, lbt.ERR_INVALID_ARG), ({"ldq": 72}, lbt.ERR_ALIGNMENT), ({"q": A + 8}, lbt.ERR_ALIGNMENT),
    ({"x": A + 2}, lbt.ERR_ALIGNMENT), ({"rows": 4, "x": None}, lbt.ERR_INVALID_ARG), ({"rows": 4, "scale": None}, lbt.ERR_INVALID_ARG),
    ({"rows": 1 << 31}, lbt.ERR_UNSUPPORTED)])
def test_rows8(change, want):
    a = {"x": A, "type": lbt.F32, "rows": 0, "cols": 64, "ld": 64, "q": A, "ldq": 64, "scale": A, **change}
    assert lbt.lib().lbt_rows8_quantize(a["x"], a["type"], a["rows"], a["cols"], a["ld"], a["q"], a["ldq"], a["scale"], None) == want


@pytest.mark.parametrize("change,want", [
    ({}, lbt.OK), ({"M": -1}, lbt.ERR_INVALID_ARG), ({"O": 0}, lbt.ERR_INVALID_ARG), ({"I": 0}, lbt.ERR_INVALID_ARG), ({"ldy": 31}, lbt.ERR_INVALID_ARG),
    ({"ldx": 63}, lbt.ERR_INVALID_ARG), ({"x_type": -1}, lbt.ERR_INVALID_ARG), ({"y_type": 7}, lbt.ERR_INVALID_ARG), ({"q_w": None}, lbt.ERR_INVALID_ARG),
    ({"s_w": None}, lbt.ERR_INVALID_ARG), ({"q_w": A + 4}, lbt.ERR_ALIGNMENT), ({"q_x": A + 8}, lbt.ERR_ALIGNMENT), ({"bias": A + 2}, lbt.ERR_ALIGNMENT),
    ({"y": A + 1}, lbt.ERR_ALIGNMENT), ({"M": 4, "y": None}, lbt.ERR_INVALID_ARG), ({"M": 4, "q_x": None}, lbt.ERR_INVALID_ARG),
    ({"I": 133145, "ldx": 133145}, lbt.ERR_ACC_RANGE), ({"M": 1 << 31}, lbt.ERR_UNSUPPORTED)])
def test_linear8_forward(change, want):
    a = {"x": A, "x_type": lbt.BF16, "ldx": 64, "q_w": A, "s_w": A, "bias": None, "y": A, "y_type": lbt.BF16, "ldy": 32, "M": 0, "O": 32, "I": 64,
         "q_x": A, "s_x": A, **change}
    assert lbt.lib().lbt_linear8_forward(a["x"], a["x_type"], a["ldx"], a["q_w"], a["s_w"], a["bias"], a["y"], a["y_type"], a["ldy"], a["M"], a["O"],
                                         a["I"], a["q_x"], a["s_x"], None, None) == want
    if not set(change) & {"ldx", "x_type"} or "I" in change:
        assert lbt.lib().lbt_linear8_matmul(a["q_x"], a["s_x"], a["q_w"], a["s_w"], a["bias"], a["y"], a["y_type"], a["ldy"], a["M"], a["O"], a["I"],
                                            None, None) == want


@pytest.mark.parametrize("change,want", [
    ({"dX": None, "dW": None, "dbias": None}, lbt.ERR_INVALID_ARG), ({"lddy": 31}, lbt.ERR_INVALID_ARG), ({"lddx": 63}, lbt.ERR_INVALID_ARG),
    ({"lddw": 63}, lbt.ERR_INVALID_ARG), ({"dw_type": 5}, lbt.ERR_INVALID_ARG), ({"q_w": None}, lbt.ERR_INVALID_ARG), ({"q_x": None}, lbt.ERR_INVALID_ARG),
    ({"s_x": None}, lbt.ERR_INVALID_ARG), ({"dY": None}, lbt.ERR_INVALID_ARG), ({"dY": A + 1}, lbt.ERR_ALIGNMENT), ({"q_x": A + 1}, lbt.ERR_ALIGNMENT),
    ({"M": 133145}, lbt.ERR_ACC_RANGE), ({"O": 133145, "lddy": 133145}, lbt.ERR_ACC_RANGE), ({"ws": None}, lbt.ERR_WORKSPACE),
    ({"ws_bytes": 1000}, lbt.ERR_WORKSPACE), ({"M": 4194241, "dW": None}, lbt.ERR_UNSUPPORTED)])
def test_linear8_backward(change, want):
    a = {"dY": A, "lddy": 32, "q_w": A, "s_w": A, "q_x": A, "s_x": A, "dX": A, "lddx": 64, "dW": A, "dw_type": lbt.F32, "lddw": 64, "dbias": A, "M": 8, "O": 32,
         "I": 64, "ws": A, "ws_bytes": 1 << 40, **change}
    assert lbt.lib().lbt_linear8_backward(a["dY"], lbt.BF16, a["lddy"], a["q_w"], a["s_w"], a["q_x"], a["s_x"], a["dX"], lbt.BF16, a["lddx"], a["dW"],
                                          a["dw_type"], a["lddw"], a["dbias"], a["M"], a["O"], a["I"], None, a["ws"], a["ws_bytes"], None) == want


def test_linear8_workspace():
    assert lbt.linear8_workspace_bytes(0, 32, 64) > 0 and lbt.linear8_workspace_bytes(-1, 32, 64) == 0
    # two code matrices, scales and maxima of rows and columns
    assert lbt.linear8_workspace_bytes(1000, 50, 64) >= 2 * 1000 * 64 + 8 * (1000 + 50)


def _desc(**change):
    d = lbt.ResnormDesc(0, 64, 0, lbt.BF16, lbt.F32, lbt.NORM_RMS, 1, 1e-6, 1e-6, 1.0, 1.0)
    for k, v in change.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,want", [
    ({}, lbt.OK), ({"M": -1}, lbt.ERR_INVALID_ARG), ({"D": 0}, lbt.ERR_INVALID_ARG), ({"type": 9}, lbt.ERR_INVALID_ARG), ({"param_type": -1}, lbt.ERR_INVALID_ARG),
    ({"kind": 2}, lbt.ERR_INVALID_ARG), ({"rows_per_gate": -1}, lbt.ERR_INVALID_ARG), ({"eps_pre": -1.0}, lbt.ERR_INVALID_ARG),
    ({"eps_post": float("nan")}, lbt.ERR_INVALID_ARG), ({"ld_h": 63}, lbt.ERR_INVALID_ARG), ({"D": 32769}, lbt.ERR_UNSUPPORTED)])
def test_resnorm_desc(change, want):
    d = _desc(**change)
    assert lbt.lib().lbt_resnorm_forward(C.addressof(d), A, A, None, A, None, A, None, A, A, None, 0, None, None, None) == want
    assert (lbt.resnorm_workspace_bytes(d) > 0) == (want == lbt.OK)


def test_resnorm_pointers():
    f, b = lbt.lib().lbt_resnorm_forward, lbt.lib().lbt_resnorm_backward
    d, at = _desc(M=4), lambda d: C.addressof(d)  # noqa: E731
    assert f(None, A, A, None, A, None, A, None, A, A, None, 0, None, None, None) == lbt.ERR_INVALID_ARG
    assert f(at(d), None, A, None, A, None, A, None, A, A, None, 0, None, None, None) == lbt.ERR_INVALID_ARG
    assert f(at(d), A, A, None, A, None, A, None, None, A, None, 0, None, None, None) == lbt.ERR_INVALID_ARG
    assert f(at(d), A + 1, A, None, A, None, A, None, A, A, None, 0, None, None, None) == lbt.ERR_ALIGNMENT
    assert f(at(d), A, A, A + 2, A, None, A, None, A, A, None, 0, None, None, None) == lbt.ERR_ALIGNMENT
    assert f(at(d), A, A, None, A, None, A, None, A, None, A, 48, A, None, None) == lbt.ERR_INVALID_ARG    # codes narrower than the row
    assert f(at(d), A, A, None, A, None, A, None, A, None, A, 72, A, None, None) == lbt.ERR_ALIGNMENT
    assert f(at(d), A, A, None, A, None, A, None, A, None, A, 64, None, None, None) == lbt.ERR_INVALID_ARG  # codes without scales
    assert f(at(d), A, A, None, A, None, A, None, A, A, None, 0, None, A + 4, None) == lbt.ERR_ALIGNMENT
    assert f(at(d), A, A, None, A, A, A, None, A, A, None, 0, None, None, None) == lbt.ERR_INVALID_ARG     # an RMS norm has no bias
    tail = lambda **k: [k.get(n) for n in ("dgate", "dw_post", "db_post", "dw_pre", "db_pre")]  # noqa: E731
    big = 1 << 40
    assert b(at(d), None, None, A, A, None, A, None, A, A, A, A, *tail(), A, big, None) == lbt.ERR_INVALID_ARG   # no gradient comes in
    assert b(at(d), A, A, A, A, None, A, None, A, None, A, A, *tail(), A, big, None) == lbt.ERR_INVALID_ARG      # no statistics
    assert b(at(d), A, A, A, A, None, A, None, A, A, A, A, *tail(dgate=A), A, big, None) == lbt.ERR_INVALID_ARG  # no gate
    assert b(at(d), A, A, A, A, None, A, None, A, A, A, A, *tail(db_pre=A), A, big, None) == lbt.ERR_INVALID_ARG  # an RMS norm's bias
    assert b(at(d), A, A, A, A, None, A, None, A, A, A, A, *tail(), None, big, None) == lbt.ERR_WORKSPACE
    assert b(at(d), A, A, A, A, None, A, None, A, A, A, A, *tail(), A, 512, None) == lbt.ERR_WORKSPACE
    d = _desc(M=4, post_norm=0)
    assert b(at(d), A, A, A, A, None, A, None, A, A, A, A, *tail(dw_post=A), A, big, None) == lbt.ERR_INVALID_ARG


@pytest.mark.parametrize("change,want", [
    ({}, lbt.OK), ({"step": 0}, lbt.ERR_INVALID_ARG), ({"beta1": 1.0}, lbt.ERR_INVALID_ARG), ({"beta2": -0.5}, lbt.ERR_INVALID_ARG),
    ({"eps": float("nan")}, lbt.ERR_INVALID_ARG), ({"state_bits": 16}, lbt.ERR_UNSUPPORTED_BITS), ({"n": 5, "p": None}, lbt.ERR_INVALID_ARG),
    ({"n": 5, "m_scale": None}, lbt.ERR_INVALID_ARG), ({"n": 5, "p_type": 4}, lbt.ERR_INVALID_ARG), ({"n": 5, "p": A + 2}, lbt.ERR_ALIGNMENT),
    ({"n": 5, "v_scale": A + 2}, lbt.ERR_ALIGNMENT), ({"n": 5, "state_bits": 32, "m": A + 1}, lbt.ERR_ALIGNMENT), ({"n": (1 << 40) + 1}, lbt.ERR_UNSUPPORTED)])
def test_adamw(change, want):
    h = lbt.AdamwHyper(0.9, 0.999, 1e-8, 1, 8, 0)
    t = (lbt.AdamwTensor * 1)(lbt.AdamwTensor(A, A, A, A, A, A, 0, 1e-3, 0.0, lbt.F32, lbt.F32))
    for k, v in change.items():
        setattr(h if hasattr(h, k) else t[0], k, v)
    assert lbt.lib().lbt_adamw_step(t, 1, C.addressof(h), None, None, None) == want
    assert lbt.lib().lbt_adamw_step(None, 1, C.addressof(h), None, None, None) == lbt.ERR_INVALID_ARG
    assert lbt.lib().lbt_adamw_step(t, 0, None, None, None, None) == lbt.ERR_INVALID_ARG


def test_a_refused_step_does_not_count():
    bad = lm.AdamW([], [], betas=(1.0, 0.9), step=3)
    for _ in range(2):
        with pytest.raises(lbt.LbtError):
            bad.step(stream=0)
    assert bad.hyper.step == bad.taken() == 3
    good = lm.AdamW([], [], step=3)   # (no tensors: nothing is launched)
    good.step(stream=0)
    assert good.hyper.step == good.taken() == 4


# ---------------------------------------------------------------------------------------------- several devices, without any
class _Tensor:
    """A contiguous tensor as the layers see one on a CUDA device: nothing behind its address."""

    def __init__(self, shape, dtype, index):
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, index
        self.device = torch.device("cpu")   # where a layer makes its scratch

    def get_device(self):
        return self.index

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return A


class _Devices:
    """Two CUDA devices as torch and the library see them: which one is current, and which one each call was made on."""

    def __init__(self, monkeypatch):
        self.current, self.calls = 0, []
        monkeypatch.setattr(lbt, "_device", lambda: self.current)
        monkeypatch.setattr(lbt, "_current_raw_stream", lambda index: 0)
        monkeypatch.setattr(lbt, "lib", lambda: self)
        monkeypatch.setattr(torch.cuda, "device", self.enter)
        monkeypatch.setattr(torch.cuda, "stream", self.enter)
        monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False)

    @contextlib.contextmanager
    def enter(self, where):
        before = self.current
        if isinstance(where, int):
            self.current = where
        elif hasattr(where, "device_index"):
            self.current = where.device_index
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


def _layer(index):
    layer = lm.Linear8.__new__(lm.Linear8)
    with torch.cuda.device(index):
        layer._set(_Tensor((32, 64), torch.int8, index), _Tensor((32,), torch.float32, index), 64, None)
    layer.status = _Tensor((1,), torch.int32, index)
    return layer


def test_calls_launch_on_their_tensors_device(monkeypatch):
    devices = _Devices(monkeypatch)
    x, y = (_Tensor(shape, torch.bfloat16, 1) for shape in ((5, 64), (5, 32)))
    q, s = _Tensor((5, 64), torch.int8, 1), _Tensor((5,), torch.float32, 1)
    layer = _layer(1)
    layer._space[0] = (1 << 20, _Tensor((1 << 20,), torch.uint8, 1))
    layer.forward(x, out=y)
    layer.forward(x, out=y, keep=True)
    layer.forward_codes(q, s, out=y, keep=True)   # (its codes are the ones kept)
    layer.backward(y, dx=x, need_dw=False)
    layer.load_weight(_Tensor((32, 64), torch.float32, 1))
    norm = lm.ResNorm(64)
    norm.forward(x, x, out=(x, x))
    assert devices.calls and {index for _, index in devices.calls} == {1} and devices.current == 0
    # on a stream: the stream's device
    stream = types.SimpleNamespace(device_index=1, cuda_stream=7)
    layer.forward(x, out=y, stream=stream)
    assert {index for _, index in devices.calls} == {1} and devices.current == 0


def test_operands_on_several_devices_are_refused(monkeypatch):
    devices = _Devices(monkeypatch)
    t = lambda shape, index, dtype=torch.bfloat16: _Tensor(shape, dtype, index)  # noqa: E731
    layer = _layer(1)
    codes = lambda index: (t((5, 64), index, torch.int8), t((5,), index, torch.float32))  # noqa: E731
    vec = lambda index: t((64,), index, torch.float32)  # noqa: E731
    away = types.SimpleNamespace(device_index=0, cuda_stream=7)
    norm = lm.ResNorm(64, w_pre=vec(0))
    q_w, s_w = t((32, 64), 1, torch.int8), t((32,), 1, torch.float32)
    for bad in (lambda: layer.forward(t((5, 64), 0), out=t((5, 32), 0)), lambda: layer.forward(t((5, 64), 1), out=t((5, 32), 0)),
                lambda: layer.forward(t((5, 64), 1), out=t((5, 32), 1), stream=away), lambda: layer.forward_codes(*codes(0), out=t((5, 32), 1)),
                lambda: layer.load_weight(t((32, 64), 0, torch.float32)), lambda: layer.forward(t((5, 64), -1), out=t((5, 32), 1)),
                lambda: norm.forward(t((5, 64), 1), t((5, 64), 1), out=(t((5, 64), 1),) * 2),
                lambda: norm.forward(t((5, 64), 0), t((5, 64), 1), out=(t((5, 64), 0),) * 2),
                lambda: norm.forward(t((5, 64), 0), t((5, 64), 0), vec(1), out=(t((5, 64), 0),) * 2),
                lambda: lm.ResNorm(64, w_pre=vec(0), w_post=vec(1)), lambda: lm.AdamW([vec(0), vec(1)], [vec(0), vec(1)], [vec(0)] * 2, [vec(0)] * 2),
                lambda: lm.AdamW([vec(0)], [vec(1)], [vec(0)], [vec(0)]),
                lambda: lbt.rows8_quantize(t((32, 64), 1, torch.float32), q_w, s_w)):   # (the binding itself enters no device)
        with pytest.raises(ValueError):
            bad()
    assert not devices.calls


def test_threads_that_share_a_layer_take_turns(monkeypatch):
    """A forward pass enqueues the quantizer and the product that reads its codes from the layer's scratch: between the two no other
    thread's pass may use the same scratch."""
    devices = _Devices(monkeypatch)
    layer = _layer(0)
    layer._space[0] = (1 << 20, _Tensor((1 << 20,), torch.uint8, 0))
    inside, overlaps, entered = [], [], threading.Event()

    def call(scratch):
        overlaps.extend(s for s in inside if s == scratch)
        inside.append(scratch)
        (entered.wait if len(inside) == 1 else entered.set)(*([0.3] if len(inside) == 1 else []))   # the first one stays for the second
        inside.remove(scratch)
        return lbt.OK

    devices.lbt_linear8_forward = lambda *a: call(a[12])    # (q_x)
    devices.lbt_linear8_backward = lambda *a: call(a[18])   # (the workspace)
    x, y = _Tensor((5, 64), torch.bfloat16, 0), _Tensor((5, 32), torch.bfloat16, 0)

    def both(work):
        entered.clear()
        threads = [threading.Thread(target=work) for _ in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join(10)

    both(lambda: layer.forward(x, out=y))
    assert not overlaps
    layer.kept = (_Tensor((5, 64), torch.int8, 0), _Tensor((5,), torch.float32, 0))
    both(lambda: layer.backward(y, dx=x, need_dw=False))
    assert not overlaps


def test_a_captured_call_keeps_no_scratch(monkeypatch):
    """Memory that a captured call takes belongs to its graph: kept for later calls it would go when they need more, or be shared with a
    replay.  Outside of a capture it is kept."""
    devices = _Devices(monkeypatch)
    devices.lbt_linear8_backward = devices.lbt_resnorm_backward = lambda *a: lbt.OK
    x, y = _Tensor((5, 64), torch.bfloat16, 0), _Tensor((5, 32), torch.bfloat16, 0)
    monkeypatch.setattr(lbt, "linear8_backward", lambda *a: None)
    monkeypatch.setattr(lbt, "_at", lambda t, device=None: A)
    monkeypatch.setattr(lbt, "_current_raw_stream", lambda index: 7)
    for capturing in (True, False):
        monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: capturing)
        layer, norm = _layer(0), lm.ResNorm(64)
        layer.forward(x, out=y)
        layer.forward(x, out=y, keep=True)
        layer.backward(y, dx=x, need_dw=False)
        norm.forward(x, x, out=(x, x), keep=True)
        norm.backward(x, x, out={"dx": x, "dh": x})
        for kept in (layer._scratch, layer._own_kept, layer._space, norm._stats, norm._space):
            assert bool(kept) != capturing
        assert layer.kept is not None and norm.kept is not None


def test_scale_and_skip_of_a_step_have_their_types(monkeypatch):
    """The kernel reads four bytes of each: a flag of one byte or a scale of another type would be read with what lies beside it."""
    devices = _Devices(monkeypatch)
    vec = lambda dtype=torch.float32, n=1: _Tensor((n,), dtype, 0)  # noqa: E731
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: _Tensor((1,), torch.int64, 0))
    opt = lm.AdamW([vec(n=9)], [vec(n=9)], [vec(n=9)], [vec(n=9)])
    for bad in ({"skip": vec(torch.bool)}, {"skip": vec(torch.float32)}, {"skip": vec(torch.int64)}, {"skip": vec(torch.int32, 2)},
                {"grad_scale": vec(torch.float64)}, {"grad_scale": vec(torch.bfloat16)}, {"grad_scale": vec(torch.float32, 0)}):
        with pytest.raises(ValueError):
            opt.step(**bad)
    assert not devices.calls and opt.hyper.step == 0
    opt.step(grad_scale=vec(), skip=vec(torch.int32))
    assert len(devices.calls) == 1 and opt.hyper.step == 1
