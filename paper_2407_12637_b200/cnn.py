"""Layers between the quantized convolutions on the library's kernels: `GroupNorm`.

As in `lm`, an object keeps what a program keeps between calls (parameters, scratch for each stream) and every step of arithmetic
runs in the library (`lbt`); outputs may be handed in, work is enqueued on `stream` (default: torch's current stream).  Threads may
share an object's forward passes without `keep`; what `keep` holds for `backward` belongs to one thread at a time.
"""
from __future__ import annotations

import ctypes as C
import threading

import torch

from . import lbt
from .lm import _capturing

ACTS = {"none": lbt.ACT_NONE, "relu": lbt.ACT_RELU, "silu": lbt.ACT_SILU}


_LAYOUTS = {}   # (shape, strides) of tensors -> distance of pixels, images and pixels


def _layout(shape, strides, name):
    channels = shape[-1]
    if channels > 1 and strides[-1] != 1:
        raise ValueError(f"{name}: channels last (contiguous)")
    ld, pixels, images = channels, 1, shape[0]
    for size in shape[1:-1]:
        pixels *= size
    if images * pixels > 0:
        step = None   # what the next larger dimension's stride has to be
        for size, stride in zip(reversed(shape[:-1]), reversed(strides[:-1])):
            if size == 1:
                continue
            if step is None:
                ld, step = stride, stride
            elif stride != step:
                raise ValueError(f"{name}: pixels and images evenly spaced")
            step *= size
        if ld < channels:
            raise ValueError(f"{name}: pixels that do not overlap")
    return ld, images, pixels


def _images(t, name, channels, device):
    """Address, element type, distance of pixels, images and pixels of a channels-last tensor [N, ..., C] whose pixels lie evenly spaced."""
    kind, shape = lbt.TYPES.get(t.dtype), t.shape
    if kind is None or len(shape) < 2 or t.get_device() != device or shape[-1] != channels:
        raise ValueError(f"{name}: a CUDA tensor [N, ..., {channels}] of fp32, bf16 or fp16, on the device of the call")
    key = (shape, t.stride())
    layout = _LAYOUTS.get(key)
    if layout is None:
        layout = _layout(*key, name)
        if len(_LAYOUTS) >= 256:   # many sizes: they are cheap to look at again
            _LAYOUTS.clear()
        _LAYOUTS[key] = layout
    ld, images, pixels = layout
    return t.data_ptr(), kind, ld, images, pixels


class GroupNorm:
    """y = act(w (x - mean) / sqrt(var + eps) + b) on channels-last images [N, ..., C], mean and variance of each image over each of
    `groups` groups of neighbouring channels at all pixels.  act: "none", "relu" or "silu".  weight, bias: [C] of one type (None: ones, zeros)."""

    def __init__(self, channels: int, groups: int, weight=None, bias=None, eps=1e-5, act="none"):
        if channels < 1 or groups < 1 or channels % groups:
            raise ValueError("channels: a multiple of groups")
        if act not in ACTS:
            raise ValueError('act: "none", "relu" or "silu"')
        given = [p for p in (weight, bias) if p is not None]
        if any(p.numel() != channels or p.dtype != given[0].dtype or p.dtype not in lbt.TYPES for p in given):
            raise ValueError(f"parameters are vectors of {channels} values of one type")
        self.channels, self.groups, self.eps, self.act = int(channels), int(groups), float(eps), act
        self.weight, self.bias, self.kept = weight, bias, None
        self.param_dtype = given[0].dtype if given else torch.float32
        self.device = given[0].get_device() if given else None
        if given:
            with lbt._place(given[0]):   # (the layer's own tensors, whose storage stays)
                self._params = (lbt._at(weight), lbt._at(bias))
        else:
            self._params = (0, 0)
        self._plans, self._stats, self._space = {}, {}, {}   # descriptors by sizes; by stream (without parameters by device and stream: the default one is 0 on each): statistics that are kept, workspace
        self._lock = threading.Lock()   # a pass is two launches that meet in the workspace (the library's call lets other threads run)

    def _plan(self, names, acts, on):
        if self.device is not None and on != self.device:
            raise ValueError(f"the norm's parameters are on device {self.device}")
        addresses, lds, like = [], [], None
        for name, t in zip(names, acts):
            if t is None:
                addresses.append(0)
                lds.append(0)
                continue
            address, kind, ld, images, pixels = _images(t, name, self.channels, on)
            if like is None:
                like = (kind, images, pixels)
            elif like != (kind, images, pixels):
                raise ValueError(f"{name}: of the size and type of {names[0]}")
            addresses.append(address)
            lds.append(ld)
        key = (*like, *names, *lds)
        plan = self._plans.get(key)
        if plan is None:
            kind, images, pixels = like
            d = lbt.GroupnormDesc(images, pixels, self.channels, self.groups, kind, lbt.TYPES[self.param_dtype], ACTS[self.act], self.eps)
            for name, ld in zip(names, lds):
                setattr(d, "ld_" + name, ld)
            if len(self._plans) >= 256:   # many sizes: the plans are cheap to make again
                self._plans.clear()
            plan = self._plans[key] = (d, C.addressof(d), lbt.groupnorm_workspace_bytes(d))
        return addresses, plan

    def _workspace(self, place, held, size, device):
        ws = self._space.get(place) if held else None
        if ws is None or ws.numel() < size:
            ws = torch.empty(size, dtype=torch.uint8, device=device)
            if held:
                self._space[place] = ws
        return ws

    def _forward(self, x, y, q, bits, clip, scale, keep, on):
        at, (held_desc, desc, size) = self._plan(("x", "y"), (x, y), on)
        if keep and at[0] == at[1] and lbt._in_place_of(y, x):
            raise ValueError("out in the place of x, which backward reads")
        raw, stats = lbt._current_raw_stream(on), None
        held, place = not _capturing(raw), raw if self.device is not None else (on, raw)
        with self._lock:
            if keep:   # a buffer for each stream, shared by one forward pass after the other
                stats = self._stats.get(place) if held else None
                if stats is None or stats.shape[0] != x.shape[0]:
                    stats = torch.empty(x.shape[0], self.groups, 2, dtype=torch.float32, device=x.device)
                    if held:
                        self._stats[place] = stats
            ws = self._workspace(place, held, size, x.device)
            w, b = self._params
            status = lbt.lib().lbt_groupnorm_forward(desc, at[0], w, b, at[1], q.data_ptr() if q is not None else 0, bits,
                                                     lbt._floats(clip, 1, "clip", on) if q is not None else 0, scale.data_ptr() if q is not None else 0,
                                                     stats.data_ptr() if keep else 0, ws.data_ptr(), size, raw)
            if status:
                raise lbt.LbtError(status, "lbt_groupnorm_forward")
            if keep:
                self.kept = (x, stats)

    def forward(self, x, out=None, keep=False, stream=None):
        """y; keep: the statistics stay for `backward` (until the next forward pass with keep=True), which also needs x unchanged: out is then
        not in its place."""
        on = x.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(x, stream):   # outputs and scratch belong to the stream that uses them
                return self.forward(x, out, keep)
        y = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else out
        self._forward(x, y, None, 0, None, None, keep, on)
        return y

    def forward_codes(self, x, clip, bits=4, out=None, keep=False, stream=None):
        """(q, scale): y clipped to [0, clip] (a device float) as the unsigned codes of lbt.quantize_act, which lbt.qconv_forward reads; out:
        y itself too, where it is wanted.  Needs a multiple of 8 channels."""
        on = x.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(x, stream):
                return self.forward_codes(x, clip, bits, out, keep)
        if clip is None:
            raise ValueError("clip: one fp32 value")
        q = torch.empty((x.numel() + 1) // 2 if bits <= 4 else x.numel(), dtype=torch.uint8, device=x.device)
        scale = torch.empty(1, dtype=torch.float32, device=x.device)
        self._forward(x, out, q, bits, clip, scale, keep, on)
        return q, scale

    def backward(self, dy, dx=None, dw=None, db=None, stream=None):
        """{"dx"} and the gradients of the parameters that there are ("dw", "db") of the last forward pass with keep=True (dx, dw, db:
        buffers to write into)."""
        if self.kept is None:
            raise RuntimeError("backward needs a forward pass with keep=True")
        on = dy.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(dy, stream):
                return self.backward(dy, dx, dw, db)
        x, stats = self.kept
        out = {"dx": torch.empty_like(x, memory_format=torch.contiguous_format) if dx is None else dx}
        grads = []
        for name, given, p in (("dw", dw, self.weight), ("db", db, self.bias)):
            if p is None:
                grads.append(0)
                continue
            g = out[name] = torch.empty_like(p) if given is None else given
            if g.numel() != p.numel() or g.dtype != p.dtype:
                raise ValueError(f"{name}: {p.numel()} values of {p.dtype}")
            grads.append(lbt._at(g, on))
        at, (held_desc, desc, size) = self._plan(("dy", "x", "dx"), (dy, x, out["dx"]), on)
        raw = lbt._current_raw_stream(on)
        w, b = self._params
        with self._lock:
            ws = self._workspace(raw if self.device is not None else (on, raw), not _capturing(raw), size, dy.device)
            status = lbt.lib().lbt_groupnorm_backward(desc, at[0], at[1], w, b, stats.data_ptr(), at[2], *grads, ws.data_ptr(), size, raw)
        if status:
            raise lbt.LbtError(status, "lbt_groupnorm_backward")
        return out
