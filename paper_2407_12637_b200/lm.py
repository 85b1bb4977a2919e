"""Layers of a transformer's residual block on the library's kernels: `Linear8`, `ResNorm` and `AdamW`.

Each object keeps what a program keeps between calls (weight codes, parameters, moments, scratch for each stream) and the
plan of its calls; every step of arithmetic runs in the library (`lbt`).  Outputs may be handed in (`out`); otherwise they
come from torch's allocator.  Work is enqueued on `stream` (default: torch's current stream); tensors that another stream
made need that stream's event first, as with any torch call.  Threads may share an object's forward passes without `keep`;
what `keep` holds for `backward` belongs to one thread at a time.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import threading

import torch

from . import lbt


_NO_SCRATCH = (0, None, 0, 0)


def _capturing(raw) -> bool:
    """Whether `raw`, the current stream, is being captured (the default stream, 0, cannot be; asking takes 0.3 us).  What a captured
    call allocates belongs to its graph, and what a graph's replays write must not be handed on: such calls neither use nor leave
    scratch that is kept from call to call."""
    return raw != 0 and torch._C._cuda_isCurrentStreamCapturing()


class Linear8:
    """A linear layer y = x W^T + b whose three products run on 8-bit integers, with a scale for each output channel of W and
    for each token of x (and of the gradient)."""

    def __init__(self, in_features: int, out_features: int, bias=None, weight=None, device="cuda"):
        if in_features < 1 or out_features < 1:
            raise ValueError("in_features and out_features are positive")
        self._set(torch.zeros(out_features, lbt.pitch8(in_features), dtype=torch.int8, device=device),
                  torch.zeros(out_features, dtype=torch.float32, device=device), in_features, bias)
        if weight is not None:
            self.load_weight(weight)

    @classmethod
    def from_codes(cls, q_w, s_w, in_features: int, bias=None):
        """A served layer: codes [O, in_features rounded up to 16] (zeros behind in_features) and scales [O] as they are."""
        self = cls.__new__(cls)
        self._set(q_w, s_w, in_features, bias)
        return self

    def _set(self, q_w, s_w, in_features, bias):
        self.I, self.O, self.pitch = int(in_features), s_w.numel(), lbt.pitch8(in_features)
        self.device = q_w.get_device()
        with lbt._place(q_w):   # (addresses of the layer's own tensors, whose storage stays)
            self._weights = (lbt._codes(q_w, self.O, self.I, "q_w"), lbt._floats(s_w, self.O, "s_w"), lbt._floats(bias, self.O, "bias"))
        self.q_w, self.s_w, self.bias, self.kept = q_w, s_w, bias, None
        self.status = torch.zeros(1, dtype=torch.int32, device=q_w.device)   # lbt.ERR_TIMEOUT if a bounded on-chip wait ran out (check)
        self._status = self.status.data_ptr()
        # never shared between streams: codes and scales of x that are not kept (rows, buffer, two addresses), those that were
        # made here to be kept (shared by one forward pass after the other), and the backward pass's workspace
        self._scratch, self._own_kept, self._space = {}, {}, {}
        self._lock = threading.Lock()   # a pass uses them for as long as it enqueues (the library's call lets other threads run)

    def check(self):
        """Raises LbtError if a bounded on-chip wait of a product ran out since the last check (waits for the device): the outputs
        that hang on it were not written.  Nothing else says so: a training or serving loop checks now and then."""
        status = int(self.status)
        if status:
            self.status.zero_()
            raise lbt.LbtError(status, "Linear8")

    def load_weight(self, weight, stream=None):
        """Quantizes the weights [O, I] (after each optimizer step)."""
        if weight.shape != (self.O, self.I):
            raise ValueError(f"weight: {self.O} x {self.I}")
        on = weight.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(weight, stream):
                return self.load_weight(weight)
        lbt.rows8_quantize(weight, self.q_w, self.s_w)

    def forward(self, x, out=None, keep=False, stream=None):
        """y for x [M, I]; keep: the codes of x stay for `backward`, until the next forward pass with keep=True."""
        on = x.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(x, stream):   # outputs and scratch belong to the stream that uses them
                return self.forward(x, out, keep)
        if on != self.device:
            raise ValueError(f"the layer's weights are on device {self.device}")
        px, tx, ldx, M = lbt._rows(x, "x", self.I, on)
        y = x.new_empty((M, self.O)) if out is None else out
        py, ty, ldy, rows = lbt._rows(y, "y", self.O, on)
        if rows != M:
            raise ValueError("out: one row per row of x")
        raw = lbt._current_raw_stream(on)
        with self._lock:
            held = raw == 0 or not _capturing(raw)
            if keep:
                mine = self._own_kept.get(raw) if held else None
                if mine is None or mine[1].shape[0] != M:
                    mine = (torch.empty(M, self.pitch, dtype=torch.int8, device=x.device), torch.empty(M, dtype=torch.float32, device=x.device))
                    if held:
                        self._own_kept[raw] = mine
                pq, ps = mine[0].data_ptr(), mine[1].data_ptr()
            else:
                rows, space, pq, ps = self._scratch.get(raw, _NO_SCRATCH) if held else _NO_SCRATCH
                if rows < M:
                    rows = -(-M // 64) * 64
                    space = torch.empty(rows * (self.pitch + 4), dtype=torch.uint8, device=x.device)
                    pq, ps = space.data_ptr(), space.data_ptr() + rows * self.pitch
                    if held:
                        self._scratch[raw] = (rows, space, pq, ps)
            q_w, s_w, bias = self._weights
            status = lbt.lib().lbt_linear8_forward(px, tx, ldx, q_w, s_w, bias, py, ty, ldy, M, self.O, self.I, pq, ps, self._status, raw)
            if status:
                raise lbt.LbtError(status, "lbt_linear8_forward")
            if keep:
                self.kept = mine
        return y

    def forward_codes(self, q_x, s_x, out=None, dtype=torch.bfloat16, keep=False, stream=None):
        """y from codes and scales that another operator made (ResNorm.forward_codes)."""
        on = q_x.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(q_x, stream):
                return self.forward_codes(q_x, s_x, out, dtype, keep)
        if on != self.device:
            raise ValueError(f"the layer's weights are on device {self.device}")
        M = s_x.numel()
        y = torch.empty(M, self.O, dtype=dtype, device=q_x.device) if out is None else out
        py, ty, ldy, rows = lbt._rows(y, "y", self.O, on)
        if rows != M:
            raise ValueError("out: one row per row of codes")
        q_w, s_w, bias = self._weights
        status = lbt.lib().lbt_linear8_matmul(lbt._codes(q_x, M, self.I, "q_x", on), lbt._floats(s_x, M, "s_x", on), q_w, s_w, bias, py, ty, ldy,
                                              M, self.O, self.I, self._status, lbt._current_raw_stream(on))
        if status:
            raise lbt.LbtError(status, "lbt_linear8_matmul")
        if keep:
            self.kept = (q_x, s_x)
        return y

    def backward(self, dy, need_dx=True, need_dw=True, dw_dtype=torch.float32, dx=None, dw=None, dbias=None, stream=None):
        """{"dx", "dw", "dbias"} of the last forward pass with keep=True (dx, dw, dbias: buffers to write into; what has one
        is computed whatever need_dx and need_dw say, and a bias's gradient comes with dw)."""
        on = dy.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(dy, stream):
                return self.backward(dy, need_dx, need_dw, dw_dtype, dx, dw, dbias)
        if self.kept is None:
            raise RuntimeError("backward needs a forward pass with keep=True")
        q_x, s_x = self.kept
        if dy.shape[0] != s_x.numel():
            raise ValueError("dy: one row per token of the forward pass")
        out = {}
        if need_dx or dx is not None:
            out["dx"] = dx if dx is not None else dy.new_empty((dy.shape[0], self.I))
        if need_dw or dw is not None:
            out["dw"] = dw if dw is not None else dy.new_empty((self.O, self.I), dtype=dw_dtype)
        if dbias is not None or ("dw" in out and self.bias is not None):
            out["dbias"] = dbias if dbias is not None else torch.empty_like(self.s_w)
        raw = lbt._current_raw_stream(on)
        with self._lock:
            held = not _capturing(raw)
            size, space = self._space.get(raw, (0, None)) if held else (0, None)
            need = lbt.linear8_workspace_bytes(dy.shape[0], self.O, self.I)
            if size < need:
                space = torch.empty(need, dtype=torch.uint8, device=dy.device)
                if held:
                    self._space[raw] = (need, space)
            lbt.linear8_backward(dy, self.q_w, self.s_w, q_x, s_x, self.I, out.get("dx"), out.get("dw"), out.get("dbias"), space, self.status)
        return out


class ResNorm:
    """What happens between two blocks: r = scale_x x + scale_h gate N_post(h), y = N_pre(r), in one pass.

    kind: "rms" or "layer"; post_norm False: h enters as it is.  Parameters are vectors of `dim` values of one type (None: ones,
    or zeros for the biases).  A gate is passed to each call: [dim], [1, dim] for all rows, or [ceil(rows / rows_per_gate), dim]."""

    def __init__(self, dim: int, kind="rms", w_post=None, b_post=None, w_pre=None, b_pre=None, eps=1e-6, scale_x=1.0, scale_h=1.0,
                 post_norm=True):
        if kind not in ("rms", "layer"):
            raise ValueError('kind: "rms" or "layer"')
        self.dim, self.layer, self.post = int(dim), kind == "layer", bool(post_norm)
        self.w_post, self.b_post, self.w_pre, self.b_pre = w_post, b_post, w_pre, b_pre
        given = [p for p in (w_post, b_post, w_pre, b_pre) if p is not None]
        if any(p.numel() != dim or p.dtype != given[0].dtype or p.dtype not in lbt.TYPES for p in given):
            raise ValueError(f"parameters are vectors of {dim} values of one type")
        if not self.layer and (b_post is not None or b_pre is not None):
            raise ValueError("an RMS norm has no bias")
        self.param_dtype = given[0].dtype if given else None
        self.eps, self.scale_x, self.scale_h = float(eps), float(scale_x), float(scale_h)
        self.kept = None
        self.device = given[0].get_device() if given else None
        with lbt._place(given[0]) if given else contextlib.nullcontext():   # (the layer's own tensors, whose storage stays)
            self._params = tuple(lbt._at(p) for p in (w_post, b_post, w_pre, b_pre))
        self._plans = {}   # (rows, types, leading dimensions) -> descriptor and its workspace size
        self._space, self._stats = {}, {}   # stream -> workspace of the backward pass, statistics that were kept

    def _plan(self, names, acts, gate, rows_per_gate, on):
        """Addresses of the activations and the descriptor of a call on tensors of these sizes (checked each time)."""
        x = acts[0]
        if self.device is not None and on != self.device:
            raise ValueError(f"the norm's parameters are on device {self.device}")
        address, kind, ld, rows = lbt._rows(x, names[0], self.dim, on)
        dtype, addresses, lds = x.dtype, [address], [ld]
        for name, t in zip(names[1:], acts[1:]):
            if t is None:
                addresses.append(0)
                lds.append(0)
                continue
            address, t_kind, ld, t_rows = lbt._rows(t, name, self.dim, on)
            if t_rows != rows or t_kind != kind:
                raise ValueError(f"{name}: {rows} rows of {dtype}")
            addresses.append(address)
            lds.append(ld)
        pd = self.param_dtype or (gate.dtype if gate is not None else dtype)
        if gate is not None:
            gates = -(-rows // rows_per_gate) if rows_per_gate else 1
            if gate.dtype != pd or gate.numel() != gates * self.dim:
                raise ValueError(f"gate: {gates} x {self.dim} values of the parameters' type")
        key = (rows, dtype, pd, rows_per_gate, *names, *lds)
        plan = self._plans.get(key)
        if plan is None:
            d = lbt.ResnormDesc(rows, self.dim, rows_per_gate or 0, lbt.TYPES[dtype], lbt.TYPES[pd],
                                lbt.NORM_LAYER if self.layer else lbt.NORM_RMS, 1 if self.post else 0, self.eps, self.eps, self.scale_x,
                                self.scale_h)
            for name, ld in zip(names, lds):
                setattr(d, "ld_" + name, ld)
            if len(self._plans) >= 256:   # many lengths: the plans are cheap to make again
                self._plans.clear()
            plan = self._plans[key] = (d, C.addressof(d), lbt.resnorm_workspace_bytes(d))
        return addresses, plan

    def _forward(self, x, h, gate, rows_per_gate, r, y, q, q_scale, keep, on):
        names, acts = (("x", "h", "r", "y"), (x, h, r, y)) if y is not None else (("x", "h", "r"), (x, h, r))
        at, (_, desc, _) = self._plan(names, acts, gate, rows_per_gate, on)
        raw, stats = lbt._current_raw_stream(on), None
        if keep:   # a buffer for each stream, shared by one forward pass after the other
            held = not _capturing(raw)
            stats = self._stats.get(raw) if held else None
            if stats is None or stats.shape[0] != x.shape[0]:
                stats = torch.empty(x.shape[0], 4, dtype=torch.float32, device=x.device)
                if held:
                    self._stats[raw] = stats
        w_post, b_post, w_pre, b_pre = self._params
        status = lbt.lib().lbt_resnorm_forward(desc, at[0], at[1], lbt._at(gate, on) if gate is not None else 0, w_post, b_post, w_pre, b_pre, at[2], at[3] if y is not None else 0,
                                               q.data_ptr() if q is not None else 0, q.shape[1] if q is not None else 0,
                                               q_scale.data_ptr() if q is not None else 0, stats.data_ptr() if keep else 0, raw)
        if status:
            raise lbt.LbtError(status, "lbt_resnorm_forward")
        if keep:
            self.kept = (x, h, gate, rows_per_gate, stats)

    def forward(self, x, h, gate=None, rows_per_gate=0, out=None, keep=False, stream=None):
        """(r, y); keep: the statistics stay for `backward` (until the next forward pass with keep=True), which also needs x and h
        unchanged."""
        on = x.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(x, stream):   # outputs and scratch belong to the stream that uses them
                return self.forward(x, h, gate, rows_per_gate, out, keep)
        r, y = out if out is not None else (torch.empty_like(x), torch.empty_like(x))
        self._forward(x, h, gate, rows_per_gate, r, y, None, None, keep, on)
        return r, y

    def forward_codes(self, x, h, gate=None, rows_per_gate=0, out=None, keep=False, stream=None):
        """(r, q, scale): y as the 8-bit rows that Linear8.forward_codes takes."""
        on = x.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(x, stream):
                return self.forward_codes(x, h, gate, rows_per_gate, out, keep)
        r = torch.empty_like(x) if out is None else out
        q = x.new_empty((x.shape[0], lbt.pitch8(self.dim)), dtype=torch.int8)
        scale = x.new_empty(x.shape[0], dtype=torch.float32)
        self._forward(x, h, gate, rows_per_gate, r, None, q, scale, keep, on)
        return r, q, scale

    def backward(self, dr, dy, out=None, stream=None):
        """Gradients of the last forward pass with keep=True: {"dx", "dh"} and those of the parameters and the gate that there are
        ("dgate", "dw_post", "db_post", "dw_pre", "db_pre").  out: buffers to write some of them into, by name."""
        if self.kept is None:
            raise RuntimeError("backward needs a forward pass with keep=True")
        x, h, gate, rows_per_gate, stats = self.kept
        on = x.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(x, stream):
                return self.backward(dr, dy, out)
        given, out, grads = out or {}, {}, []
        for name in ("dx", "dh"):
            out[name] = given[name] if name in given else torch.empty_like(x)
        for name, p in (("dgate", gate), ("dw_post", self.w_post if self.post else None), ("db_post", self.b_post if self.post else None),
                        ("dw_pre", self.w_pre), ("db_pre", self.b_pre)):
            if p is not None:
                g = out[name] = given[name] if name in given else torch.empty_like(p)
                if g.numel() != p.numel() or g.dtype != p.dtype:
                    raise ValueError(f"{name}: {p.numel()} values of {p.dtype}")
                grads.append(lbt._at(g, on))
            else:
                grads.append(0)
        at, (_, desc, size) = self._plan(("x", "h", "dr", "dy", "dx", "dh"), (x, h, dr, dy, out["dx"], out["dh"]), gate, rows_per_gate, on)
        raw = lbt._current_raw_stream(on)
        held = not _capturing(raw)
        ws = self._space.get(raw) if held else None
        if ws is None or ws.numel() < size:
            ws = torch.empty(size, dtype=torch.uint8, device=x.device)
            if held:
                self._space[raw] = ws
        w_post, b_post, w_pre, _ = self._params
        status = lbt.lib().lbt_resnorm_backward(desc, at[2], at[3], at[0], at[1], lbt._at(gate, on) if gate is not None else 0, w_post, b_post, w_pre, stats.data_ptr(), at[4], at[5],
                                                *grads, ws.data_ptr(), size, raw)
        if status:
            raise lbt.LbtError(status, "lbt_resnorm_backward")
        return out


class AdamW:
    """AdamW over lists of parameter and gradient tensors (fixed storage, as the library's other calls write it), all in one launch.

    m, v: the moments' tensors; None: new ones, in fp32 or (state_bits=8) as e4m3 codes with a scale for each block of 256 elements
    (m, and the root of v).  With moments given, their type decides.  lr and weight_decay: one value, or one for each tensor."""

    def __init__(self, params, grads, m=None, v=None, m_scale=None, v_scale=None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01,
                 step=0, state_bits=8):
        n = len(params)
        if len(grads) != n:
            raise ValueError("one gradient for each parameter")
        if m is not None:
            state_bits = 32 if all(t.dtype == torch.float32 for t in m) else 8
        if state_bits not in (8, 32):
            raise ValueError("state_bits: 8 or 32")
        if state_bits == 8 and ((m is not None and m_scale is None) or (v is not None and v_scale is None)):
            raise ValueError("moments in 8 bits come with their scales (new ones would be 0, and the moments with them)")
        state = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        blocks = [-(-p.numel() // lbt.ADAMW_BLOCK) for p in params]
        new = lambda kind, sizes: [torch.zeros(s, dtype=kind, device=p.device) for s, p in zip(sizes, params)]  # noqa: E731
        self.params, self.grads = list(params), list(grads)
        self.m = list(m) if m is not None else new(state, [p.numel() for p in params])
        self.v = list(v) if v is not None else new(state, [p.numel() for p in params])
        self.m_scale = (list(m_scale) if m_scale is not None else new(torch.float32, blocks)) if state_bits == 8 else [None] * n
        self.v_scale = (list(v_scale) if v_scale is not None else new(torch.float32, blocks)) if state_bits == 8 else [None] * n
        lrs, wds = (list(x) if isinstance(x, (list, tuple)) else [x] * n for x in (lr, weight_decay))
        if any(len(x) != n for x in (self.m, self.v, self.m_scale, self.v_scale, lrs, wds)):
            raise ValueError("one of each for each parameter")
        self.device = self.params[0].get_device() if n else None
        if n and self.device < 0:
            raise ValueError("parameters are CUDA tensors")
        self.table = (lbt.AdamwTensor * n)()
        for i, (p, g) in enumerate(zip(self.params, self.grads)):
            if p.dtype not in lbt.TYPES or g.dtype not in lbt.TYPES or g.numel() != p.numel():
                raise ValueError("parameters and gradients: fp32, bf16 or fp16, of equal sizes")
            for t, size, kind in ((self.m[i], p.numel(), state), (self.v[i], p.numel(), state), (self.m_scale[i], blocks[i], torch.float32),
                                  (self.v_scale[i], blocks[i], torch.float32)):
                if t is not None and (t.numel() != size or t.dtype != kind):
                    raise ValueError(f"moments: {p.numel()} values of {state}; with 8 bits one fp32 scale for each {lbt.ADAMW_BLOCK}")
            e = self.table[i]
            e.p, e.g, e.m, e.v, e.m_scale, e.v_scale = (lbt._at(t, self.device) for t in (p, g, self.m[i], self.v[i], self.m_scale[i], self.v_scale[i]))
            e.n, e.lr, e.weight_decay, e.p_type, e.g_type = p.numel(), lrs[i], wds[i], lbt.TYPES[p.dtype], lbt.TYPES[g.dtype]
        self.hyper = lbt.AdamwHyper(betas[0], betas[1], eps, step, state_bits, 0)   # (its step counts the calls)
        # calls that were held back, counted once there may be some (a launch that need not look starts 0.5 us earlier)
        self.skipped, self._counting = torch.zeros(1, dtype=torch.int64, device=self.params[0].device) if n else None, False
        self._skipped = self.skipped.data_ptr() if n else 0
        self._replayed = False   # whether a step is in a captured graph

    def set_lr(self, lr):
        """One learning rate for all tensors, or one for each."""
        for e, x in zip(self.table, lr if isinstance(lr, (list, tuple)) else [lr] * len(self.table)):
            e.lr = x

    def step(self, grad_scale=None, skip=None, stream=None):
        """One step.  grad_scale: device float the gradients are multiplied by; skip: device int32, non-zero = leave everything (the
        step then counts for nothing: the next one corrects as this one would have)."""
        raw = stream
        if self.params:
            if stream is not None or self.device != lbt._device():
                with lbt._place(self.params[0], stream):
                    return self.step(grad_scale, skip)
            raw = lbt._current_raw_stream(self.device)
            if not self._replayed and raw != 0 and _capturing(raw):
                self._replayed = True
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1):
            raise ValueError("grad_scale: one fp32 value")
        if skip is not None and (skip.dtype != torch.int32 or skip.numel() != 1):
            raise ValueError("skip: one int32 value")
        if skip is not None or self._replayed:
            self._counting = True
        self.hyper.step += 1
        try:
            status = lbt.lib().lbt_adamw_step_ex(self.table, len(self.params), C.addressof(self.hyper), lbt._at(grad_scale, self.device) if grad_scale is not None else 0,
                                                 lbt._at(skip, self.device) if skip is not None else 0, self._skipped if self._counting else 0, raw)
            if status:
                raise lbt.LbtError(status, "lbt_adamw_step_ex")
        except Exception:   # refused: nothing was enqueued
            self.hyper.step -= 1
            raise
        if self._replayed:   # a graph holds this call's step: from the first capture on the host's count rests and the device's runs
            self.hyper.step -= 1
            self.skipped.sub_(1)

    def taken(self) -> int:
        """Steps taken so far, as `step` of a resumed optimizer (waits for the device)."""
        return self.hyper.step - (int(self.skipped) if self.params else 0)

    def moments(self):
        """The moments (m, v) as fp32 values, one tensor for each parameter (a checkpoint reader's view)."""
        if self.hyper.state_bits == 32:
            return self.m, self.v
        wide = lambda q, s: q.float() * s.repeat_interleave(lbt.ADAMW_BLOCK)[:q.numel()].view(q.shape)  # noqa: E731
        return ([wide(q, s) for q, s in zip(self.m, self.m_scale)], [wide(q, s).square() for q, s in zip(self.v, self.v_scale)])
