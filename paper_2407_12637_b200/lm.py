"""Layers of a transformer's residual block on the library's kernels: `Linear8`, `Adapters`, `ResNorm`, `GradClip` and `AdamW`.

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


class Adapters:
    """Low-rank adapters beside a linear layer (a `Linear8` whose weights stay as they are): out[m] = base[m] + s_i (x[m] A_i^T) B_i for
    the tokens m of each run of neighbouring tokens with adapter i.

    a [adapters, rank, I], b [adapters, rank, O]: both rank first, of one type (the activations'); scale [adapters] fp32 (None: ones).
    Runs: offsets (runs + 1 ascending int32 on the device) and index (int32 [runs], an adapter each; -1: none).  Both None: all tokens
    are one run with adapter 0.  Rows of no run are left as they are."""

    def __init__(self, a, b, scale=None):
        if a.dim() != 3 or b.dim() != 3 or a.shape[:2] != b.shape[:2] or a.dtype != b.dtype or a.dtype not in lbt.TYPES:
            raise ValueError("a: [adapters, rank, I], b: [adapters, rank, O], of one type: fp32, bf16 or fp16")
        self.n, self.rank, self.I = a.shape
        self.O = b.shape[2]
        if not 1 <= self.rank <= lbt.MAX_RANK or min(self.n, self.I, self.O) < 1:
            raise ValueError(f"ranks of 1 to {lbt.MAX_RANK}, at least one adapter, input and output")
        self.a, self.b, self.scale, self.dtype, self.device = a, b, scale, a.dtype, a.get_device()
        with lbt._place(a):   # (addresses of the adapters' own tensors, whose storage stays)
            self._weights = (lbt._at(a), lbt._at(b), lbt._floats(scale, self.n, "scale"))
        self.status = torch.zeros(1, dtype=torch.int32, device=a.device)   # lbt.ERR_TIMEOUT if a bounded on-chip wait ran out (check)
        self._status = self.status.data_ptr()
        self.kept = None
        self._plans, self._own_kept, self._space = {}, {}, {}   # descriptors by sizes; by stream: h that is kept, workspace of the backward pass
        self._lock = threading.Lock()   # a backward pass is two launches that meet in the workspace (the library's call lets other threads run)

    def check(self):
        """Raises LbtError if a bounded on-chip wait ran out since the last check (waits for the device): see Linear8.check."""
        status = int(self.status)
        if status:
            self.status.zero_()
            raise lbt.LbtError(status, "Adapters")

    def _runs(self, offsets, index):
        if offsets is None and index is None:
            return 0, 0, 0
        if offsets is None or index is None or offsets.dtype != torch.int32 or index.dtype != torch.int32 or offsets.numel() != index.numel() + 1:
            raise ValueError("offsets: int32, one more than index; index: int32, an adapter for each run")
        return index.numel(), lbt._at(offsets, self.device), lbt._at(index, self.device)

    def _plan(self, names, acts, widths, runs):
        """Addresses of the activations (None: 0) and the descriptor of a call on tensors of these sizes."""
        addresses, lds, M = [], [], None
        for name, t, width in zip(names, acts, widths):
            if t is None:
                addresses.append(0)
                lds.append(0)
                continue
            address, _, ld, rows = lbt._rows(t, name, width, self.device)
            if t.dtype != self.dtype or (M is not None and rows != M):
                raise ValueError(f"{name}: one row per token, of the adapters' type {self.dtype}")
            if ld < width:   # (a leading dimension of 0 stands for the row's length in the descriptor)
                raise ValueError(f"{name}: rows that do not overlap")
            M = rows
            addresses.append(address)
            lds.append(ld)
        key = (M, runs, *names, *lds)
        plan = self._plans.get(key)
        if plan is None:
            d = lbt.AdaptersDesc(M, self.I, self.O, runs, self.n, self.rank, lbt.TYPES[self.dtype], 0)
            for name, ld in zip(names, lds):
                setattr(d, "ld_" + name, ld)
            if len(self._plans) >= 256:   # many lengths: the plans are cheap to make again
                self._plans.clear()
            plan = self._plans[key] = (d, C.addressof(d), lbt.adapters_workspace_bytes(d))
        return M, addresses, plan

    def forward(self, x, base, offsets=None, index=None, out=None, keep=False, stream=None):
        """out for x [M, I] and base [M, O] (the layer's output; out None: added in place).  keep: x, the runs and h stay for `backward`,
        until the next forward pass with keep=True; x is then not overwritten by out."""
        on = x.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(x, stream):
                return self.forward(x, base, offsets, index, out, keep)
        if on != self.device:
            raise ValueError(f"the adapters are on device {self.device}")
        out = base if out is None else out
        runs, at_offsets, at_index = self._runs(offsets, index)
        M, at, plan = self._plan(("x", "base", "out"), (x, base, out), (self.I, self.O, self.O), runs)   # (holds the descriptor while the library reads it)
        if keep and at[0] == at[2] and lbt._in_place_of(out, x):
            raise ValueError("out in the place of x, which backward reads")
        raw, h = lbt._current_raw_stream(on), None
        if keep:   # a buffer for each stream, shared by one forward pass after the other
            held = not _capturing(raw)
            h = self._own_kept.get(raw) if held else None
            if h is None or h.shape[0] != M:
                h = torch.empty(M, self.rank, dtype=torch.float32, device=x.device)
                if held:
                    self._own_kept[raw] = h
        a, b, scale = self._weights
        status = lbt.lib().lbt_adapters_forward(plan[1], at[0], a, b, scale, at_offsets, at_index, at[1], at[2], h.data_ptr() if keep else 0, self._status, raw)
        if status:
            raise lbt.LbtError(status, "lbt_adapters_forward")
        if keep:
            self.kept = (x, h, offsets, index)
        return out

    def backward(self, dy, dbase=None, dx=None, da=None, db=None, grad_dtype=torch.float32, stream=None):
        """{"dx", "da", "db"} of the last forward pass with keep=True.  dbase: the layer's gradient of x, to which the adapters' is
        added (dx None: in place); without it there is no dx.  da, db: buffers to write into, else new ones of grad_dtype (fp32, or the adapters' type)."""
        if self.kept is None:
            raise RuntimeError("backward needs a forward pass with keep=True")
        on = dy.get_device()
        if stream is not None or on != lbt._device():
            with lbt._place(dy, stream):
                return self.backward(dy, dbase, dx, da, db, grad_dtype)
        if on != self.device:
            raise ValueError(f"the adapters are on device {self.device}")
        x, h, offsets, index = self.kept
        if dx is not None and dbase is None:
            raise ValueError("dx is the layer's gradient dbase and the adapters' part: it needs dbase")
        dx = dbase if dx is None else dx
        kinds = {t.dtype for t in (da, db) if t is not None} or {grad_dtype}
        if len(kinds) != 1 or not kinds <= {torch.float32, self.dtype}:
            raise ValueError("da and db: both fp32, or both of the adapters' type")
        kind = kinds.pop()
        out = {"dx": dx} if dx is not None else {}
        for name, given, like in (("da", da, self.a), ("db", db, self.b)):
            out[name] = torch.empty_like(like, dtype=kind) if given is None else given
            if out[name].shape != like.shape:
                raise ValueError(f"{name}: of the shape {tuple(like.shape)}")
        runs, at_offsets, at_index = self._runs(offsets, index)
        M, at, (held_desc, desc, size) = self._plan(("dy", "x", "dbase", "dx"), (dy, x, dbase, dx), (self.O, self.I, self.I, self.I), runs)
        raw = lbt._current_raw_stream(on)
        at_da, at_db = lbt._at(out["da"], on), lbt._at(out["db"], on)
        a, b, scale = self._weights
        with self._lock:
            held = not _capturing(raw)
            ws = self._space.get(raw) if held else None
            if ws is None or ws.numel() < size:
                ws = torch.empty(size, dtype=torch.uint8, device=dy.device)
                if held:
                    self._space[raw] = ws
            status = lbt.lib().lbt_adapters_backward(desc, at[0], at[1], h.data_ptr(), a, b, scale, at_offsets, at_index, at[2], at[3], at_da, at_db,
                                                     lbt.TYPES[kind], self._status, ws.data_ptr(), size, raw)
        if status:
            raise lbt.LbtError(status, "lbt_adapters_backward")
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
        self._space, self._stats = {}, {}   # device and stream (0 on each device) -> workspace of the backward pass, statistics that were kept

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
        if min(l for l, a in zip(lds, acts) if a is not None) < self.dim:   # (0 stands for the row's length in the descriptor)
            raise ValueError("rows that do not overlap")
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
        at, plan = self._plan(names, acts, gate, rows_per_gate, on)   # (holds the descriptor while the library reads it)
        raw, stats = lbt._current_raw_stream(on), None
        if keep:   # a buffer for each stream, shared by one forward pass after the other
            held = not _capturing(raw)
            stats = self._stats.get((on, raw)) if held else None
            if stats is None or stats.shape[0] != x.shape[0]:
                stats = torch.empty(x.shape[0], 4, dtype=torch.float32, device=x.device)
                if held:
                    self._stats[on, raw] = stats
        w_post, b_post, w_pre, b_pre = self._params
        status = lbt.lib().lbt_resnorm_forward(plan[1], at[0], at[1], lbt._at(gate, on) if gate is not None else 0, w_post, b_post, w_pre, b_pre, at[2], at[3] if y is not None else 0,
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
        at, (held_desc, desc, size) = self._plan(("x", "h", "dr", "dy", "dx", "dh"), (x, h, dr, dy, out["dx"], out["dh"]), gate, rows_per_gate, on)
        raw = lbt._current_raw_stream(on)
        held = not _capturing(raw)
        ws = self._space.get((on, raw)) if held else None
        if ws is None or ws.numel() < size:
            ws = torch.empty(size, dtype=torch.uint8, device=x.device)
            if held:
                self._space[on, raw] = ws
        w_post, b_post, w_pre, _ = self._params
        status = lbt.lib().lbt_resnorm_backward(desc, at[2], at[3], at[0], at[1], lbt._at(gate, on) if gate is not None else 0, w_post, b_post, w_pre, stats.data_ptr(), at[4], at[5],
                                                *grads, ws.data_ptr(), size, raw)
        if status:
            raise lbt.LbtError(status, "lbt_resnorm_backward")
        return out


class GradClip:
    """The norm of all gradients in `grads` (fixed storage, read where it lay when the object was made: gradients that are allocated anew
    need a new object), and clipping to `max_norm` by it.

    `measure` leaves `norm`, `scale` = min(1, max_norm / norm), `skip` (1: a gradient is not finite) and each tensor's norm in `norms`,
    all on the device; scale and skip go to AdamW.step(grad_scale=clip.scale, skip=clip.skip), which then needs no pass over the
    gradients more than it makes anyway.  `clip` also writes the clipped gradients, for an optimizer that takes them as they are: into
    `out` (tensors of the gradients' sizes, of any type), by default in place; with skip set it writes nothing.  Outputs overlap neither
    each other nor the other gradients.  An object is used by one thread and one stream at a time."""

    def __init__(self, grads, max_norm=float("inf"), out=None):
        n = len(grads)
        if out is not None and len(out) != n:
            raise ValueError("one output for each gradient")
        if not max_norm > 0:
            raise ValueError("max_norm is positive")
        self.grads, self.out, self.max_norm = list(grads), list(out) if out is not None else list(grads), float(max_norm)
        self.device = self.grads[0].get_device() if n else None
        if n and self.device < 0:
            raise ValueError("gradients are CUDA tensors")
        self.table = (lbt.GradTensor * n)()
        spans = []   # first byte, end, whether it is written
        for e, g, o in zip(self.table, self.grads, self.out):
            kind, count, at = lbt.TYPES.get(g.dtype), g.numel(), lbt._at(g, self.device)
            to_kind, to = (kind, at) if o is g else (lbt.TYPES.get(o.dtype), lbt._at(o, self.device))
            if kind is None or to_kind is None or (o is not g and count != o.numel()):
                raise ValueError("gradients and outputs: fp32, bf16 or fp16, of equal sizes")
            e.g, e.out, e.n, e.g_type, e.out_type = at, to, count, kind, to_kind
            if count:
                if at == to and kind != to_kind:
                    raise ValueError("an output in its gradient's place has its type")
                spans.append((to, to + (count << 2 if to_kind == lbt.F32 else count << 1), True))
                if at != to:
                    spans.append((at, at + (count << 2 if kind == lbt.F32 else count << 1), False))
        end, end_written = 0, 0   # of the spans so far
        for first, last, written in sorted(spans):
            if first < (end if written else end_written):
                raise ValueError("an output lies in its gradient's place or apart from all others: a gradient given twice would be clipped twice, another's might be read after it was written")
            end, end_written = max(end, last), max(end_written, last) if written else end_written
        where = self.grads[0].device if n else "cpu"
        self._result = torch.zeros(4, dtype=torch.int32, device=where)
        parts = self._result.view(torch.float32)
        self.norm, self.scale, self.skip = parts[0:1], parts[1:2], self._result[2:3]
        self.norms = torch.zeros(n, dtype=torch.float32, device=where)
        if n == 0:
            self.scale.fill_(1.0)
        else:
            with lbt._place(self.grads[0]):
                self._addresses = (lbt._at(self._result), lbt._at(self.norms))
            self._bytes, self._space = lbt.grad_norm_workspace_bytes(self.table), {}

    def measure(self, grad_scale=None, stream=None):
        """Enqueues the measurement; returns `norm` (a device float).  grad_scale: device float that the gradients are still to be
        multiplied by (a loss scale's reciprocal): norm is of the products, and `scale` contains it."""
        if not self.grads:
            return self.norm
        if stream is not None or self.device != lbt._device():
            with lbt._place(self.grads[0], stream):
                return self.measure(grad_scale)
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1):
            raise ValueError("grad_scale: one fp32 value")
        raw = lbt._current_raw_stream(self.device)
        held = not _capturing(raw)
        ws = self._space.get(raw) if held else None
        if ws is None:
            ws = torch.empty(self._bytes, dtype=torch.uint8, device=self.norms.device)
            if held:
                self._space[raw] = ws
        result, norms = self._addresses
        status = lbt.lib().lbt_grad_norm(self.table, len(self.table), self.max_norm, lbt._at(grad_scale, self.device) if grad_scale is not None else 0,
                                         result, norms, ws.data_ptr(), self._bytes, raw)
        if status:
            raise lbt.LbtError(status, "lbt_grad_norm")
        return self.norm

    def clip(self, grad_scale=None, stream=None):
        """`measure`, and the gradients times `scale` into `out`."""
        if not self.grads:
            return self.norm
        if stream is not None or self.device != lbt._device():
            with lbt._place(self.grads[0], stream):
                return self.clip(grad_scale)
        self.measure(grad_scale)
        status = lbt.lib().lbt_grad_clip(self.table, len(self.table), self._addresses[0], lbt._current_raw_stream(self.device))
        if status:
            raise lbt.LbtError(status, "lbt_grad_clip")
        return self.norm


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
