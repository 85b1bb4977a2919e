"""Cases of the transformer-side operators: linear8 (8-bit integer linear layer with a scale per token and channel),
resnorm (norm, gate, residual and norm in one pass) and adamw (AdamW over many tensors, states in 8 or 32 bits).

`run` computes them in plain torch operations in 32 bits (`own` false) or through the framework (`own` true)."""
import math
import random

import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token through a square projection: a chat session's decode step, latency counts
        {"name": "serve 1 x 4096 -> 4096", "op": "linear8", "M": 1, "I": 4096, "O": 4096, "dtype": "bfloat16", "bias": False},
        # a decode batch of 29 sequences: the weights are read once for all of them
        {"name": "serve 29 x 8192 -> 8192", "op": "linear8", "M": 29, "I": 8192, "O": 8192, "dtype": "float16", "bias": True},
        # a prompt of 2048 tokens through an up-projection
        {"name": "serve 2048 x 4096 -> 16384", "op": "linear8", "M": 2048, "I": 4096, "O": 16384, "dtype": "bfloat16", "bias": True},
        # one training step of the 8192^3 linear layer of the framework's benchmark
        {"name": "train 8192 x 8192 x 8192", "op": "linear8_train", "M": 8192, "I": 8192, "O": 8192, "dtype": "bfloat16", "bias": False},
        # a classifier head with odd sizes, all in fp32
        {"name": "train 1111 x 2047 -> 1000", "op": "linear8_train", "M": 1111, "I": 2047, "O": 1000, "dtype": "float32", "bias": True},
        # one token between two blocks
        {"name": "resnorm 1 x 4096", "op": "resnorm", "M": 1, "D": 4096, "dtype": "bfloat16", "pdtype": "bfloat16", "kind": "rms",
         "gate": "channel", "rows_per_gate": 1, "scale_x": 1.0, "scale_h": 1.0},
        # training on four sequences of 2048 tokens with a gate for each sequence
        {"name": "resnorm train 8192 x 4096", "op": "resnorm_train", "M": 8192, "D": 4096, "dtype": "bfloat16", "pdtype": "bfloat16",
         "kind": "rms", "gate": "rows", "rows_per_gate": 2048, "scale_x": 1.0, "scale_h": 0.5},
        # layer norms in fp32 on an odd width, one gate for all tokens
        {"name": "resnorm train 1003 x 1111", "op": "resnorm_train", "M": 1003, "D": 1111, "dtype": "float32", "pdtype": "float32",
         "kind": "layer", "gate": "channel", "rows_per_gate": 1, "scale_x": 0.9, "scale_h": 0.3},
        # from one block's output to the next block's projection, a decode batch of 64
        {"name": "block 64 x 4096 -> 8192", "op": "block", "M": 64, "D": 4096, "O": 8192, "dtype": "bfloat16", "pdtype": "bfloat16",
         "kind": "rms", "gate": "channel", "rows_per_gate": 1, "scale_x": 1.0, "scale_h": 1.0},
        # ResNet-18 with fp32 states: 62 tensors from 64 to 2.4 M elements
        {"name": "adamw 32 resnet18", "op": "adamw", "layout": "resnet18", "a": 0, "b": 0, "bits": 32, "dtype": "float32", "gdtype": "float32"},
        # eight transformer blocks of width 2048, 8-bit states, fp32 masters with bf16 gradients: 0.4 G elements
        {"name": "adamw 8 blocks 8 x 2048", "op": "adamw", "layout": "blocks", "a": 8, "b": 2048, "bits": 8, "dtype": "float32", "gdtype": "bfloat16"},
        # adapters: many small tensors of odd lengths (one element among them), bf16 weights
        {"name": "adamw 8 ragged 96", "op": "adamw", "layout": "ragged", "a": 96, "b": 20000, "bits": 8, "dtype": "bfloat16", "gdtype": "bfloat16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear8", "linear8_train", "resnorm", "resnorm_train", "block", "adamw"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if op in ("linear8", "linear8_train"):
        return {"op": op, "M": _log(rng, 1 if op == "linear8" else 32, 8192), "I": _log(rng, 256, 8192), "O": _log(rng, 256, 8192),
                "dtype": dtype, "bias": rng.random() < 0.5}
    if op == "adamw":
        layout = rng.choice(["blocks", "ragged"])
        a, b = (rng.randint(1, 8), 8 * rng.randint(32, 256)) if layout == "blocks" else (_log(rng, 1, 400), _log(rng, 10, 1000000))
        return {"op": op, "layout": layout, "a": a, "b": b, "bits": rng.choice([8, 32]), "dtype": rng.choice(["float32", "bfloat16"]),
                "gdtype": rng.choice(["float32", "bfloat16"])}
    if op == "block" and dtype == "float32":
        dtype = "bfloat16"   # 8-bit projections are served on 16-bit streams
    M = _log(rng, 1, 8192) if op != "block" else _log(rng, 1, 512)
    gate = rng.choice(["none", "channel", "rows"])
    c = {"op": op, "M": M, "D": _log(rng, 128, 8192), "dtype": dtype, "pdtype": dtype, "kind": rng.choice(["rms", "layer"]), "gate": gate,
         "rows_per_gate": _log(rng, 1, M) if gate == "rows" else 1, "scale_x": rng.choice([1.0, 0.8]), "scale_h": rng.choice([1.0, 0.25])}
    if op == "block":
        c["O"] = _log(rng, 256, 8192)
    return c


def _sizes(case):
    """The element counts of an AdamW case's tensors."""
    a, b = case["a"], case["b"]
    if case["layout"] == "resnet18":
        sizes, width_in = [64 * 3 * 49, 64, 64], 64
        for width in (64, 128, 256, 512):
            for block in range(2):
                sizes += [width * width_in * 9, width, width, width * width * 9, width, width]
                if width_in != width:
                    sizes += [width * width_in, width, width]
                width_in = width
        return sizes + [512 * 1000, 1000]
    if case["layout"] == "blocks":
        return ([b * b] * 4 + [4 * b * b] * 2 + [b] * 4 + [4 * b, b]) * a
    rng = random.Random(a * 1000003 + b)
    return [1] + [_log(rng, 1, b) for _ in range(a - 1)]


def _offsets(sizes):
    """Where each tensor begins in flat storage: at multiples of 256 elements."""
    at, offs = 0, []
    for n in sizes:
        offs.append(at)
        at += -(-n // 256) * 256
    return offs, at


def work(case):
    size = {"float32": 4, "bfloat16": 2, "float16": 2}
    e = size[case["dtype"]]
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        return {"bytes": n * (2 * e + size[case["gdtype"]] + (16 if case["bits"] == 32 else 4 + 16 / 256)), "flops": 15 * n}
    M = case["M"]
    if case["op"] == "linear8":
        I, O = case["I"], case["O"]
        return {"bytes": M * I * e + O * I + 4 * O + M * O * e, "flops": 2 * M * I * O}
    if case["op"] == "linear8_train":
        I, O = case["I"], case["O"]
        return {"bytes": M * I * e + 4 * O * I + M * O * e + M * O * e + M * I * e + 4 * O * I, "flops": 6 * M * I * O}
    D, gates = case["D"], {"none": 0, "channel": 1, "rows": -(-M // case["rows_per_gate"])}[case["gate"]]
    if case["op"] == "resnorm":
        return {"bytes": 4 * M * D * e + gates * D * e, "flops": 15 * M * D}
    if case["op"] == "resnorm_train":   # forward: x, h -> r, y; backward: dr, dy, x, h -> dx, dh
        return {"bytes": 10 * M * D * e + 3 * gates * D * e, "flops": 50 * M * D}
    return {"bytes": 3 * M * D * e + gates * D * e + D * case["O"] + M * case["O"] * e, "flops": 2 * M * D * case["O"]}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def _activations(g, M, D, dtype):
    """Normal activations with one channel in 64 that is ten times as large, as transformers' streams have."""
    big = torch.where(torch.rand(D, generator=g, device="cuda") < 1 / 64, 10.0, 1.0)
    return (torch.randn(M, D, generator=g, device="cuda") * big).to(dtype)


def _gradient(g, M, D, std, dtype):
    """Zero-centred with a long tail."""
    u = torch.rand(M, D, generator=g, device="cuda") - 0.5
    return (-torch.sign(u) * torch.log1p(-2 * u.abs() * (1 - 1e-6)) * std).to(dtype)


def _rows8(t):
    """Codes and scales of the rows of t (fp32)."""
    most = t.abs().amax(1, keepdim=True)
    inv = torch.where(most > 1e-36, 127.0 / most, 0.0)
    return torch.round(t * inv), torch.where(most > 1e-36, most / 127.0, 0.0)


def _weights(g, O, I, bias):
    """A served layer's weights: codes [O, I rounded up to 16] (zeros behind column I), scales, bias."""
    q, s = _rows8(_normal(g, O, I, std=0.02))
    codes = torch.zeros(O, -(-I // 16) * 16, dtype=torch.int8, device="cuda")
    codes[:, :I] = q.to(torch.int8)
    return codes, s.reshape(-1).contiguous(), _normal(g, O, std=0.1) if bias else None


def _inputs(case, seed):
    g, op, t = _gen(seed), case["op"], TYPES[case["dtype"]]
    if op == "linear8":
        M, I, O = case["M"], case["I"], case["O"]
        q, s, b = _weights(g, O, I, case["bias"])
        return {"x": _activations(g, M, I, t), "q_w": q, "s_w": s, "bias": b, "y": torch.empty(M, O, dtype=t, device="cuda")}
    if op == "linear8_train":
        M, I, O = case["M"], case["I"], case["O"]
        return {"x": _activations(g, M, I, t), "w": _normal(g, O, I, std=0.02), "bias": _normal(g, O, std=0.1) if case["bias"] else None,
                "dy": _gradient(g, M, O, 1e-2, t)}
    if op == "adamw":
        sizes = _sizes(case)
        offs, total = _offsets(sizes)
        real = torch.zeros(total + 1, device="cuda")    # 1 where an element belongs to a tensor
        real.index_add_(0, torch.tensor(offs, device="cuda"), torch.ones(len(sizes), device="cuda"))
        real.index_add_(0, torch.tensor([o + n for o, n in zip(offs, sizes)], device="cuda"), -torch.ones(len(sizes), device="cuda"))
        real = torch.cumsum(real[:-1].to(torch.int32), 0, dtype=torch.int32).bool()
        zero = torch.zeros((), device="cuda")
        p = torch.where(real, _normal(g, total, std=0.02), zero).to(t)
        grad = torch.where(real, _gradient(g, 1, total, 1e-3, torch.float32)[0], zero).to(TYPES[case["gdtype"]])
        m = torch.where(real, _normal(g, total, std=3e-4), zero)
        u = torch.where(real, 1e-3 * (0.05 + torch.rand(total, generator=g, device="cuda")), zero)   # root of v
        s = {"p": p, "g": grad, "lr": 1e-4, "b1": 0.9, "b2": 0.999, "eps": 1e-8, "step": 1000, "sizes": sizes, "offs": offs,
             "wd": [0.01 if n > 4096 else 0.0 for n in sizes]}     # matrices decay, norms and biases do not
        if case["bits"] == 32:
            s["m"], s["v"] = m, u * u
        else:
            for name, x in (("m", m), ("v", u)):
                blocks = x.reshape(-1, 256)
                most = blocks.abs().amax(1, keepdim=True)
                s[name] = (blocks * torch.where(most > 0, 448.0 / most, 0.0)).to(torch.float8_e4m3fn).reshape(-1)
                s["s" + name] = (most / 448.0).reshape(-1)
        blocks = torch.tensor([-(-n // 256) for n in sizes], device="cuda")
        s["block_decay"] = torch.repeat_interleave(torch.tensor([1 - s["lr"] * w for w in s["wd"]], device="cuda"), blocks)[:, None]
        return s
    M, D, pt = case["M"], case["D"], TYPES[case["pdtype"]]
    gates = {"none": 0, "channel": 1, "rows": -(-M // case["rows_per_gate"])}[case["gate"]]
    s = {"x": _activations(g, M, D, t), "h": _normal(g, M, D, std=0.7, dtype=t),
         "gate": _normal(g, gates, D, std=0.5, dtype=pt) if gates else None,
         "rows_per_gate": case["rows_per_gate"] if case["gate"] == "rows" else M,
         "w_post": (1 + _normal(g, D, std=0.1)).to(pt), "w_pre": (1 + _normal(g, D, std=0.1)).to(pt)}
    for name in ("b_post", "b_pre"):
        s[name] = _normal(g, D, std=0.1, dtype=pt) if case["kind"] == "layer" else None
    if op == "resnorm":
        s["r"], s["y"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    if op == "resnorm_train":
        s["dr"], s["dy"] = _gradient(g, M, D, 1e-2, t), _gradient(g, M, D, 1e-2, t)
    if op == "block":
        s["q_w"], s["s_w"], s["bias"] = _weights(g, case["O"], D, False)
        s["r"], s["y"] = torch.empty_like(s["x"]), torch.empty(M, case["O"], dtype=t, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:   # the layer objects that a program keeps
        from paper_2407_12637_b200 import lm
        op = case["op"]
        if op in ("linear8", "block"):
            s["linear"] = lm.Linear8.from_codes(s["q_w"], s["s_w"], s["x"].shape[1], bias=s["bias"])
        if op == "linear8_train":
            s["linear"] = lm.Linear8(case["I"], case["O"], bias=s["bias"])
        if op in ("resnorm", "resnorm_train", "block"):
            s["norm"] = lm.ResNorm(case["D"], kind=case["kind"], w_post=s["w_post"], b_post=s["b_post"], w_pre=s["w_pre"], b_pre=s["b_pre"],
                                   eps=1e-6, scale_x=case["scale_x"], scale_h=case["scale_h"])
        if op == "adamw":
            cut = lambda name: [s[name][o:o + n] for o, n in zip(s["offs"], s["sizes"])]  # noqa: E731
            blocks = lambda name: [s[name][o // 256:o // 256 + -(-n // 256)] for o, n in zip(s["offs"], s["sizes"])]  # noqa: E731
            scales = {"m_scale": blocks("sm"), "v_scale": blocks("sv")} if case["bits"] == 8 else {}
            s["adamw"] = lm.AdamW(cut("p"), cut("g"), cut("m"), cut("v"), **scales, lr=s["lr"], betas=(s["b1"], s["b2"]), eps=s["eps"],
                                  weight_decay=s["wd"], step=s["step"])
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if own:
        if op == "linear8":
            return s["linear"].forward(s["x"], out=s["y"])
        if op == "linear8_train":
            s["linear"].load_weight(s["w"])
            y = s["linear"].forward(s["x"], keep=True)
            return {"y": y, **s["linear"].backward(s["dy"])}
        if op == "adamw":
            s["adamw"].step()
            return {k: s[k] for k in ("p", "m", "v", "sm", "sv") if k in s}
        if op == "resnorm":
            r, y = s["norm"].forward(s["x"], s["h"], s["gate"], s["rows_per_gate"], out=(s["r"], s["y"]))
            return {"r": r, "y": y}
        if op == "resnorm_train":
            r, y = s["norm"].forward(s["x"], s["h"], s["gate"], s["rows_per_gate"], keep=True)
            return {"r": r, "y": y, **s["norm"].backward(s["dr"], s["dy"])}
        r, q, scale = s["norm"].forward_codes(s["x"], s["h"], s["gate"], s["rows_per_gate"], out=s["r"])
        return {"r": r, "y": s["linear"].forward_codes(q, scale, out=s["y"])}
    if op == "linear8":
        return _plain_linear8(s["x"].float(), s)
    if op == "linear8_train":
        return _plain_linear8_train(s)
    if op == "adamw":
        return _plain_adamw(s)
    f = _plain_resnorm(s)
    if op == "resnorm":
        return {k: f[k].to(s["x"].dtype) for k in ("r", "y")}
    if op == "resnorm_train":
        return _plain_resnorm_backward(s, f)
    return {"r": f["r"].to(s["x"].dtype), "y": _plain_linear8(f["y"], s)}


def _plain_linear8(x, s):
    q, scale = _rows8(x)
    y = (q @ s["q_w"][:, :x.shape[1]].float().t()) * (scale * s["s_w"])
    return (y + s["bias"] if s["bias"] is not None else y).to(s["x"].dtype)


def _plain_linear8_train(s):
    t = s["x"].dtype
    q_w, s_w = _rows8(s["w"])
    q_x, s_x = _rows8(s["x"].float())
    y = (q_x @ q_w.t()) * (s_x * s_w.t())
    if s["bias"] is not None:
        y = y + s["bias"]
    dy = s["dy"].float()
    q_r, s_r = _rows8(dy * s_w.t())
    q_c, s_c = _rows8((dy * s_x).t())
    out = {"y": y.to(t), "dx": ((q_r @ q_w) * s_r).to(t), "dw": (q_c @ q_x) * s_c}
    if s["bias"] is not None:
        out["dbias"] = dy.sum(0)
    return out


def _plain_norm(v, w, b, layer):
    d = v - v.mean(1, keepdim=True) if layer else v
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-6)
    k = d * rstd
    y = k * w.float()
    return (y + b.float() if b is not None else y), k, rstd


def _plain_resnorm(s):
    c = s["case"]
    layer = c["kind"] == "layer"
    u, k_post, rstd_post = _plain_norm(s["h"].float(), s["w_post"], s["b_post"], layer)
    M = u.shape[0]
    gate = s["gate"].float().repeat_interleave(s["rows_per_gate"], 0)[:M] if s["gate"] is not None else None
    r = c["scale_x"] * s["x"].float() + c["scale_h"] * (u if gate is None else gate * u)
    y, k_pre, rstd_pre = _plain_norm(r, s["w_pre"], s["b_pre"], layer)
    return {"u": u, "gate": gate, "r": r, "y": y, "k_post": k_post, "rstd_post": rstd_post, "k_pre": k_pre, "rstd_pre": rstd_pre}


def _plain_norm_backward(d, w, k, rstd, layer):
    e = d * w.float()
    back = e - k * (e * k).mean(1, keepdim=True)
    return (back - e.mean(1, keepdim=True) if layer else back) * rstd


def _plain_resnorm_backward(s, f):
    c, t = s["case"], s["x"].dtype
    layer, pt = c["kind"] == "layer", s["w_pre"].dtype
    dy = s["dy"].float()
    d = s["dr"].float() + _plain_norm_backward(dy, s["w_pre"], f["k_pre"], f["rstd_pre"], layer)
    du = c["scale_h"] * (d if f["gate"] is None else d * f["gate"])
    out = {"r": f["r"].to(t), "y": f["y"].to(t), "dx": (c["scale_x"] * d).to(t),
           "dh": _plain_norm_backward(du, s["w_post"], f["k_post"], f["rstd_post"], layer).to(t),
           "dw_pre": (dy * f["k_pre"]).sum(0).to(pt), "dw_post": (du * f["k_post"]).sum(0).to(pt)}
    if layer:
        out["db_pre"], out["db_post"] = dy.sum(0).to(pt), du.sum(0).to(pt)
    if s["gate"] is not None:
        n, rows = s["gate"].shape[0], s["rows_per_gate"]
        each = torch.zeros(n * rows, d.shape[1], device="cuda")
        each[:d.shape[0]] = c["scale_h"] * d * f["u"]
        out["dgate"] = each.reshape(n, rows, -1).sum(1).to(pt)
    return out


def _plain_adamw(s):
    b1, b2 = s["b1"], s["b2"]
    s["step"] += 1
    c1, c2 = s["lr"] / (1 - b1 ** s["step"]), math.sqrt(1 - b2 ** s["step"])
    g = s["g"].float().reshape(-1, 256)
    p = s["p"].float().reshape(-1, 256)
    if "sm" in s:
        m = s["m"].float().reshape(-1, 256) * s["sm"][:, None]
        v = (s["v"].float().reshape(-1, 256) * s["sv"][:, None]).square()
    else:
        m, v = s["m"].reshape(-1, 256), s["v"].reshape(-1, 256)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * (g * g)
    u = torch.sqrt(v)
    p = s["block_decay"] * p - c1 * m / (u / c2 + s["eps"])
    s["p"].copy_(p.reshape(-1))
    if "sm" not in s:
        s["m"].copy_(m.reshape(-1))
        s["v"].copy_(v.reshape(-1))
        return {"p": s["p"], "m": s["m"], "v": s["v"]}
    most_m, most_u = m.abs().amax(1, keepdim=True), u.amax(1, keepdim=True)
    s["m"].copy_((m * torch.where(most_m > 1e-36, 448.0 / most_m, 0.0)).reshape(-1))
    codes = u * torch.where(most_u > 1e-36, 448.0 / most_u, 0.0)
    s["v"].copy_(torch.where(u > 0, codes.clamp(min=2.0 ** -9), codes).reshape(-1))   # a positive root is not stored as 0
    s["sm"].copy_(most_m.reshape(-1) / 448.0)
    s["sv"].copy_(most_u.reshape(-1) / 448.0)
    return {k: s[k] for k in ("p", "m", "v", "sm", "sv")}


# ---------------------------------------------------------------------------------------------- 64 bits
def _exact_codes(t, dim):
    top = torch.amax(torch.abs(t), dim, keepdim=True)
    step = top / 127
    return torch.round(t / torch.where(step > 0, step, torch.ones_like(step))), step


def _exact_standard(v, kind):
    centre = torch.mean(v, 1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    dev = torch.sqrt(torch.mean((v - centre) ** 2, 1, keepdim=True) + 1e-6)
    return (v - centre) / dev, dev


def _e4m3(x):
    """Nearest e4m3 value (ties to even, subnormal step 2^-9)."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), torch.clamp(e - 4, min=-9))
    return torch.round(x / step) * step


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    D = lambda name: s[name].double()  # noqa: E731
    if op == "linear8":
        q, a = _exact_codes(D("x"), 1)
        y = torch.matmul(q, D("q_w")[:, :case["I"]].T) * a * D("s_w")
        return y if s["bias"] is None else y + D("bias")
    if op == "linear8_train":
        qw, aw = _exact_codes(D("w"), 1)
        qx, ax = _exact_codes(D("x"), 1)
        y = torch.matmul(qx * ax, (qw * aw).T)
        qr, ar = _exact_codes(D("dy") * aw.T, 1)
        qc, ac = _exact_codes(D("dy") * ax, 0)
        out = {"y": y if s["bias"] is None else y + D("bias"), "dx": torch.matmul(qr * ar, qw), "dw": torch.matmul((qc * ac).T, qx)}
        if s["bias"] is not None:
            out["dbias"] = torch.sum(D("dy"), 0)
        return out
    if op == "adamw":
        t = s["step"] + 1
        g, p, m, v = D("g").view(-1, 256), D("p").view(-1, 256), D("m").view(-1, 256), D("v").view(-1, 256)
        if case["bits"] == 8:
            m, v = m * D("sm")[:, None], (v * D("sv")[:, None]) ** 2
        m = m * 0.9 + g * (1 - 0.9)
        v = v * 0.999 + g ** 2 * (1 - 0.999)
        mhat, vhat = m / (1 - 0.9 ** t), v / (1 - 0.999 ** t)
        lengths = torch.tensor([-(-n // 256) for n in s["sizes"]], device="cuda")
        decay = torch.repeat_interleave(torch.tensor(s["wd"], dtype=torch.float64, device="cuda"), lengths)[:, None]
        p = p - s["lr"] * decay * p - s["lr"] * mhat / (vhat ** 0.5 + s["eps"])
        if case["bits"] == 32:
            return {"p": p.view(-1), "m": m.view(-1), "v": v.view(-1)}
        u, out = v ** 0.5, {"p": p.view(-1)}
        for name, x in (("m", m), ("v", u)):
            scale = torch.amax(torch.abs(x), 1, keepdim=True) / 448
            code = _e4m3(x / torch.where(scale > 0, scale, torch.ones_like(scale)))
            out[name] = (torch.where((x > 0) & (code == 0), torch.full_like(code, 2.0 ** -9), code) if name == "v" else code).view(-1)
            out["s" + name] = scale.view(-1)
        return out
    M = case["M"]
    rows = torch.arange(M, device="cuda") // s["rows_per_gate"]
    gate = D("gate")[rows] if s["gate"] is not None else torch.ones_like(D("x"))
    k1, dev1 = _exact_standard(D("h"), case["kind"])
    u = k1 * D("w_post") + (D("b_post") if s["b_post"] is not None else 0)
    r = case["scale_x"] * D("x") + case["scale_h"] * gate * u
    k2, dev2 = _exact_standard(r, case["kind"])
    y = k2 * D("w_pre") + (D("b_pre") if s["b_pre"] is not None else 0)
    if op == "resnorm":
        return {"r": r, "y": y}
    if op == "block":
        q, a = _exact_codes(y, 1)
        return {"r": r, "y": torch.matmul(q * a, (D("q_w")[:, :case["D"]] * D("s_w")[:, None]).T)}

    def back(d, w, k, dev):
        e = d * w
        out = e - k * torch.mean(e * k, 1, keepdim=True)
        return (out - torch.mean(e, 1, keepdim=True) if case["kind"] == "layer" else out) / dev

    d = D("dr") + back(D("dy"), D("w_pre"), k2, dev2)
    du = case["scale_h"] * gate * d
    out = {"r": r, "y": y, "dx": case["scale_x"] * d, "dh": back(du, D("w_post"), k1, dev1),
           "dw_pre": torch.einsum("md,md->d", D("dy"), k2), "dw_post": torch.einsum("md,md->d", du, k1)}
    if case["kind"] == "layer":
        out["db_pre"], out["db_post"] = torch.sum(D("dy"), 0), torch.sum(du, 0)
    if s["gate"] is not None:
        out["dgate"] = torch.zeros_like(D("gate")).index_add_(0, rows, case["scale_h"] * u * d)
    return out
