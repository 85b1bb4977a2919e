"""Cases of the operators around the framework's layers: clip (norm of all gradients, and clipping by it), adapters (low-rank
adapters of many requests beside a linear layer, their training step) and groupnorm (group norm with an activation on
channels-last images, its training step).

`run` computes them in plain torch operations in 32 bits (`own` false) or through the framework (`own` true)."""
import math
import random

import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
SIZES = {"float32": 4, "bfloat16": 2, "float16": 2}


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # gradients of adapters: many small tensors of odd lengths, clipped ahead of their optimizer's step; latency counts
        {"name": "clip 96 ragged", "op": "clip", "layout": "ragged", "a": 96, "b": 20000, "dtype": "bfloat16", "odtype": "bfloat16"},
        # ResNet-18's 62 gradients in fp32: the norm alone, whose factor the optimizer takes
        {"name": "norm resnet18", "op": "norm", "layout": "resnet18", "a": 0, "b": 0, "dtype": "float32", "odtype": "float32"},
        # eight transformer blocks of width 2048 (0.4 G elements), bf16 gradients clipped
        {"name": "clip 8 blocks x 2048", "op": "clip", "layout": "blocks", "a": 8, "b": 2048, "dtype": "bfloat16", "odtype": "bfloat16"},
        # one token of one request: a chat session's decode step
        {"name": "adapters 1 x 4096 -> 4096", "op": "adapters", "M": 1, "runs": 1, "n": 1, "r": 16, "I": 4096, "O": 4096, "dtype": "bfloat16"},
        # a decode batch of 64 requests with 16 adapters among them, some requests without one
        {"name": "adapters 64 x 4096 -> 8192", "op": "adapters", "M": 64, "runs": 64, "n": 16, "r": 16, "I": 4096, "O": 8192, "dtype": "bfloat16"},
        # prompts of eleven requests, of ragged lengths, adapters of rank 64
        {"name": "adapters 2085 x 4096 -> 4096", "op": "adapters", "M": 2085, "runs": 11, "n": 6, "r": 64, "I": 4096, "O": 4096, "dtype": "float16"},
        # fine-tuning: one adapter on 8192 tokens, forward and backward pass
        {"name": "adapters train 8192 x 4096", "op": "adapters_train", "M": 8192, "runs": 1, "n": 1, "r": 16, "I": 4096, "O": 4096,
         "dtype": "bfloat16"},
        # three adapters trained at once in fp32 on a classifier head with odd sizes
        {"name": "adapters train 1111 x 2047", "op": "adapters_train", "M": 1111, "runs": 7, "n": 3, "r": 5, "I": 2047, "O": 1000,
         "dtype": "float32"},
        # the last stage's image of a served ResNet, one image
        {"name": "groupnorm 1 x 7 x 7 x 512", "op": "groupnorm", "N": 1, "H": 7, "W": 7, "C": 512, "G": 32, "act": "relu", "dtype": "bfloat16"},
        # super-resolution: whole images in fp16
        {"name": "groupnorm 16 x 96 x 96 x 64", "op": "groupnorm", "N": 16, "H": 96, "W": 96, "C": 64, "G": 16, "act": "silu",
         "dtype": "float16"},
        # ResNet-18's first stage, training with a smooth activation (the slope of a ReLU jumps where a sum of many roundings crosses
        # 0: outputs next to that border say nothing about a kernel)
        {"name": "groupnorm train 64 x 56 x 56 x 64", "op": "groupnorm_train", "N": 64, "H": 56, "W": 56, "C": 64, "G": 32, "act": "silu",
         "dtype": "bfloat16"},
        # odd images and channels in fp32
        {"name": "groupnorm train 5 x 33 x 17 x 90", "op": "groupnorm_train", "N": 5, "H": 33, "W": 17, "C": 90, "G": 6, "act": "silu",
         "dtype": "float32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "clip", "adapters", "adapters", "adapters_train", "groupnorm", "groupnorm_train"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if op in ("norm", "clip"):
        layout = rng.choice(["blocks", "ragged"])
        a, b = (rng.randint(1, 8), 8 * rng.randint(32, 256)) if layout == "blocks" else (_log(rng, 1, 400), _log(rng, 10, 500000))
        return {"op": op, "layout": layout, "a": a, "b": b, "dtype": dtype, "odtype": rng.choice([dtype, "float32"]) if a * b < 8000 else dtype}
    if op in ("adapters", "adapters_train"):
        r = rng.choice([4, 8, 16, 32, 64, rng.randint(1, 64)])
        M = _log(rng, 1 if op == "adapters" else 32, 8192)
        return {"op": op, "M": M, "runs": _log(rng, 1, min(M, 128)), "n": rng.randint(1, 16), "r": r, "I": _log(rng, 256, 8192 if M < 4096 else 4096),
                "O": _log(rng, 256, 8192 if M < 4096 else 4096), "dtype": dtype}
    G = _log(rng, 1, 32)
    C = G * _log(rng, 1, max(1, 512 // G))
    H, W = _log(rng, 4, 112), _log(rng, 4, 112)
    return {"op": op, "N": _log(rng, 1, max(1, min(64, 12000000 // (H * W * C)))), "H": H, "W": W, "C": C, "G": G,
            "act": rng.choice(["none", "relu", "silu"] if op == "groupnorm" else ["none", "silu"]), "dtype": dtype}


def _lengths(case):
    """The element counts of a clip case's tensors."""
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


def _runs(case, rng):
    """(offsets of the runs of tokens, adapter of each): ragged lengths, a few of them empty; from eight runs on one in eight has
    no adapter (-1); the last tokens of a served batch of more than 200 belong to no run."""
    M, R, n = case["M"], case["runs"], case["n"]
    if R == M:
        offs = list(range(M + 1))
    else:
        end = M - (M // 100 if R > 1 and M > 200 and case["op"] == "adapters" else 0)
        offs = [0] + sorted(rng.randint(0, end) for _ in range(R - 1)) + [end]
    with_one = R - R // 8
    ids = [i % n for i in range(with_one)] + [-1] * (R // 8)
    rng.shuffle(ids)
    return offs, ids


def work(case):
    e = SIZES[case["dtype"]]
    if case["op"] in ("norm", "clip"):
        n = sum(_lengths(case))
        if case["op"] == "norm":
            return {"bytes": n * e, "flops": 2 * n}
        return {"bytes": n * (e + SIZES[case["odtype"]]), "flops": 3 * n}   # (every gradient read once, were there room to keep it)
    if case["op"] in ("adapters", "adapters_train"):
        M, I, O, r = case["M"], case["I"], case["O"], case["r"]
        weights = min(case["n"], case["runs"] - case["runs"] // 8) * r * (I + O)
        if case["op"] == "adapters":
            return {"bytes": e * (M * I + 2 * M * O + weights), "flops": 2 * M * r * (I + O)}
        # forward as above; backward: dy, x and the layer's dx read, dx and the gradients (fp32) written
        return {"bytes": e * (M * I + 2 * M * O + weights) + e * (M * O + 3 * M * I + weights) + 4 * case["n"] * r * (I + O),
                "flops": 6 * M * r * (I + O)}
    n = case["N"] * case["H"] * case["W"] * case["C"]
    if case["op"] == "groupnorm":
        return {"bytes": 2 * n * e, "flops": 10 * n}
    return {"bytes": 5 * n * e, "flops": 30 * n}   # forward: x -> y; backward: x, dy -> dx


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


def _gradient(g, *shape, std, dtype):
    """Zero-centred with a long tail."""
    u = torch.rand(*shape, generator=g, device="cuda") - 0.5
    return (-torch.sign(u) * torch.log1p(-2 * u.abs() * (1 - 1e-6)) * std).to(dtype)


def _inputs(case, seed):
    g, t = _gen(seed), TYPES[case["dtype"]]
    if case["op"] in ("norm", "clip"):
        sizes = _lengths(case)
        offs, total = _offsets(sizes)
        grad = _gradient(g, total, std=1e-3, dtype=t)
        ends = torch.zeros(total + 1, dtype=torch.int8, device="cuda")    # 1 where an element belongs to a tensor
        ends.index_add_(0, torch.tensor(offs, device="cuda"), torch.ones(len(sizes), dtype=torch.int8, device="cuda"))
        ends.index_add_(0, torch.tensor([o + n for o, n in zip(offs, sizes)], device="cuda"), -torch.ones(len(sizes), dtype=torch.int8, device="cuda"))
        grad.mul_(torch.cumsum(ends[:-1], 0, dtype=torch.int8))
        blocks = torch.tensor([-(-n // 256) for n in sizes], device="cuda")
        s = {"g": grad, "max_norm": 1.0, "sizes": sizes, "offs": offs,
             "owner": torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), blocks)}
        if case["op"] == "clip":
            s["out"] = torch.zeros(total, dtype=TYPES[case["odtype"]], device="cuda")
        return s
    if case["op"] in ("adapters", "adapters_train"):
        M, I, O, r, n = (case[k] for k in ("M", "I", "O", "r", "n"))
        offs, ids = _runs(case, random.Random(seed))
        s = {"x": _activations(g, M, I, t), "base": _normal(g, M, O, dtype=t), "a": _normal(g, n, r, I, std=I ** -0.5, dtype=t),
             "b": _normal(g, n, r, O, std=0.1 * r ** -0.5, dtype=t), "scale": 0.5 + torch.rand(n, generator=g, device="cuda"),
             "offsets": torch.tensor(offs, dtype=torch.int32, device="cuda"), "index": torch.tensor(ids, dtype=torch.int32, device="cuda"),
             "offs": offs, "ids": ids}
        s["out"] = torch.zeros(M, O, dtype=t, device="cuda")
        if case["op"] == "adapters_train":
            s["dy"], s["dbase"] = _gradient(g, M, O, std=1e-2, dtype=t), _normal(g, M, I, std=1e-3, dtype=t)
            s["dx"] = torch.zeros(M, I, dtype=t, device="cuda")
        return s
    N, H, W, C = (case[k] for k in "NHWC")
    # channels of different means and spreads, as a convolution leaves them
    x = _normal(g, N, H, W, C) * (0.5 + torch.rand(C, generator=g, device="cuda")) + _normal(g, C, std=0.7)
    s = {"x": x.to(t), "w": 1 + _normal(g, C, std=0.2), "b": _normal(g, C, std=0.2)}
    if case["op"] == "groupnorm":
        s["out"] = torch.empty(N, H, W, C, dtype=t, device="cuda")
    else:
        s["dy"] = _gradient(g, N, H, W, C, std=1e-2, dtype=t)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:   # the objects that a program keeps
        from paper_2407_12637_b200 import cnn, lm
        if case["op"] in ("norm", "clip"):
            cut = lambda name: [s[name][o:o + n] for o, n in zip(s["offs"], s["sizes"])]  # noqa: E731
            s["clip"] = lm.GradClip(cut("g"), s["max_norm"], out=cut("out") if case["op"] == "clip" else None)
        elif case["op"] in ("adapters", "adapters_train"):
            s["adapters"] = lm.Adapters(s["a"], s["b"], s["scale"])
        else:
            s["norm"] = cnn.GroupNorm(case["C"], case["G"], s["w"], s["b"], eps=1e-5, act=case["act"])
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if own:
        if op == "norm":
            s["clip"].measure()
            return {"norm": s["clip"].norm, "scale": s["clip"].scale, "norms": s["clip"].norms}
        if op == "clip":
            s["clip"].clip()
            return {"norm": s["clip"].norm, "scale": s["clip"].scale, "norms": s["clip"].norms, "clipped": s["out"]}
        if op == "adapters":
            return s["adapters"].forward(s["x"], s["base"], s["offsets"], s["index"], out=s["out"])
        if op == "adapters_train":
            y = s["adapters"].forward(s["x"], s["base"], s["offsets"], s["index"], out=s["out"], keep=True)
            return {"y": y, **s["adapters"].backward(s["dy"], s["dbase"], dx=s["dx"])}
        if op == "groupnorm":
            return s["norm"].forward(s["x"], out=s["out"])
        y = s["norm"].forward(s["x"], keep=True)
        return {"y": y, **s["norm"].backward(s["dy"])}
    if op in ("norm", "clip"):
        return _plain_clip(s)
    if op == "adapters":
        y, _, covered = _plain_adapters(s)
        return torch.where(covered, y.to(s["out"].dtype), s["out"])
    if op == "adapters_train":
        return _plain_adapters_train(s)
    f = _plain_groupnorm(s)
    return f["y"].to(s["x"].dtype) if op == "groupnorm" else _plain_groupnorm_backward(s, f)


def _plain_clip(s):
    g = s["g"].float()
    sums = (g * g).reshape(-1, 256).sum(1).double()
    squares = torch.zeros(len(s["sizes"]), dtype=torch.float64, device="cuda").index_add_(0, s["owner"], sums)
    norm = torch.sqrt(squares.sum()).float().reshape(1)
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    out = {"norm": norm, "scale": scale, "norms": torch.sqrt(squares).float()}
    if "out" in s:
        out["clipped"] = s["out"].copy_(g * scale)
    return out


def _tokens(s):
    """Which adapters' ranks each token uses, times the adapter's scale [M, n r]; which tokens belong to a run [M, 1]."""
    M, (n, r, _) = s["x"].shape[0], s["a"].shape
    at = torch.arange(M, device="cuda")
    run_of = torch.searchsorted(s["offsets"], at, right=True) - 1
    covered = (run_of >= 0) & (at < s["offsets"][-1])
    adapter = torch.where(covered, s["index"].long()[run_of.clamp(0, s["index"].numel() - 1)], -1)
    mine = (adapter[:, None] == torch.arange(n, device="cuda")) * s["scale"]
    return mine.repeat_interleave(r, 1), covered[:, None]


def _plain_adapters(s):
    n, r, I = s["a"].shape
    mask, covered = _tokens(s)
    h = (s["x"].float() @ s["a"].float().reshape(n * r, I).t()) * mask
    return s["base"].float() + h @ s["b"].float().reshape(n * r, -1), (h, mask), covered


def _plain_adapters_train(s):
    t, (n, r, I) = s["x"].dtype, s["a"].shape
    y, (h, mask), covered = _plain_adapters(s)
    dy = s["dy"].float()
    dh = (dy @ s["b"].float().reshape(n * r, -1).t()) * mask
    dx = s["dbase"].float() + dh @ s["a"].float().reshape(n * r, I)
    return {"y": y.to(t), "dx": dx.to(t), "da": (dh.t() @ s["x"].float()).reshape(n, r, I), "db": (h.t() @ dy).reshape(n, r, -1)}


def _plain_groupnorm(s):
    c = s["case"]
    x = s["x"].float().reshape(c["N"], c["H"] * c["W"], c["G"], -1)
    d = x - x.mean((1, 3), keepdim=True)
    rstd = 1.0 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + 1e-5)
    k = d * rstd
    z = k * s["w"].reshape(c["G"], -1) + s["b"].reshape(c["G"], -1)
    gate = 1.0 / (1.0 + torch.exp(-z)) if c["act"] == "silu" else (z > 0).float() if c["act"] == "relu" else None
    y = z if gate is None else z * gate
    return {"y": y.reshape(s["x"].shape), "z": z, "k": k, "rstd": rstd, "gate": gate}


def _plain_groupnorm_backward(s, f):
    c, t = s["case"], s["x"].dtype
    e = s["dy"].float().reshape(f["z"].shape)
    if c["act"] == "silu":
        e = e * f["gate"] * (1.0 + f["z"] * (1.0 - f["gate"]))
    dk = e * s["w"].reshape(c["G"], -1)
    dx = (dk - dk.mean((1, 3), keepdim=True) - f["k"] * (dk * f["k"]).mean((1, 3), keepdim=True)) * f["rstd"]
    return {"y": f["y"].to(t), "dx": dx.reshape(s["x"].shape).to(t), "dw": (e * f["k"]).sum((0, 1)).reshape(-1), "db": e.sum((0, 1)).reshape(-1)}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    D = lambda name: s[name].double()  # noqa: E731
    if case["op"] in ("norm", "clip"):
        norms = torch.stack([torch.linalg.vector_norm(s["g"][o:o + n].double()) for o, n in zip(s["offs"], s["sizes"])])
        norm = torch.linalg.vector_norm(norms).reshape(1)
        factor = torch.clamp(s["max_norm"] / norm, max=1.0)
        out = {"norm": norm, "scale": factor, "norms": norms}
        if case["op"] == "clip":
            out["clipped"] = D("g") * factor
        return out
    if case["op"] in ("adapters", "adapters_train"):
        runs = [(slice(lo, hi), i) for lo, hi, i in zip(s["offs"], s["offs"][1:], s["ids"]) if i >= 0 and hi > lo]
        y = D("base")
        for at, i in runs:
            y[at] += s["scale"][i].double() * (s["x"][at].double() @ s["a"][i].double().T @ s["b"][i].double())
        if case["op"] == "adapters":
            y[s["offs"][-1]:] = 0    # (as the caller's buffer was)
            return y
        dx, da, db = D("dbase"), torch.zeros_like(D("a")), torch.zeros_like(D("b"))
        for at, i in runs:
            scale, x, dy, a, b = s["scale"][i].double(), s["x"][at].double(), s["dy"][at].double(), s["a"][i].double(), s["b"][i].double()
            back = scale * torch.einsum("mo,ro->mr", dy, b)
            dx[at] += back @ a
            da[i] += torch.einsum("mr,mi->ri", back, x)
            db[i] += scale * torch.einsum("mr,mo->ro", x @ a.T, dy)
        return {"y": y, "dx": dx, "da": da, "db": db}
    N, P, C, G = case["N"], case["H"] * case["W"], case["C"], case["G"]
    x = D("x").view(N, P, G, C // G)
    var, mean = torch.var_mean(x, (1, 3), keepdim=True, correction=0)
    dev = torch.sqrt(var + 1e-5)
    k = (x - mean) / dev
    w = D("w").view(G, C // G)
    z = k * w + D("b").view(G, C // G)
    slope = torch.ones_like(z)
    y = z
    if case["act"] == "relu":
        y = torch.relu(z)
    elif case["act"] == "silu":
        sig = torch.sigmoid(z)
        y, slope = z * sig, sig + z * sig * (1 - sig)
    if case["op"] == "groupnorm":
        return y.view(s["x"].shape)
    e = D("dy").view(N, P, G, C // G) * slope
    back = e * w
    dx = (back - back.mean((1, 3), keepdim=True) - k * (back * k).mean((1, 3), keepdim=True)) / dev
    return {"y": y.view(s["x"].shape), "dx": dx.view(s["x"].shape), "dw": (e * k).sum((0, 1)).view(-1), "db": e.sum((0, 1)).view(-1)}
