"""A stack of residual blocks trained with 8-bit products and 8-bit optimizer states.

    python -m paper_2407_12637_b200.block_train [--depth 4] [--dim 1024] [--tokens 4096] [--steps 50] [--max-norm 1.0] [--rank 16]

Block l: h = W_l y + b_l on 8-bit integers, r = r + gate N_post(h), y = N_pre(r) -- the norm writes y as the 8-bit codes that
the next block's product reads.  The model learns to map random inputs to the outputs of a fixed random map (synthetic
data, mean squared error on the last y); backward pass, AdamW step and requantization all run in the library's kernels.
With --max-norm the norm of all gradients is measured ahead of each step, which is then scaled by it (and held back if a gradient is not
finite).  With --rank the 8-bit weights stay as they are: low-rank adapters beside them are trained with the norms (fine-tuning).
"""
from __future__ import annotations

import argparse

import torch

from . import lm


class Stack:
    """`depth` blocks of width `dim`: fp32 master weights with their 8-bit layers, norms and gates, gradients in fixed buffers."""

    def __init__(self, depth, dim, lr=1e-3, state_bits=8, seed=0, device="cuda", max_norm=None, rank=0, dtype=torch.bfloat16):
        g = torch.Generator(device=device).manual_seed(seed)
        self.weights = [torch.randn(dim, dim, generator=g, device=device) * dim ** -0.5 for _ in range(depth)]
        self.biases = [torch.zeros(dim, device=device) for _ in range(depth)]
        vec = lambda v: torch.full((dim,), v, device=device)  # noqa: E731
        self.norm_params = [{"gate": vec(0.5), "w_post": vec(1.0), "w_pre": vec(1.0)} for _ in range(depth)]
        self.layers = [lm.Linear8(dim, dim, bias=b, weight=w) for w, b in zip(self.weights, self.biases)]
        self.norms = [lm.ResNorm(dim, "rms", p["w_post"], None, p["w_pre"], None) for p in self.norm_params]
        # adapters of the activations' type, with fp32 masters
        self.masters = [(torch.randn(1, rank, dim, generator=g, device=device) * dim ** -0.5, torch.zeros(1, rank, dim, device=device)) for _ in range(depth if rank else 0)]
        self.adapters = [lm.Adapters(a.to(dtype), b.to(dtype)) for a, b in self.masters]
        weights = [a for a, _ in self.masters] + [b for _, b in self.masters] if rank else self.weights + self.biases
        params = weights + [p[k] for p in self.norm_params for k in ("gate", "w_post", "w_pre")]
        grads = [torch.zeros_like(p) for p in params]
        self.dw, self.db = grads[:depth], grads[depth:2 * depth]   # (of W and b, or of A and B)
        rest = iter(grads[2 * depth:])
        self.dnorm = [{"dgate": next(rest), "dw_post": next(rest), "dw_pre": next(rest)} for _ in range(depth)]
        self.optimizer = lm.AdamW(params, grads, lr=lr, weight_decay=[0.01] * depth + [0.0] * (len(params) - depth), state_bits=state_bits)
        self.clip = lm.GradClip(grads, max_norm) if max_norm is not None else None

    def forward(self, x):
        """The last block's y for x [tokens, dim]."""
        r, q, scale = x, None, None
        if self.adapters:   # (they read y itself, where the 8-bit product alone needs its codes)
            y = x
            for layer, norm, p, adapters in zip(self.layers, self.norms, self.norm_params, self.adapters):
                h = adapters.forward(y, layer.forward(y, keep=True), keep=True)
                r, y = norm.forward(r, h, p["gate"], keep=True)
            return y
        for i, (layer, norm, p) in enumerate(zip(self.layers, self.norms, self.norm_params)):
            h = layer.forward(x, keep=True) if q is None else layer.forward_codes(q, scale, dtype=x.dtype, keep=True)
            if i + 1 < len(self.layers):
                r, q, scale = norm.forward_codes(r, h, p["gate"], keep=True)
            else:
                r, y = norm.forward(r, h, p["gate"], keep=True)
        return y

    def backward(self, dy):
        """Fills the gradient buffers from the gradient of the last y; returns the gradient of x."""
        dr = None
        for i in reversed(range(len(self.layers))):
            g = self.norms[i].backward(dr, dy, out=self.dnorm[i])
            if self.adapters:
                dx = self.layers[i].backward(g["dh"], need_dw=False)["dx"]
                dr, dy = g["dx"], self.adapters[i].backward(g["dh"], dx, da=self.dw[i], db=self.db[i])["dx"]
            else:
                dr, dy = g["dx"], self.layers[i].backward(g["dh"], dw=self.dw[i], dbias=self.db[i])["dx"]
        return dr + dy   # x is the first block's residual stream and its product's input

    def step(self, x, target):
        """One training step; the loss (a device scalar)."""
        y = self.forward(x)
        diff = y.float() - target.float()
        self.backward((diff * (2.0 / diff.numel())).to(x.dtype))
        if self.clip is not None:
            self.clip.measure()
            self.optimizer.step(grad_scale=self.clip.scale, skip=self.clip.skip)
        else:
            self.optimizer.step()
        if self.adapters:
            for adapters, (a, b) in zip(self.adapters, self.masters):
                adapters.a.copy_(a)
                adapters.b.copy_(b)
        else:
            for layer, w in zip(self.layers, self.weights):
                layer.load_weight(w)
        return (diff * diff).mean()

    def check(self):
        """Raises if a product's output is missing (waits for the device)."""
        for layer in self.layers + self.adapters:
            layer.check()


def train(depth=4, dim=1024, tokens=4096, steps=50, dtype=torch.bfloat16, state_bits=8, lr=1e-3, seed=0, report=None, max_norm=None, rank=0):
    """The losses of `steps` steps on fresh synthetic batches."""
    model = Stack(depth, dim, lr=lr, state_bits=state_bits, seed=seed, max_norm=max_norm, rank=rank, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    teacher = torch.randn(dim, dim, generator=g, device="cuda") * dim ** -0.5
    losses = []
    for i in range(steps):
        x = torch.randn(tokens, dim, generator=g, device="cuda").to(dtype)
        target = torch.tanh(x.float() @ teacher)
        losses.append(model.step(x, target))
        if report is not None and (i % 10 == 0 or i + 1 == steps):
            model.check()
            report(i, float(losses[-1]))
    model.check()
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("depth", 4), ("dim", 1024), ("tokens", 4096), ("steps", 50), ("state-bits", 8), ("rank", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--max-norm", type=float, default=None)
    a = ap.parse_args()
    train(a.depth, a.dim, a.tokens, a.steps, state_bits=a.state_bits, max_norm=a.max_norm, rank=a.rank, report=lambda i, v: print(f"step {i:4d}  loss {v:.5f}", flush=True))


if __name__ == "__main__":
    main()
