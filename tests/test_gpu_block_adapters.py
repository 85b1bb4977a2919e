"""The example with adapters beside frozen 8-bit layers and clipped steps: gradients of a whole stack against the same model in 64 bits, a step."""
import math

import pytest
import torch

from paper_2407_12637_b200 import block_train

pytestmark = pytest.mark.gpu


def _plain(model, x, target):
    """Loss and gradients of the stack with the weights that the codes stand for and exact products, in 64 bits."""
    ws = [l.q_w[:, :l.I].double() * l.s_w.double()[:, None] for l in model.layers]
    ab = [(a.a[0].double().requires_grad_(), a.b[0].double().requires_grad_()) for a in model.adapters]
    ps = [{k: v.double().requires_grad_() for k, v in p.items()} for p in model.norm_params]
    norm = lambda v, w: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * w  # noqa: E731
    r = y = x.double()
    for w, bias, (a, b), p in zip(ws, model.biases, ab, ps):
        h = y @ w.T + bias.double() + y @ a.T @ b
        r = r + p["gate"] * norm(h, p["w_post"])
        y = norm(r, p["w_pre"])
    loss = ((y - target.double()) ** 2).mean()
    loss.backward()
    return loss, ab, ps


def test_gradients_of_the_stack():
    """The layers' inputs and their gradients pass through 8 bits (a relative error of about 1 / (127 sqrt(3)) of a row's largest value each): directions
    agree to 0.99, lengths to a tenth, as without adapters."""
    model = block_train.Stack(3, 192, rank=8, max_norm=1e-3, dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(3)
    for a in model.adapters:
        a.b.copy_(torch.randn(a.b.shape, generator=g, device="cuda") * 0.2)
    x, target = (torch.randn(500, 192, generator=g, device="cuda") for _ in range(2))
    want_loss, ab, ps = _plain(model, x, target)
    y = model.forward(x)
    diff = y - target
    model.backward(diff * (2.0 / diff.numel()))
    assert abs(float((diff * diff).mean()) - float(want_loss)) <= 0.02 * float(want_loss)
    pairs = [(got[0], t.grad) for got, t in zip(model.dw, (a for a, _ in ab))] + [(got[0], t.grad) for got, t in zip(model.db, (b for _, b in ab))]
    for got, p in zip(model.dnorm, ps):
        pairs += [(got["dgate"], p["gate"].grad), (got["dw_post"], p["w_post"].grad), (got["dw_pre"], p["w_pre"].grad)]
    for got, want in pairs:
        a, b = got.double().flatten(), want.detach().flatten()
        assert float(a @ b) >= 0.99 * float(a.norm() * b.norm())
        assert abs(float(a.norm() / b.norm()) - 1) <= 0.1
    model.clip.measure()
    total = math.sqrt(sum(float(t.double().square().sum()) for t in model.clip.grads))
    assert abs(float(model.clip.norm) - total) <= 4 * 2.0 ** -24 * total and float(model.clip.scale) < 1


@pytest.mark.parametrize("rank,max_norm", [(0, 1.0), (8, None), (8, 1.0)])
def test_it_runs(rank, max_norm):
    losses = block_train.train(depth=2, dim=256, tokens=300, steps=4, rank=rank, max_norm=max_norm)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)


def test_a_step_with_a_gradient_that_is_not_finite_changes_nothing():
    model = block_train.Stack(2, 128, rank=4, max_norm=1.0)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, target = torch.randn(64, 128, generator=g, device="cuda").bfloat16(), torch.randn(64, 128, generator=g, device="cuda")
    model.step(x, target)
    before = [t.clone() for t in model.optimizer.params]
    target[3, 7] = math.inf
    model.step(x, target)
    assert int(model.clip.skip) == 1 and all(torch.equal(a, b) for a, b in zip(model.optimizer.params, before))
    model.check()
