"""The example that runs the operators together: gradients of a whole stack against the same model in 64 bits, and a training run."""
import pytest
import torch

from paper_2407_12637_b200 import block_train

pytestmark = pytest.mark.gpu


def _plain(model, x, target):
    """Loss and gradients of the stack with exact products, in 64 bits."""
    ws = [w.double().requires_grad_() for w in model.weights]
    bs = [b.double().requires_grad_() for b in model.biases]
    ps = [{k: v.double().requires_grad_() for k, v in p.items()} for p in model.norm_params]
    norm = lambda v, w: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * w  # noqa: E731
    r = y = x.double()
    for w, b, p in zip(ws, bs, ps):
        h = y @ w.T + b
        r = r + p["gate"] * norm(h, p["w_post"])
        y = norm(r, p["w_pre"])
    loss = ((y - target.double()) ** 2).mean()
    loss.backward()
    return loss, [w.grad for w in ws], [b.grad for b in bs], [{k: v.grad for k, v in p.items()} for p in ps]


def test_gradients_of_the_stack():
    """8-bit products carry a relative error of about 1 / (127 sqrt(3)) of the largest value a row holds: a few percent of a
    gradient after three blocks.  The directions have to agree to 0.99 and the lengths to a tenth."""
    model = block_train.Stack(3, 192)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(500, 192, generator=g, device="cuda")
    target = torch.randn(500, 192, generator=g, device="cuda")
    want_loss, dw, db, dn = _plain(model, x, target)
    y = model.forward(x)
    diff = y - target
    model.backward(diff * (2.0 / diff.numel()))
    assert abs(float((diff * diff).mean()) - float(want_loss)) <= 0.02 * float(want_loss)
    pairs = list(zip(model.dw + model.db, dw + db))
    for got, want in zip(model.dnorm, dn):
        pairs += [(got["dgate"], want["gate"]), (got["dw_post"], want["w_post"]), (got["dw_pre"], want["w_pre"])]
    for got, want in pairs:
        a, b = got.double().flatten(), want.flatten()
        assert float(a @ b) >= 0.99 * float(a.norm() * b.norm())
        assert abs(float(a.norm() / b.norm()) - 1) <= 0.1


@pytest.mark.parametrize("state_bits", [8, 32])
def test_loss_falls(state_bits):
    losses = block_train.train(depth=2, dim=256, tokens=1024, steps=60, state_bits=state_bits, lr=3e-3)
    assert losses[-1] < 0.5 * losses[0]
