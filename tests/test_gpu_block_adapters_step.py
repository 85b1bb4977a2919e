"""What a step of the example with adapters changes: the adapters' masters and copies, the norms; and what it leaves: the 8-bit weights and their biases."""
import pytest
import torch

from paper_2407_12637_b200 import block_train

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_norm", [None, 1e-3])
def test_a_step_trains_the_adapters(max_norm):
    model = block_train.Stack(2, 128, rank=4, max_norm=max_norm)
    g = torch.Generator(device="cuda").manual_seed(7)
    x, target = torch.randn(96, 128, generator=g, device="cuda").bfloat16(), torch.randn(96, 128, generator=g, device="cuda")
    frozen = [t for layer in model.layers for t in (layer.q_w, layer.s_w, layer.bias)]
    before, kept = [t.clone() for t in model.optimizer.params], [t.clone() for t in frozen]
    for _ in range(2):   # (B begins at 0: in the first step nothing reaches A)
        model.step(x, target)
    model.check()
    assert all(torch.equal(a, b) for a, b in zip(frozen, kept))
    assert all(not torch.equal(a, b) and a.isfinite().all() for a, b in zip(model.optimizer.params, before))
    for adapters, (a, b), da, db in zip(model.adapters, model.masters, model.dw, model.db):
        assert torch.equal(adapters.a, a.bfloat16()) and torch.equal(adapters.b, b.bfloat16()) and b.any() and da.any() and db.any()
