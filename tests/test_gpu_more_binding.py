"""The binding's functions of gradient norm, adapters and group norm: the bits of the objects that make the same calls themselves."""
import pytest
import torch

from paper_2407_12637_b200 import cnn, lbt, lm

pytestmark = pytest.mark.gpu


def _randn(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s, dtype=torch.float32: torch.randn(*s, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("stream", [None, "side"])
def test_gradient_norm_and_clipping(stream):
    randn, stream = _randn(1), torch.cuda.Stream() if stream else None
    grads = [randn(n, dtype=t) for n, t in ((5000, torch.float32), (1, torch.bfloat16), (777, torch.float16), (0, torch.float32))]
    want, out = [torch.empty(g.shape, device="cuda") for g in grads], [torch.empty(g.shape, device="cuda") for g in grads]
    clip, s = lm.GradClip(grads, 0.5, out=want), torch.tensor([0.25], device="cuda")
    clip.clip(grad_scale=s)
    table = (lbt.GradTensor * 4)(*[lbt.GradTensor(g.data_ptr(), o.data_ptr(), g.numel(), lbt.TYPES[g.dtype], lbt.F32) for g, o in zip(grads, out)])
    result, norms = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda")
    torch.cuda.synchronize()
    lbt.grad_norm(table, result, 0.5, norms, s, stream=stream)
    lbt.grad_clip(table, result, stream=stream)
    torch.cuda.synchronize()
    parts = result.view(torch.float32)
    assert torch.equal(parts[0:1], clip.norm) and torch.equal(parts[1:2], clip.scale) and torch.equal(result[2:3], clip.skip) and not result[3]
    assert torch.equal(norms, clip.norms) and all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_adapters(dtype):
    randn = _randn(2)
    n, r, M, I, O = 3, 8, 70, 64, 40
    a, b, scale = randn(n, r, I, dtype=dtype), randn(n, r, O, dtype=dtype), randn(n)
    x, base, dy, dbase = (randn(M, w, dtype=dtype) for w in (I, O, O, I))
    offsets, index = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 30, 30, 65, 70], [2, 0, -1, 1]))
    adapters = lm.Adapters(a, b, scale)
    y = adapters.forward(x, base, offsets, index, out=torch.empty_like(base), keep=True)
    want = adapters.backward(dy, dbase, dx=torch.empty_like(x))
    d = lbt.AdaptersDesc(M, I, O, 4, n, r, lbt.TYPES[dtype], 0)
    out, h, status = torch.empty_like(base), torch.empty(M, r, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    dx, da, db = torch.empty_like(x), torch.empty(n, r, I, device="cuda"), torch.empty(n, r, O, device="cuda")
    lbt.adapters_forward(d, x, a, b, scale, offsets, index, base, out, h, status)
    lbt.adapters_backward(d, dy, x, h, a, b, scale, offsets, index, dbase, dx, da, db, dev_status=status)
    assert torch.equal(out, y) and torch.equal(dx, want["dx"]) and torch.equal(da, want["da"]) and torch.equal(db, want["db"]) and not status
    half = [torch.empty_like(a), torch.empty_like(b)]   # one gradient at a time, of the adapters' type
    lbt.adapters_backward(d, dy, x, h, a, b, scale, offsets, index, da=half[0], grad_type=lbt.TYPES[dtype])
    lbt.adapters_backward(d, dy, x, h, a, b, scale, offsets, index, db=half[1], grad_type=lbt.TYPES[dtype])
    assert torch.equal(half[0], da.to(dtype)) and torch.equal(half[1], db.to(dtype))


@pytest.mark.parametrize("P", [50, 60000])
def test_group_norm(P):
    randn = _randn(3)
    x, dy, w, b, clip = randn(2, P, 24), randn(2, P, 24), randn(24), randn(24), torch.ones(1, device="cuda")
    norm = cnn.GroupNorm(24, 3, w, b, act="silu")
    y = norm.forward(x, keep=True)
    want = norm.backward(dy)
    q, s = norm.forward_codes(x, clip)
    d = lbt.GroupnormDesc(2, P, 24, 3, lbt.F32, lbt.F32, lbt.ACT_SILU, 1e-5)
    out, codes, scale, stats = torch.empty_like(x), torch.empty_like(q), torch.empty(1, device="cuda"), torch.empty(2, 3, 2, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    lbt.groupnorm_forward(d, x, w, b, out, codes, 4, clip, scale, stats)
    lbt.groupnorm_backward(d, dy, x, w, b, stats, dx, dw, db)
    for got, ref in ((out, y), (codes, q), (scale, s), (dx, want["dx"]), (dw, want["dw"]), (db, want["db"])):
        assert torch.equal(got, ref)
