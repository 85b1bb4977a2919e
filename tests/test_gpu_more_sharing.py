"""Adapters, group norm and gradient clipping where threads share an object or tensors share memory, on the device."""
import threading

import pytest
import torch

from paper_2407_12637_b200 import cnn, lbt, lm

pytestmark = pytest.mark.gpu


def test_two_threads_share_a_group_norm():
    """Images too large for a cluster, two launches a pass, on the default stream: the bits that each thread gets alone."""
    norm = cnn.GroupNorm(24, 3, act="silu")
    xs = [torch.randn(2, 40000, 24, device="cuda") * (i + 1) + i for i in range(2)]
    want, got = [norm.forward(x) for x in xs], [[], []]

    def work(i):
        for _ in range(100):
            got[i].append(norm.forward(xs[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(2) for y in got[i])


def test_two_threads_share_adapters():
    """Forward passes without `keep`, and gradients of two dy for one kept pass, on the default stream."""
    g = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    adapters = lm.Adapters(randn(2, 8, 96), randn(2, 8, 64))
    offsets, index = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 100, 300], [1, 0]))
    x, base, dys, xs = randn(300, 96), randn(300, 64), [randn(300, 64) * (i + 1) for i in range(2)], [randn(300, 96) for _ in range(2)]
    adapters.forward(x, base.clone(), offsets, index, keep=True)
    passes = [lambda i=i: (adapters.forward(xs[i], base, offsets, index, out=torch.empty_like(base)), *adapters.backward(dys[i], torch.zeros(300, 96, device="cuda")).values())
              for i in range(2)]
    want, got = [p() for p in passes], [[], []]

    def work(i):
        for _ in range(100):
            got[i].append(passes[i]())

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for out in got[i] for a, b in zip(out, want[i]))


def test_adapters_out_in_the_place_of_x():
    """Refused where backward reads x, whatever tensor lies there; without `keep` the same as elsewhere."""
    g = torch.Generator(device="cuda").manual_seed(2)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    for M, I, dtype in ((5, 64, torch.float32), (300, 96, torch.bfloat16), (300, 63, torch.bfloat16), (700, 128, torch.float16)):
        adapters, x, base = lm.Adapters(randn(1, 8, I).to(dtype), randn(1, 8, I).to(dtype)), randn(M, I).to(dtype), randn(M, I).to(dtype)
        want, before = adapters.forward(x, base, out=torch.empty_like(x)), x.clone()
        for bad in (lambda: adapters.forward(x, base, out=x, keep=True), lambda: adapters.forward(x, base, out=x.view(M, I), keep=True), lambda: adapters.forward(x, x[:], keep=True)):
            with pytest.raises(ValueError):
                bad()
        assert torch.equal(x, before) and adapters.kept is None
        assert torch.equal(adapters.forward(x, base, out=x), want)


def test_group_norm_out_in_the_place_of_x():
    for shape in ((2, 9, 16), (2, 40000, 24)):
        x, clip = torch.randn(*shape, device="cuda"), torch.ones(1, device="cuda")
        norm = cnn.GroupNorm(shape[-1], 2)
        want, before = norm.forward(x), x.clone()
        for bad in (lambda: norm.forward(x, out=x, keep=True), lambda: norm.forward(x, out=x[:], keep=True), lambda: norm.forward_codes(x, clip, out=x, keep=True)):
            with pytest.raises(ValueError):
                bad()
        assert torch.equal(x, before) and norm.kept is None
        norm.forward(x, out=torch.empty_like(x), keep=True)
        q, s = norm.forward_codes(x, clip)
        assert torch.equal(norm.forward(x, out=x), want)
        x.copy_(before)
        got = norm.forward_codes(x, clip, out=x)
        assert torch.equal(x, want) and torch.equal(got[0], q) and torch.equal(got[1], s)


def test_clipped_outputs_lie_apart():
    """Outputs in other gradients' places are refused; in flat storage side by side, in place or elsewhere, they hold what each alone would."""
    flat, other = torch.randn(300, device="cuda"), torch.zeros(300, device="cuda")
    cut = lambda t: [t[0:100], t[100:101], t[101:300]]  # noqa: E731
    before = flat.clone()
    for out in ([flat[1:101], other[100:101], other[101:300]], [other[0:100], flat[0:1], other[101:300]], [other[0:100], other[99:100], other[101:300]]):
        with pytest.raises(ValueError):
            lm.GradClip(cut(flat), 1.0, out=out)
    for out in (cut(other), cut(flat)):
        lm.GradClip(cut(flat), 1.0, out=out).clip()
    want = before * (1.0 / before.double().norm()).float()
    assert torch.equal(other, flat) and ((other - want).abs() <= 2.0 ** -22 * want.abs()).all()


@pytest.mark.parametrize("clip", [1.5, 0.0])
def test_codes_of_no_images(clip):
    c, x, want = torch.tensor([clip], device="cuda"), torch.empty(0, 5, 16, device="cuda"), torch.empty(1, device="cuda")
    used = torch.full((1,), 7.0, device="cuda")   # (what the next allocation of that size may find)
    del used
    q, scale = cnn.GroupNorm(16, 2).forward_codes(x, c, bits=4)
    lbt.quantize_act(x, c, 4, torch.empty_like(q), want)
    assert q.numel() == 0 and torch.equal(scale, want) and float(want) == torch.tensor(clip / 15).float()
