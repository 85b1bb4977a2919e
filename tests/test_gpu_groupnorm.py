"""Group norm with an activation against the formulas in 64 bits.

Tolerances, by element.  Means and variances are sums of at most n = 64 + P / 8 fp32 numbers that follow one another, so k = (x - mean) rstd is off by
n 2^-24 (|k| + 1 + |mean| rstd); z = k w + b adds a few roundings; a sigmoid is good to 2^-20 of itself (2^-22 in fp32); outputs are rounded to
their type once.  The gradients' group means are sums of as many numbers, each as far off as its terms.  The slope of a ReLU jumps at z = 0:
elements whose z is within its own tolerance of 0 are left out, and count with their whole size in the sums over their group and channel.
"""
import math

import pytest
import torch

from paper_2407_12637_b200 import cnn, lbt

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
ACTS = ["none", "relu", "silu"]


def _inputs(shape, dtype, pdtype, seed=0, mean=0.7):
    g = torch.Generator(device="cuda").manual_seed(seed)
    C = shape[-1]
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = randn(*shape) * (0.5 + torch.rand(C, generator=g, device="cuda")) + randn(C) * 0.5 + mean
    return x.to(dtype), randn(*shape).mul(0.1).to(dtype), (1 + 0.3 * randn(C)).to(pdtype), (0.3 * randn(C)).to(pdtype)


def _check(x, dy, w, b, G, act, eps, y=None, grads=None):
    N, C = x.shape[0], x.shape[-1]
    P = x[0].numel() // C
    X, E = x.double().reshape(N, P, G, C // G), dy.double().reshape(N, P, G, C // G)
    W = (w.double() if w is not None else torch.ones(C, device="cuda").double()).view(G, -1)
    B = (b.double() if b is not None else torch.zeros(C, device="cuda").double()).view(G, -1)
    mean = X.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(((X - mean) ** 2).mean((1, 3), keepdim=True) + eps)
    k = (X - mean) * rstd
    n = (64 + P / 8) * EPS
    ek = n * (k.abs() + 1 + mean.abs() * rstd)
    z = k * W + B
    ez = ek * W.abs() + 4 * EPS * (z.abs() + (k * W).abs() + B.abs())
    sig, esig = torch.sigmoid(z), (2.0 ** -22 if x.dtype == torch.float32 else 2.0 ** -20)
    border = (z.abs() <= ez) if act == "relu" else torch.zeros_like(z, dtype=torch.bool)
    if y is not None:
        want = {"none": z, "relu": z.clamp(min=0), "silu": z * sig}[act]
        tol = (1.2 if act == "silu" else 1) * ez + 1.01 * HALF_ULP[y.dtype] * want.abs() + (esig * want.abs() if act == "silu" else 0)
        err = (y.double().reshape(want.shape) - want).abs()
        tol = tol + (2.0 ** -25 if y.dtype == torch.float16 else 1e-37)
        assert (err <= tol).all(), float((err / tol).max())
    if grads is None:
        return
    slope = {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": sig * (1 + z * (1 - sig))}[act]
    eslope = (0.5 * ez + esig * (sig * (1 + z.abs()))) if act == "silu" else border.double()
    e, ee = E * slope, E.abs() * (eslope + 4 * EPS * slope.abs())
    we, wee = e * W, ee * W.abs()
    m1, m2 = we.mean((1, 3), keepdim=True), (we * k).mean((1, 3), keepdim=True)
    s1, s2 = (wee + n * we.abs()).mean((1, 3), keepdim=True), (wee * k.abs() + we.abs() * (ek + n * k.abs())).mean((1, 3), keepdim=True)
    dx = rstd * (we - m1 - k * m2)
    tol = rstd * (wee + s1 + k.abs() * s2 + ek * m2.abs() + (n + 8 * EPS) * (we.abs() + m1.abs() + (k * m2).abs())) + 1.01 * HALF_ULP[x.dtype] * dx.abs()
    tol = tol + (2.0 ** -25 if x.dtype == torch.float16 else 1e-37)
    err = (grads["dx"].double().reshape(dx.shape) - dx).abs()
    ok = (err <= tol) | border
    assert ok.all(), float((err / tol)[~border].max())
    n2 = (64 + P / 8 + N) * EPS
    for name, want, terms, p in (("dw", (e * k).sum((0, 1)), ee * k.abs() + e.abs() * (ek + n2 * k.abs()), w), ("db", e.sum((0, 1)), ee + n2 * e.abs(), b)):
        assert (name in grads) == (p is not None)
        if p is not None:
            tol = terms.sum((0, 1)) + 1.01 * HALF_ULP[p.dtype] * want.abs() + 1e-30
            err = (grads[name].double().view(G, -1) - want).abs()
            assert (err <= tol).all(), (name, float((err / tol).max()))


def _run(shape, G, dtype, act, pdtype=torch.float32, eps=1e-5, seed=0, mean=0.7, params=True):
    x, dy, w, b = _inputs(shape, dtype, pdtype, seed, mean)
    if not params:
        w = b = None
    norm = cnn.GroupNorm(shape[-1], G, w, b, eps=eps, act=act)
    y = norm.forward(x, keep=True)
    _check(x, dy, w, b, G, act, eps, y, norm.backward(dy))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", list(HALF_ULP), ids=str)
@pytest.mark.parametrize("shape,G", [((3, 7, 9, 64), 8), ((2, 5, 5, 90), 6), ((2, 33, 17, 15), 5), ((1, 1, 1, 32), 4), ((4, 11, 8), 1), ((2, 6, 6, 48), 48),
                                     ((5, 3, 513), 27), ((1, 2, 1030), 2), ((2, 200, 24), 3)])
def test_forward_and_gradients(shape, G, dtype, act):
    _run(shape, G, dtype, act, seed=G)


@pytest.mark.parametrize("shape,G,dtype,act", [((1, 40000, 64), 8, torch.float32, "silu"), ((2, 30001, 66), 11, torch.bfloat16, "silu"),
                                               ((1, 9000, 333), 9, torch.float16, "none"), ((3, 700, 2304), 4, torch.bfloat16, "silu"),
                                               ((1, 300, 4099), 1, torch.float32, "none"), ((2, 9216, 64), 16, torch.float16, "silu"),
                                               ((700, 9, 40), 5, torch.float32, "silu"), ((1, 3000, 2050), 2, torch.float16, "relu")])
def test_images_that_do_not_fit_on_chip_and_many_of_them(shape, G, dtype, act):
    _run(shape, G, dtype, act, seed=3)


@pytest.mark.parametrize("pdtype", list(HALF_ULP), ids=str)
def test_parameter_types(pdtype):
    _run((3, 40, 32), 4, torch.bfloat16, "silu", pdtype=pdtype, seed=5)


def test_without_parameters():
    _run((3, 40, 30), 3, torch.float32, "silu", params=False, seed=7)


@pytest.mark.parametrize("P", [50, 60000])
def test_a_mean_far_from_zero(P):
    """Values of 300 +- 1, the first pixel 0: the variance does not lose itself in the mean."""
    x, dy, w, b = _inputs((2, P, 32), torch.float32, torch.float32, seed=9, mean=300.0)
    x[:, 0] = 0.0
    norm = cnn.GroupNorm(32, 4, w, b)
    y = norm.forward(x, keep=True)
    _check(x, dy, w, b, 4, "none", 1e-5, y, norm.backward(dy))


def test_a_constant_image():
    """Variance 0: rstd is the root of 1 / eps, k what the mean's rounding leaves of 0 times that, y the activation of b but for it."""
    x, dy = torch.full((2, 50, 16), 3.0, device="cuda"), torch.ones(2, 50, 16, device="cuda")
    w, b = torch.ones(16, device="cuda"), torch.linspace(-1, 1, 16, device="cuda")
    norm = cnn.GroupNorm(16, 4, w, b, act="relu")
    y = norm.forward(x, keep=True)
    _check(x, dy, w, b, 4, "relu", 1e-5, y, norm.backward(dy))


def test_an_image_that_is_not_finite_stays_alone():
    for shape in ((3, 60, 24), (3, 60000, 24), (3, 61, 23)):
        x, dy, w, b = _inputs(shape, torch.float32, torch.float32, seed=11)
        norm = cnn.GroupNorm(shape[-1], 1, w, b, act="silu")
        want, dx = norm.forward(x, keep=True).clone(), norm.backward(dy)["dx"].clone()
        for bad in (math.nan, math.inf):
            x[1, 5, 3] = bad
            y = norm.forward(x, keep=True)
            got = norm.backward(dy)["dx"]
            assert torch.equal(y[[0, 2]], want[[0, 2]]) and torch.equal(got[[0, 2]], dx[[0, 2]])
            assert not torch.isfinite(y[1, 5, 3]) and y[1].isnan().sum() >= 1


def test_strides_neighbours_and_in_place():
    """Channels of a wider tensor: what lies beside them stays; the output in the input's place is the same."""
    for width, pad in ((32, 8), (30, 3), (30, 2)):
        x, dy, w, b = _inputs((2, 9, 7, width + pad), torch.bfloat16, torch.float32, seed=13)
        w, b = w[:width].contiguous(), b[:width].contiguous()
        norm = cnn.GroupNorm(width, 2, w, b, act="silu")
        out, dx = torch.full_like(x, 5.0), torch.full_like(x, 5.0)
        norm.forward(x[..., :width], out=out[..., :width], keep=True)
        grads = norm.backward(dy[..., :width], dx=dx[..., :width])
        _check(x[..., :width].contiguous(), dy[..., :width].contiguous(), w, b, 2, "silu", 1e-5, out[..., :width].contiguous(), {**grads, "dx": dx[..., :width].contiguous()})
        assert (out[..., width:] == 5.0).all() and (dx[..., width:] == 5.0).all()
        assert torch.equal(norm.backward(dy[..., :width], dx=dy[..., :width])["dx"].contiguous(), dx[..., :width].contiguous())
        assert torch.equal(norm.forward(x[..., :width], out=x[..., :width]).contiguous(), out[..., :width].contiguous())


def test_gradient_against_differences():
    """Along random directions, by a central difference of the kernel's own fp32 outputs: off by the step's square times a third derivative, which is
    below 8 of the loss's terms here (directions of size 1, rstd about 1), and by the outputs' rounding over the step."""
    x, dy, w, b = _inputs((2, 16, 8), torch.float32, torch.float32, seed=15)
    g = torch.Generator(device="cuda").manual_seed(16)
    d = {k: torch.randn(v.shape, generator=g, device="cuda") for k, v in (("x", x), ("w", w), ("b", b))}
    step = 2.0 ** -6
    loss = lambda s: float((cnn.GroupNorm(8, 2, w + s * d["w"], b + s * d["b"], act="silu").forward(x + s * d["x"]).double() * dy.double()).sum())  # noqa: E731
    norm = cnn.GroupNorm(8, 2, w, b, act="silu")
    norm.forward(x, keep=True)
    grads = norm.backward(dy)
    want = sum(float((grads[n].double() * d[k].double()).sum()) for n, k in (("dx", "x"), ("dw", "w"), ("db", "b")))
    size = float(dy.double().abs().sum())
    assert abs((loss(step) - loss(-step)) / (2 * step) - want) <= size * (8 * step ** 2 + 16 * EPS / step)


@pytest.mark.parametrize("bits", [2, 4, 5, 8])
@pytest.mark.parametrize("shape,G,act", [((3, 7, 9, 64), 8, "relu"), ((2, 31, 16), 2, "silu"), ((2, 40000, 24), 3, "relu"), ((1, 9, 2064), 2, "none")])
def test_codes_are_those_of_the_quantizer(shape, G, act, bits):
    x, _, w, b = _inputs(shape, torch.float32, torch.float32, seed=17)
    norm = cnn.GroupNorm(shape[-1], G, w, b, act=act)
    y = norm.forward(x)
    for clip in (1.5, 0.0, math.inf):
        c = torch.tensor([clip], device="cuda")
        q, scale = norm.forward_codes(x, c, bits=bits)
        want, s = torch.empty_like(q), torch.empty(1, device="cuda")
        lbt.quantize_act(y, c, bits, want, s)
        assert torch.equal(q, want) and torch.equal(scale, s)
    kept = torch.empty_like(y)
    norm.forward_codes(x, torch.tensor([1.5], device="cuda"), bits=bits, out=kept)
    assert torch.equal(kept, y)


def test_between_two_quantized_convolutions():
    """The norm's codes go into the next convolution's product as they are, and that convolution's dX comes back through the norm."""
    N, H, C, K = 2, 8, 32, 16
    x, _, w, b = _inputs((N, H, H, C), torch.float32, torch.float32, seed=19)
    norm = cnn.GroupNorm(C, 8, w, b, act="relu")
    clip = torch.tensor([2.0], device="cuda")
    desc = lbt.ConvDesc(N=N, C=C, H=H, W=H, K=K, R=3, S=3, stride=1, pad=1)
    q_w = torch.randint(0, 256, (K * 9 * C // 2,), dtype=torch.uint8, device="cuda")
    s_w = torch.tensor([0.05], device="cuda")
    ws = torch.empty(max(lbt.workspace_bytes(op, desc) for op in (lbt.OP_CONV_FORWARD, lbt.OP_CONV_BACKWARD)), dtype=torch.uint8, device="cuda")
    q, s_x = norm.forward_codes(x, clip, bits=4, keep=True)
    y = norm.forward(x)
    q2, s2 = torch.empty_like(q), torch.empty(1, device="cuda")
    lbt.quantize_act(y, clip, 4, q2, s2)
    outs = []
    for codes, scale in ((q, s_x), (q2, s2)):
        out = torch.empty(N, H, H, K, device="cuda")
        lbt.qconv_forward(desc, codes, q_w, scale, s_w, out, None, 4, 4, ws)
        outs.append(out)
    assert torch.equal(*outs)
    state, stats = lbt.new_state(gamma=0.5, rounding=lbt.ROUND_NEAREST), lbt.new_stats()
    dX, dY = torch.empty(N, H, H, C, device="cuda"), torch.randn(N, H, H, K, device="cuda")
    lbt.qconv_backward(desc, dY, q_w, q, s_w, s_x, state, stats, torch.empty(dY.numel() // 2, dtype=torch.uint8, device="cuda"), dX, None, None, None, 4, ws)
    _check(x, dX, w, b, 8, "relu", 1e-5, grads=norm.backward(dX))


def test_streams_graphs_and_the_same_bits():
    x, dy, w, b = _inputs((4, 12, 12, 64), torch.bfloat16, torch.float32, seed=21)
    norm, side = cnn.GroupNorm(64, 8, w, b, act="silu"), torch.cuda.Stream()
    want = norm.forward(x, keep=True).clone()
    grads = {k: v.clone() for k, v in norm.backward(dy).items()}
    side.wait_stream(torch.cuda.current_stream())
    y = norm.forward(x, keep=True, stream=side)
    got = norm.backward(dy, stream=side)
    side.synchronize()
    assert torch.equal(y, want) and all(torch.equal(got[k], grads[k]) for k in grads)
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            y = norm.forward(x, keep=True)
            graphs[-1].result = (y, norm.backward(dy))
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for graph in graphs:
        y, got = graph.result
        assert torch.equal(y, want) and all(torch.equal(got[k], grads[k]) for k in grads)
    norm.forward(x, keep=True)
    assert torch.equal(norm.backward(dy)["dx"], grads["dx"])


def test_no_image():
    norm = cnn.GroupNorm(16, 2, torch.ones(16, device="cuda"), torch.ones(16, device="cuda"))
    x = torch.empty(0, 5, 16, device="cuda")
    assert norm.forward(x, keep=True).shape == x.shape
    grads = norm.backward(x)
    assert grads["dx"].shape == x.shape and not grads["dw"].any() and not grads["db"].any()


def test_refusals():
    x, dy, w, b = _inputs((2, 5, 5, 16), torch.float32, torch.float32)
    norm = cnn.GroupNorm(16, 2, w, b)
    for bad in (lambda: cnn.GroupNorm(16, 3), lambda: cnn.GroupNorm(16, 2, w[:8]), lambda: cnn.GroupNorm(16, 2, w, b.half()), lambda: cnn.GroupNorm(16, 2, act="gelu"),
                lambda: norm.forward(x[..., :8]), lambda: norm.forward(x.permute(0, 3, 1, 2)), lambda: norm.forward(x[:, ::2]), lambda: norm.forward(x, out=torch.empty_like(x).half()),
                lambda: norm.forward(x.cpu()), lambda: norm.forward(x, out=torch.empty_like(x)[:1]), lambda: norm.forward(x[:, :1, :1, :].expand(2, 5, 5, 16)),
                lambda: norm.forward_codes(x, torch.tensor([1.0, 2.0], device="cuda")), lambda: norm.forward_codes(x, None)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        norm.backward(dy)
    with pytest.raises(lbt.LbtError):   # codes of a width that is no multiple of eight
        cnn.GroupNorm(12, 2).forward_codes(torch.zeros(2, 4, 12, device="cuda"), torch.ones(1, device="cuda"))
    with pytest.raises(lbt.LbtError):
        norm.forward_codes(x, torch.ones(1, device="cuda"), bits=9)
    norm.forward(x, keep=True)
    with pytest.raises(ValueError):
        norm.backward(dy, dw=torch.zeros(8, device="cuda"))
