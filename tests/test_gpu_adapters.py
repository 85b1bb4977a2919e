"""Low-rank adapters against the formulas in 64 bits.

Tolerances, by element, from magnitudes formed in 64 bits.  H = sum |x| |A| bounds h's terms: at most 40 + I / 64 sums follow one another
(a step's four or eight instructions, the steps of a warp, the warps and CTAs), each off by 2^-23 of what it holds (the tensor core cuts
off): e_h = (40 + I / 64) 2^-23 H; fp32 operands are split into two parts that leave 2^-20 of a product.  h enters its second product with 2^-16 of it lost
for bf16 (two parts of 8 bits), 2^-20 for the others, and 2 rank / 8 + 8 sums follow.  Weight gradients: f's own error, 2^-20 of each term, and at
most 40 + tokens / 64 sums.  Outputs are then rounded to their type once.
"""
import math

import pytest
import torch

from paper_2407_12637_b200 import lm

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = list(HALF_ULP)
PART = {torch.float32: 2.0 ** -20, torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -20}
OP = {torch.float32: 2.0 ** -20, torch.bfloat16: 0.0, torch.float16: 0.0}


def _make(M, I, O, r, n, dtype, seed=0, pad=0, scale=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    rows = lambda w, std=1.0: (randn(M, w + pad) * std).to(dtype)[:, :w]  # noqa: E731
    a, b = (randn(n, r, I) * I ** -0.5).to(dtype), (randn(n, r, O) * r ** -0.5).to(dtype)
    s = (0.5 + torch.rand(n, generator=g, device="cuda")) if scale else None
    return {"x": rows(I), "base": rows(O), "dy": rows(O, 0.1), "dbase": rows(I, 0.1), "a": a, "b": b, "scale": s}


def _runs(lengths, ids, start=0):
    offs = [start]
    for n in lengths:
        offs.append(offs[-1] + n)
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return t(offs), t(ids), [(slice(lo, hi), i) for lo, hi, i in zip(offs, offs[1:], ids)]


def _side(x, base, a, b, s, rank, dtype):
    """One run: (h, its error bound, base + s h b, its bound)."""
    x, a, b = x.double(), a.double(), b.double()
    h, H = x @ a.T, x.abs() @ a.abs().T
    eh = H * ((40 + x.shape[1] / 64) * 2.0 ** -23 + OP[dtype])
    out = base.double() + s * (h @ b)
    tol = s * ((eh + h.abs() * (PART[dtype] + OP[dtype] + (rank / 4 + 8) * 2.0 ** -23)) @ b.abs()) + 1.01 * HALF_ULP[dtype] * out.abs() + 2.0 ** -24 * base.double().abs()
    return h, eh, out, tol + (2.0 ** -25 if dtype == torch.float16 else 0)


def _check(t, runs, dtype, y, grads=None):
    n, rank, _ = t["a"].shape
    scale = t["scale"].double() if t["scale"] is not None else torch.ones(n, dtype=torch.float64, device="cuda")
    da, db = (torch.zeros_like(t[k], dtype=torch.float64) for k in ("a", "b"))
    ta, tb = torch.zeros_like(da), torch.zeros_like(db)
    for at, i in runs:
        if i < 0 or i >= n:
            assert torch.equal(y[at], t["base"][at])
            if grads:
                assert torch.equal(grads["dx"][at], t["dbase"][at])
            continue
        x, dy = t["x"][at], t["dy"][at]
        h, eh, out, tol = _side(x, t["base"][at], t["a"][i], t["b"][i], scale[i], rank, dtype)
        assert ((y[at].double() - out).abs() <= tol).all(), float(((y[at].double() - out).abs() / tol).max())
        if grads is None:
            continue
        dh, edh, dx, tdx = _side(dy, t["dbase"][at], t["b"][i], t["a"][i], scale[i], rank, dtype)
        assert ((grads["dx"][at].double() - dx).abs() <= tdx).all(), float(((grads["dx"][at].double() - dx).abs() / tdx).max())
        step = 2.0 ** -20 + OP[dtype] + (40 + x.shape[0] / 64) * 2.0 ** -23
        da[i] += scale[i] * dh.T @ x.double()
        db[i] += scale[i] * h.T @ dy.double()
        ta[i] += scale[i] * (edh + dh.abs() * step).T @ x.double().abs()
        tb[i] += scale[i] * (eh + h.abs() * step).T @ dy.double().abs()
    if grads:
        for name, want, tol in (("da", da, ta), ("db", db, tb)):
            got = grads[name]
            tol = tol + 1.01 * HALF_ULP[got.dtype] * want.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 1e-30)
            assert ((got.double() - want).abs() <= tol).all(), (name, float(((got.double() - want).abs() / tol).max()))


LAYOUTS = {"one": ([77], [0]), "tokens": ([1] * 9, [0, 1, 2, -1, 1, 1, 0, 2, 5]), "ragged": ([0, 5, 130, 0, 33, 16, 1], [2, 1, 0, 0, 1, -1, 2]),
           "long": ([300, 129], [1, 0])}


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("I,O", [(64, 128), (520, 264), (131, 77), (66, 1)])
@pytest.mark.parametrize("rank", [1, 16, 40])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_forward_and_gradients(dtype, rank, I, O, layout):
    lengths, ids = LAYOUTS[layout]
    offsets, index, runs = _runs(lengths, ids)
    t = _make(sum(lengths), I, O, rank, 3, dtype, seed=rank + I)
    ad = lm.Adapters(t["a"], t["b"], t["scale"])
    y = ad.forward(t["x"], t["base"], offsets, index, out=torch.empty_like(t["base"]), keep=True)
    grads = ad.backward(t["dy"], t["dbase"], dx=torch.empty_like(t["dbase"]))
    assert grads["da"].dtype == torch.float32
    _check(t, runs, dtype, y, grads)


@pytest.mark.parametrize("M,I,O,rank,dtype", [(1, 4096, 4096, 16, torch.bfloat16), (2500, 512, 1024, 16, torch.bfloat16), (1100, 1024, 512, 64, torch.float16),
                                             (2100, 513, 259, 24, torch.bfloat16), (1100, 515, 130, 63, torch.float16), (4200, 256, 129, 8, torch.float32),
                                             (600, 640, 200, 128, torch.bfloat16), (600, 333, 200, 100, torch.float32), (4300, 64, 64, 128, torch.float16),
                                             (9000, 128, 128, 3, torch.float32)])
def test_sizes_of_every_kernel(M, I, O, rank, dtype):
    """One run of all tokens (no run given at all), aligned and not, few tokens and tiles of 128."""
    t = _make(M, I, O, rank, 2, dtype, seed=M)
    ad = lm.Adapters(t["a"], t["b"], t["scale"])
    y = ad.forward(t["x"], t["base"], out=torch.empty_like(t["base"]), keep=True)
    _check(t, [(slice(0, M), 0)], dtype, y, ad.backward(t["dy"], t["dbase"], dx=torch.empty_like(t["dbase"])))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_many_short_runs(dtype):
    """More runs than a warp looks at together, most of one token, adapters in no order; one adapter has none."""
    g = torch.Generator().manual_seed(1)
    ids = torch.randint(-1, 5, (150,), generator=g).tolist()
    ids = [6 if i == 4 else i for i in ids]   # (of seven: 4 and 5 have no token)
    lengths = torch.randint(0, 4, (150,), generator=g).tolist()
    offsets, index, runs = _runs(lengths, ids)
    t = _make(sum(lengths), 200, 136, 16, 7, dtype, seed=2)
    ad = lm.Adapters(t["a"], t["b"], t["scale"])
    y = ad.forward(t["x"], t["base"], offsets, index, out=torch.empty_like(t["base"]), keep=True)
    grads = ad.backward(t["dy"], t["dbase"], dx=torch.empty_like(t["dbase"]))
    _check(t, runs, dtype, y, grads)
    assert not grads["da"][4:6].any() and not grads["db"][4:6].any()


@pytest.mark.parametrize("pad", [8, 3])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_rows_of_wider_matrices_keep_their_neighbours(dtype, pad):
    lengths, ids = [140, 3], [0, 1]
    offsets, index, runs = _runs(lengths, ids, start=5)
    M = 160
    t = _make(M, 136, 72, 8, 2, dtype, seed=4, pad=pad)
    wide_y, wide_x = torch.full((M, 72 + pad), 9.0, device="cuda").to(dtype), torch.full((M, 136 + pad), 9.0, device="cuda").to(dtype)
    ad = lm.Adapters(t["a"], t["b"], t["scale"])
    ad.forward(t["x"], t["base"], offsets, index, out=wide_y[:, :72], keep=True)
    grads = ad.backward(t["dy"], t["dbase"], dx=wide_x[:, :136])
    _check(t, runs, dtype, wide_y[:, :72], grads)
    for w, width in ((wide_y, 72), (wide_x, 136)):   # columns beside the matrix; rows ahead of the first run and behind the last one
        assert (w[:, width:] == 9.0).all() and (w[:5] == 9.0).all() and (w[148:] == 9.0).all()


def test_a_tensor_that_begins_in_the_middle_of_a_word():
    """Two-byte aligned tensors: nothing ahead of their first element is read."""
    t = _make(50, 37, 23, 5, 1, torch.bfloat16, seed=6)
    shifted = {}
    for k, v in t.items():
        if k == "scale":
            continue
        raw = torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")
        shifted[k] = raw[1:].view(v.shape)
        shifted[k].copy_(v)
    ad = lm.Adapters(shifted["a"], shifted["b"], t["scale"])
    y = ad.forward(shifted["x"], shifted["base"], out=torch.empty_like(t["base"]), keep=True)
    grads = ad.backward(shifted["dy"], shifted["dbase"], dx=torch.empty_like(t["dbase"]))
    _check(t, [(slice(0, 50), 0)], torch.bfloat16, y, grads)


@pytest.mark.parametrize("M", [40, 2200])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_in_place_is_the_same_bits(dtype, M):
    t = _make(M, 96, 160, 16, 1, dtype, seed=8)
    ad = lm.Adapters(t["a"], t["b"])
    y = ad.forward(t["x"], t["base"], out=torch.empty_like(t["base"]), keep=True)
    dx = ad.backward(t["dy"], t["dbase"], dx=torch.empty_like(t["dbase"]))["dx"]
    base, dbase = t["base"].clone(), t["dbase"].clone()
    assert ad.forward(t["x"], base, keep=True) is base and torch.equal(base, y)
    assert ad.backward(t["dy"], dbase)["dx"] is dbase and torch.equal(dbase, dx)


def test_what_the_runs_may_hold():
    """Offsets are cut to the tokens, an index outside the adapters is none, no runs leave everything as it was."""
    t = _make(30, 64, 64, 4, 2, torch.bfloat16, seed=10)
    ad = lm.Adapters(t["a"], t["b"], t["scale"])
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    y = ad.forward(t["x"], t["base"], i32([-7, 4, 20, 1000]), i32([1, 2147483647, 0]), out=torch.full_like(t["base"], 5.0))
    _check(t, [(slice(0, 4), 1), (slice(4, 20), -1), (slice(20, 30), 0)], torch.bfloat16, y)
    out = torch.full_like(t["base"], 5.0)
    ad.forward(t["x"], t["base"], i32([0]), i32([]), out=out, keep=True)
    assert (out == 5.0).all()
    grads = ad.backward(t["dy"], t["dbase"], dx=out.clone())
    assert (grads["dx"] == 5.0).all() and not grads["da"].any() and not grads["db"].any()
    empty = t["x"][:0]
    ad.forward(empty, t["base"][:0], keep=True)
    grads = ad.backward(t["dy"][:0], t["dbase"][:0])
    assert not grads["da"].any() and not grads["db"].any()


@pytest.mark.parametrize("M", [20, 2300])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_a_token_that_is_not_finite_stays_alone(dtype, M):
    t = _make(M, 72, 80, 8, 1, dtype, seed=12)
    ad = lm.Adapters(t["a"], t["b"])
    want = ad.forward(t["x"], t["base"], out=torch.empty_like(t["base"])).clone()
    t["x"][3, 5], t["x"][17, 0], t["x"][11, 2] = math.nan, math.inf, -math.inf
    y = ad.forward(t["x"], t["base"], out=torch.empty_like(t["base"]))
    bad = [3, 11, 17]
    assert not torch.isfinite(y[bad]).any()
    rest = [m for m in range(M) if m not in bad]
    assert torch.equal(y[rest], want[rest])


def test_fp16_values_of_h_beyond_its_range():
    """h of 1e6 and of 1e-6, and gradients to match: neither overflows nor vanishes on the way."""
    for size in (3e4, 1e-4):
        t = _make(200, 64, 48, 16, 1, torch.float16, seed=14)
        t["x"].mul_(size / 100)
        t["a"].mul_(100.0 if size > 1 else 0.01)
        t["b"].mul_(1e-6 / size if size > 1 else 1.0)
        t["dy"].mul_(10.0 if size > 1 else 1e-3)
        ad = lm.Adapters(t["a"], t["b"], t["scale"])
        y = ad.forward(t["x"], t["base"], out=torch.empty_like(t["base"]), keep=True)
        _check(t, [(slice(0, 200), 0)], torch.float16, y, ad.backward(t["dy"], t["dbase"], dx=torch.empty_like(t["dbase"])))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_gradients_of_the_adapters_type_and_some_of_them(dtype):
    t = _make(90, 64, 40, 8, 2, dtype, seed=16)
    ad = lm.Adapters(t["a"], t["b"], t["scale"])
    offsets, index, runs = _runs([50, 40], [1, 0])
    y = ad.forward(t["x"], t["base"], offsets, index, out=torch.empty_like(t["base"]), keep=True)
    grads = ad.backward(t["dy"], t["dbase"], dx=torch.empty_like(t["dbase"]), grad_dtype=dtype)
    assert grads["da"].dtype == grads["db"].dtype == dtype
    _check(t, runs, dtype, y, grads)
    wide = ad.backward(t["dy"])
    assert set(wide) == {"da", "db"} and torch.equal(wide["da"].to(dtype), grads["da"]) and torch.equal(wide["db"].to(dtype), grads["db"])
    buffers = {k: torch.full_like(wide[k], 3.0) for k in ("da", "db")}
    again = ad.backward(t["dy"], **buffers)
    assert all(again[k] is buffers[k] and torch.equal(buffers[k], wide[k]) for k in buffers)


def test_gradients_against_differences():
    """d/dt of sum(dy * out) along a random direction of x, A and B, by a central difference of the kernel's own fp32 outputs: it is a cubic in
    the step, so the difference is off by step^2 / 6 of its third derivative (3 terms of the size of the value) and by the outputs' rounding over the step."""
    t = _make(64, 48, 40, 8, 1, torch.float32, seed=18)
    g = torch.Generator(device="cuda").manual_seed(19)
    d = {k: torch.randn(t[k].shape, generator=g, device="cuda") * t[k].abs().mean() for k in ("x", "a", "b")}
    step = 2.0 ** -7

    def loss(sign):
        ad = lm.Adapters(t["a"] + sign * step * d["a"], t["b"] + sign * step * d["b"])
        y = ad.forward(t["x"] + sign * step * d["x"], t["base"], out=torch.empty_like(t["base"]))
        return float((y.double() * t["dy"].double()).sum()), float((y.double().abs() * t["dy"].double().abs()).sum())
    (hi, size), (lo, _) = loss(1), loss(-1)
    ad = lm.Adapters(t["a"], t["b"])
    ad.forward(t["x"], t["base"], out=torch.empty_like(t["base"]), keep=True)
    grads = ad.backward(t["dy"], torch.zeros_like(t["dbase"]))
    want = sum(float((grads[n].double() * d[k].double()).sum()) for n, k in (("dx", "x"), ("da", "a"), ("db", "b")))
    third = float((t["dy"].double().abs() * ((d["x"].double().abs() @ d["a"][0].double().abs().T) @ d["b"][0].double().abs())).sum())
    assert abs((hi - lo) / (2 * step) - want) <= step ** 2 * third + size * 2.0 ** -20 / step


def test_the_same_call_gives_the_same_bits():
    t = _make(700, 264, 136, 16, 3, torch.bfloat16, seed=20)
    offsets, index, _ = _runs([100, 3, 597], [1, 0, 2])
    ad, seen = lm.Adapters(t["a"], t["b"], t["scale"]), None
    for _ in range(5):
        y = ad.forward(t["x"], t["base"], offsets, index, out=torch.empty_like(t["base"]), keep=True)
        got = [y, *ad.backward(t["dy"], t["dbase"], dx=torch.empty_like(t["dbase"])).values()]
        assert seen is None or all(torch.equal(a, b) for a, b in zip(got, seen))
        seen = [v.clone() for v in got]


def test_streams_graphs_and_runs_that_change_between_replays():
    t = _make(64, 128, 96, 8, 3, torch.bfloat16, seed=22)
    offsets, index, runs = _runs([30, 34], [0, 2])
    ad, side = lm.Adapters(t["a"], t["b"], t["scale"]), torch.cuda.Stream()
    out, dx = torch.empty_like(t["base"]), torch.empty_like(t["dbase"])
    want = ad.forward(t["x"], t["base"], offsets, index, out=torch.empty_like(out)).clone()
    side.wait_stream(torch.cuda.current_stream())
    ad.forward(t["x"], t["base"], offsets, index, out=out, keep=True, stream=side)
    ad.backward(t["dy"], t["dbase"], dx=dx, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graphs = []
    for _ in range(2):   # two captured training steps, whose scratch is their own
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            y = ad.forward(t["x"], t["base"], offsets, index, out=torch.empty_like(out), keep=True)
            g = ad.backward(t["dy"], t["dbase"], dx=torch.empty_like(dx))
        graphs[-1].result = (y, g)
    for lengths, ids in (([30, 34], [0, 2]), ([1, 63], [2, 1]), ([64, 0], [-1, 0])):
        o, i, runs = _runs(lengths, ids)
        offsets.copy_(o)
        index.copy_(i)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for graph in graphs:
            _check(t, runs, torch.bfloat16, *graph.result)


def test_beside_a_linear8_layer():
    """A frozen 8-bit layer and its adapters: the sum of what each gives alone, and their gradients of x."""
    t = _make(100, 96, 64, 8, 2, torch.bfloat16, seed=24)
    layer = lm.Linear8(96, 64, weight=torch.randn(64, 96, device="cuda") * 0.1)
    offsets, index, runs = _runs([60, 40], [1, 0])
    ad = lm.Adapters(t["a"], t["b"], t["scale"])
    t["base"] = layer.forward(t["x"], keep=True).clone()
    y = ad.forward(t["x"], layer.forward(t["x"], keep=True), offsets, index, keep=True)
    t["dbase"] = layer.backward(t["dy"], need_dw=False)["dx"].clone()
    grads = ad.backward(t["dy"], layer.backward(t["dy"], need_dw=False)["dx"])
    _check(t, runs, torch.bfloat16, y, grads)
    layer.check()


def test_refusals():
    t = _make(10, 16, 8, 4, 2, torch.float32, seed=26)
    ad = lm.Adapters(t["a"], t["b"], t["scale"])
    offsets, index, _ = _runs([10], [0])
    for bad in (lambda: ad.forward(t["x"].half(), t["base"]), lambda: ad.forward(t["x"][:9], t["base"]), lambda: ad.forward(t["x"][:, :15], t["base"]),
                lambda: ad.forward(t["x"], t["base"].T), lambda: ad.forward(t["x"], t["base"], offsets), lambda: ad.forward(t["x"], t["base"], offsets, index.long()),
                lambda: ad.forward(t["x"], t["base"], offsets[:1], index), lambda: ad.forward(t["x"].cpu(), t["base"].cpu()),
                lambda: lm.Adapters(t["a"], t["b"].half()), lambda: lm.Adapters(t["a"], t["b"][:1]), lambda: lm.Adapters(t["a"], t["b"], t["scale"][:1]),
                lambda: lm.Adapters(t["a"][0], t["b"][0]), lambda: lm.Adapters(torch.zeros(1, 129, 8, device="cuda"), torch.zeros(1, 129, 8, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        ad.backward(t["dy"])
    ad.forward(t["x"], t["base"], out=torch.empty_like(t["base"]), keep=True)
    for bad in (lambda: ad.backward(t["dy"][:9]), lambda: ad.backward(t["dy"], dx=t["dbase"]), lambda: ad.backward(t["dy"], grad_dtype=torch.float16),
                lambda: ad.backward(t["dy"], da=torch.zeros(2, 4, 15, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):   # rows that overlap
        ad.forward(t["x"], t["base"], out=t["base"][:1].expand(10, 8))
