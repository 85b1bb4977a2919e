"""Norm, gate, residual and norm in one pass, against the formula in 64 bits and against differences of it.

Tolerances.  fp32 arithmetic on rows of D values: a row's sums carry a relative error of a few 2^-24 sqrt(D) (pairwise over
threads), every output a dozen roundings: 2^-24 (16 + sqrt(D)) of the magnitudes that enter it, plus one rounding to its
type.  Magnitudes that enter: what the formula gives with every term's absolute value, bounded here by the row's (or the
column's) largest term.  A sum over M rows adds 2^-24 sqrt(M) per term in magnitude; types of 16 bits round once at the end.
"""
import ctypes as C
import math

import pytest
import torch

from guard import Guard
from paper_2407_12637_b200 import lbt, lm

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _formula(c, x, h, gate, w1, b1, w2, b2):
    """r, y in 64 bits (autograd tensors)."""
    def norm(v, w, b):
        mu = v.mean(1, keepdim=True) if c["kind"] == "layer" else 0.0
        y = (v - mu) / torch.sqrt(((v - mu) ** 2).mean(1, keepdim=True) + 1e-6)
        y = y * w if w is not None else y
        return y + b if b is not None else y
    u = norm(h, w1, b1) if c["post"] else h
    if gate is not None:
        rows = torch.arange(x.shape[0], device=x.device) // (c["rpg"] or x.shape[0])
        u = gate.reshape(-1, x.shape[1])[rows] * u
    r = c["sx"] * x + c["sh"] * u
    return r, norm(r, w2, b2)


def _case(M, D, dtype, pdtype, kind, gate, rpg, seed, post=True, params=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    rows = {"none": 0, "one": 1, "rows": -(-M // rpg) if rpg else 1}[gate]
    vec = lambda on, centre: (centre + 0.2 * rand(D)).to(pdtype) if on else None  # noqa: E731
    layer = kind == "layer"
    t = {"x": (2 * rand(M, D) + 0.3).to(dtype), "h": (0.7 * rand(M, D) - 0.2).to(dtype), "gate": (0.5 * rand(rows, D)).to(pdtype) if rows else None,
         "w1": vec(params and post, 1.0), "b1": vec(params and layer and post, 0.0), "w2": vec(params, 1.0), "b2": vec(params and layer, 0.0)}
    c = {"kind": kind, "post": post, "rpg": rpg, "sx": 0.9, "sh": 0.6}
    norm = lm.ResNorm(D, kind, t["w1"], t["b1"], t["w2"], t["b2"], eps=1e-6, scale_x=0.9, scale_h=0.6, post_norm=post)
    return c, t, norm, (rand(M, D) * 0.1).to(dtype), (rand(M, D) * 0.1).to(dtype)


def _near(got, ref, size, terms, name):
    """|got - ref| within (16 + sqrt(terms)) 2^-24 of `size` (the largest term that enters) and half an ulp of the type."""
    d = (got.double() - ref).abs()
    tol = (16 + math.sqrt(terms)) * 2.0 ** -24 * size + 1.01 * HALF_ULP[got.dtype] * ref.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 0)
    worst = float((d / tol).max()) if d.numel() else 0.0
    assert worst <= 1.0, (name, worst)


CASES = [(1, 1, "rms", "none", 0), (1, 4096, "rms", "one", 0), (3, 7, "layer", "one", 0), (5, 255, "rms", "rows", 2), (33, 256, "layer", "rows", 33),
         (64, 257, "rms", "rows", 1), (40, 512, "layer", "none", 0), (19, 1000, "rms", "one", 0), (700, 1024, "layer", "rows", 100),
         (350, 1111, "layer", "one", 0), (1200, 96, "rms", "rows", 7), (600, 2048, "rms", "rows", 250), (9, 2050, "layer", "rows", 4),
         (310, 4096, "layer", "rows", 150), (7, 4100, "rms", "one", 0), (300, 8192, "rms", "rows", 200), (5, 8200, "layer", "rows", 2),
         (4, 16384, "rms", "one", 0), (3, 20001, "layer", "one", 0), (2, 32768, "rms", "rows", 1), (5000, 320, "layer", "rows", 1)]


@pytest.mark.parametrize("M,D,kind,gate,rpg", CASES)
@pytest.mark.parametrize("dtype,pdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)], ids=str)
def test_forward_and_backward(M, D, kind, gate, rpg, dtype, pdtype):
    c, t, norm, dr, dy = _case(M, D, dtype, pdtype, kind, gate, rpg, M + D)
    guard = Guard()
    r, y = guard.alloc((M, D), dtype), guard.alloc((M, D), dtype)
    norm.forward(t["x"], t["h"], t["gate"], rpg, out=(r, y), keep=True)
    out = norm.backward(dr, dy)
    guard.check()
    wide = {k: v.double().requires_grad_() if v is not None else None for k, v in t.items()}
    r64, y64 = _formula(c, *(wide[k] for k in ("x", "h", "gate", "w1", "b1", "w2", "b2")))
    big = lambda v: v.abs().amax(1, keepdim=True).detach() + 1e-6  # noqa: E731  (a row's largest magnitude)
    # a row of one value (or of nearly equal ones) is divided by its tiny deviation: errors of v grow by |v| / deviation
    def stretch(v):
        dev = torch.sqrt(((v - (v.mean(1, keepdim=True) if kind == "layer" else 0)) ** 2).mean(1, keepdim=True) + 1e-6).detach()
        return dev, big(v) / dev
    dev1, s1 = stretch(wide["h"])
    dev2, s2 = stretch(r64)
    size_u = (s1 if c["post"] else big(wide["h"])) * 1.6 + 1
    size_r = big(wide["x"]) + size_u * (wide["gate"].abs().max().item() if gate != "none" else 1)
    _near(r, r64.detach(), size_r, D, "r")
    _near(y, y64.detach(), (size_r / dev2) * 1.6 * (1 + s2) + 1, D, "y")
    (r64 * dr.double()).sum().add((y64 * dy.double()).sum()).backward()
    size_d = big(dr) + 1.6 * big(dy) / dev2 * (2 + s2) * (1 + size_r / dev2)
    _near(out["dx"], wide["x"].grad, size_d, D, "dx")
    gmax = wide["gate"].abs().max().item() if gate != "none" else 1.0
    size_du = size_d * gmax
    _near(out["dh"], wide["h"].grad, 1.6 * size_du / dev1 * (2 + s1) * (1 + s1) if c["post"] else size_du, D, "dh")
    col = lambda s: s.amax() * M  # noqa: E731  (M terms, each at most the largest row's)
    for name, key, size in (("dw_post", "w1", size_du * (1 + s1)), ("db_post", "b1", size_du), ("dw_pre", "w2", big(dy) * (1 + s2) * (1 + size_r / dev2)),
                            ("db_pre", "b2", big(dy)), ("dgate", "gate", size_d * size_u)):
        if wide[key] is not None:
            _near(out[name], wide[key].grad, col(size) / math.sqrt(M), max(D, M), name)
        else:
            assert name not in out


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_against_differences(kind):
    """Central differences of the 64-bit formula along random directions of every input."""
    M, D = 24, 96
    c, t, norm, dr, dy = _case(M, D, torch.float32, torch.float32, kind, "rows", 5, 3)
    norm.forward(t["x"], t["h"], t["gate"], 5, keep=True)
    out = norm.backward(dr, dy)
    keys = ("x", "h", "gate", "w1", "b1", "w2", "b2")
    names = dict(zip(keys, ("dx", "dh", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")))
    g = torch.Generator(device="cuda").manual_seed(8)

    def loss(v):
        r, y = _formula(c, *(v[k] for k in keys))
        return float((r * dr.double()).sum() + (y * dy.double()).sum())

    for k in keys:
        if t[k] is None:
            continue
        for _ in range(3):
            way = torch.randn(t[k].shape, generator=g, device="cuda", dtype=torch.float64)
            v = {n: (a.double() if a is not None else None) for n, a in t.items()}
            e = 1e-5
            up = loss({**v, k: v[k] + e * way})
            down = loss({**v, k: v[k] - e * way})
            got = float((out[names[k]].double() * way).sum())
            room = 1e-5 * float(out[names[k]].double().norm() * way.norm()) + 1e-6   # fp32 gradients, differences good to 1e-8
            assert abs(got - (up - down) / (2 * e)) <= room, k


@pytest.mark.parametrize("dr_on,dy_on,post,gate", [(True, False, True, "one"), (False, True, True, "rows"), (True, True, False, "rows"), (False, True, False, "none")])
def test_parts_left_out(dr_on, dy_on, post, gate):
    """One incoming gradient only, no norm on h, no gate, no parameters."""
    M, D = 50, 200
    c, t, norm, dr, dy = _case(M, D, torch.float32, torch.float32, "rms", gate, 7 if gate == "rows" else 0, 5, post=post, params=False)
    norm.forward(t["x"], t["h"], t["gate"], c["rpg"], keep=True)
    out = norm.backward(dr if dr_on else None, dy if dy_on else None)
    assert set(out) == {"dx", "dh"} | ({"dgate"} if gate != "none" else set())
    wide = {k: v.double().requires_grad_() if v is not None else None for k, v in t.items()}
    r, y = _formula(c, *(wide[k] for k in ("x", "h", "gate", "w1", "b1", "w2", "b2")))
    ((r * dr.double()).sum() * dr_on + (y * dy.double()).sum() * dy_on).backward()
    for name, k in (("dx", "x"), ("dh", "h"), ("dgate", "gate")):
        if wide[k] is not None:
            ref = wide[k].grad
            assert (out[name].double() - ref).abs().max() <= 1e-5 * ref.abs().max()


@pytest.mark.parametrize("M,D", [(1, 4096), (5, 1000), (130, 300), (9, 5000), (2, 1)])
def test_codes_are_the_rows_of_y(M, D):
    """The codes are those of the fp32 y; padding columns are zero; r is the same as without codes."""
    c, t, norm, _, _ = _case(M, D, torch.float32, torch.float32, "layer", "one", 0, 6)
    r, y = norm.forward(t["x"], t["h"], t["gate"])
    r2, q, scale = norm.forward_codes(t["x"], t["h"], t["gate"])
    want_q, want_s = torch.empty_like(q), torch.empty_like(scale)
    lbt.rows8_quantize(y, want_q, want_s)
    assert torch.equal(r, r2) and torch.equal(q, want_q) and torch.equal(scale, want_s) and not q[:, D:].any()


def test_in_place_strides_and_another_stream():
    """Rows of wider tensors at odd offsets, on a side stream: sums are taken in another order there, so a 16-bit result may fall to
    the other side of a rounding (one ulp, 2^-7).  r written over x and y over h: the same bits as out of place."""
    c, t, norm, dr, dy = _case(37, 600, torch.bfloat16, torch.bfloat16, "rms", "rows", 10, 7)
    r, y = norm.forward(t["x"], t["h"], t["gate"], 10, keep=True)
    want = norm.backward(dr, dy)
    wide = lambda v, off: torch.full((37, 640), 3.0, dtype=v.dtype, device="cuda")[:, off:off + 600].copy_(v)  # noqa: E731
    x2, h2, dr2, dy2 = wide(t["x"], 1), wide(t["h"], 8), wide(dr, 16), wide(dy, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r2, y2 = norm.forward(x2, h2, t["gate"], 10, keep=True, stream=side)
    got = norm.backward(dr2, dy2, stream=side)
    side.synchronize()
    for a, b in ((r2, r), (y2, y), *((got[k], want[k]) for k in want)):
        assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-5 * b.float().abs().max()).all()
    norm.forward(x2, h2, t["gate"], 10, out=(x2, h2))
    assert torch.equal(x2, r2) and torch.equal(h2, y2) and (x2._base[:, 601:] == 3).all() and (x2._base[:, :1] == 3).all()
    x3, h3 = t["x"].clone(), t["h"].clone()
    norm.forward(x3, h3, t["gate"], 10, out=(x3, h3))
    assert torch.equal(x3, r) and torch.equal(h3, y)


def test_non_finite_rows_stay_alone():
    c, t, norm, dr, dy = _case(20, 300, torch.float32, torch.float32, "rms", "one", 0, 8)
    t["x"][3, 7] = float("nan")
    t["h"][5, 0] = float("inf")
    r, y = norm.forward(t["x"], t["h"], t["gate"], keep=True)
    out = norm.backward(dr, dy)
    clean = [i for i in range(20) if i not in (3, 5)]
    for v in (y, out["dx"], out["dh"]):
        assert torch.isfinite(v[clean]).all() and v[5].isnan().any()
    assert y[3].isnan().all() and torch.isfinite(r[3]).sum() == 299
    r2, q, scale = norm.forward_codes(t["x"], t["h"], t["gate"])
    assert scale[3].isnan() and not q[3].any() and torch.isfinite(scale[clean]).all()


def test_repeats_bit_for_bit():
    c, t, norm, dr, dy = _case(900, 384, torch.bfloat16, torch.float32, "layer", "rows", 64, 9)
    norm.forward(t["x"], t["h"], t["gate"], 64, keep=True)
    first = norm.backward(dr, dy)
    for _ in range(3):
        again = norm.backward(dr, dy)
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_zero_rows_and_refusals():
    norm = lm.ResNorm(64, w_post=torch.ones(64, device="cuda"), w_pre=torch.ones(64, device="cuda"))
    x = torch.empty(0, 64, device="cuda")
    r, y = norm.forward(x, x, keep=True)
    out = norm.backward(x, x)
    assert r.shape == (0, 64) and not out["dw_pre"].any() and not out["dw_post"].any()
    x = torch.randn(4, 64, device="cuda")
    for bad in ((x[:, :63], x[:, :63]), (x, x[:3]), (x, x.half()), (x.double(), x.double())):
        with pytest.raises((ValueError, KeyError)):
            norm.forward(*bad)
    with pytest.raises(ValueError):
        norm.forward(x, x, torch.ones(3, 64, device="cuda"), 2)
    with pytest.raises(ValueError):
        norm.forward(x, x, torch.ones(1, 64, device="cuda").half())
    with pytest.raises(ValueError):
        lm.ResNorm(64, "rms", b_pre=torch.ones(64, device="cuda"))
    with pytest.raises(ValueError):
        lm.ResNorm(64, "batch")
    with pytest.raises(RuntimeError):
        lm.ResNorm(64).backward(x, x)
    wide = torch.empty(1, 40000, device="cuda")
    with pytest.raises(lbt.LbtError) as e:
        lm.ResNorm(40000).forward(wide, wide)
    assert e.value.status == lbt.ERR_UNSUPPORTED


@pytest.mark.parametrize("D", [1, 100, 128, 300, 1111, 4096, 8200, 20001])
def test_codes_in_a_wider_matrix(D):
    M, pitch = 4, lbt.pitch8(D)
    ldq = pitch + 48
    c, t, norm, _, _ = _case(M, D, torch.float32, torch.float32, "rms", "one", 0, 6)
    r, want, want_s = norm.forward_codes(t["x"], t["h"], t["gate"])
    q, s = torch.full((M, ldq), 77, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    d = lbt.ResnormDesc(M, D, 0, lbt.F32, lbt.F32, lbt.NORM_RMS, 1, 1e-6, 1e-6, 0.9, 0.6)
    at = lambda v: v.data_ptr()  # noqa: E731
    assert lbt.lib().lbt_resnorm_forward(C.addressof(d), at(t["x"]), at(t["h"]), at(t["gate"]), at(t["w1"]), None, at(t["w2"]), None, at(r), None,
                                         at(q), ldq, at(s), None, None) == lbt.OK
    torch.cuda.synchronize()
    assert torch.equal(q[:, :pitch], want) and torch.equal(s, want_s) and (q[:, pitch:] == 77).all()


def test_gradient_of_a_gate_without_rows():
    """No tokens and one gate row for all of them: its gradient is zero, as the parameters' are."""
    x = torch.empty(0, 64, device="cuda")
    for kind in ("rms", "layer"):
        norm = lm.ResNorm(64, kind, w_post=torch.ones(64, device="cuda"), w_pre=torch.ones(64, device="cuda"))
        for gate in (torch.ones(64, device="cuda"), torch.ones(1, 64, device="cuda")):
            norm.forward(x, x, gate, keep=True)
            out = norm.backward(x, x, out={"dgate": torch.full_like(gate, 5.0)})
            assert not out["dgate"].any() and not out["dw_pre"].any()
        none = torch.empty(0, 64, device="cuda")   # (no rows, no gate rows)
        norm.forward(x, x, none, 3, keep=True)
        assert norm.backward(x, x)["dgate"].shape == (0, 64)


@pytest.mark.parametrize("dtype,pdtype", [(torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float32, torch.bfloat16), (torch.float32, torch.float16)], ids=str)
@pytest.mark.parametrize("M,D,kind,gate,rpg,post", [(70, 256, "rms", "one", 0, True), (300, 1111, "layer", "rows", 40, True), (64, 4096, "rms", "none", 0, False),
                                                     (40, 2048, "layer", "rows", 7, False), (9, 8192, "rms", "rows", 3, True), (500, 512, "layer", "one", 0, True)])
def test_types(M, D, kind, gate, rpg, post, dtype, pdtype):
    """Whole tensors in the Euclidean norm: every element carries a relative error of a rounding to its type (2^-8, 2^-11, 2^-24 at most) and of
    fp32 arithmetic (about 2^-24 sqrt(D) of the largest terms, well below 2^-15 of the tensor's norm)."""
    c, t, norm, dr, dy = _case(M, D, dtype, pdtype, kind, gate, rpg, M + D, post=post)
    r, y = norm.forward(t["x"], t["h"], t["gate"], rpg, keep=True)
    out = norm.backward(dr, dy)
    wide = {k: v.double().requires_grad_() if v is not None else None for k, v in t.items()}
    r64, y64 = _formula(c, *(wide[k] for k in ("x", "h", "gate", "w1", "b1", "w2", "b2")))
    (r64 * dr.double()).sum().add((y64 * dy.double()).sum()).backward()
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
    for got, ref in ((r, r64.detach()), (y, y64.detach()), (out["dx"], wide["x"].grad), (out["dh"], wide["h"].grad)):
        assert (got.double() - ref).norm() <= (half[dtype] + 2.0 ** -15) * ref.norm()
    for name, key in (("dw_post", "w1"), ("db_post", "b1"), ("dw_pre", "w2"), ("db_pre", "b2"), ("dgate", "gate")):
        if wide[key] is not None:
            ref = wide[key].grad
            assert (out[name].double() - ref).norm() <= (half[pdtype] + 2.0 ** -15) * ref.norm(), name
        else:
            assert name not in out


def test_the_binding_gives_the_norms_bits():
    M, D = 70, 256
    c, t, norm, dr, dy = _case(M, D, torch.bfloat16, torch.bfloat16, "rms", "rows", 30, 15)
    r, y = norm.forward(t["x"], t["h"], t["gate"], 30, keep=True)
    want = norm.backward(dr, dy)
    d = lbt.ResnormDesc(M, D, 30, lbt.BF16, lbt.BF16, lbt.NORM_RMS, 1, 1e-6, 1e-6, 0.9, 0.6)
    r2, y2, stats = torch.empty_like(r), torch.empty_like(y), torch.empty(M, 4, device="cuda")
    lbt.resnorm_forward(d, t["x"], t["h"], t["gate"], t["w1"], None, t["w2"], None, r2, y2, stats=stats)
    dx, dh, dgate, dw1, dw2 = (torch.empty_like(v) for v in (r, r, t["gate"], t["w1"], t["w2"]))
    lbt.resnorm_backward(d, dr, dy, t["x"], t["h"], t["gate"], t["w1"], None, t["w2"], stats, dx, dh, dgate=dgate, dw_post=dw1, dw_pre=dw2)
    for a, b in ((r2, r), (y2, y), (dx, want["dx"]), (dh, want["dh"]), (dgate, want["dgate"]), (dw1, want["dw_post"]), (dw2, want["dw_pre"])):
        assert torch.equal(a, b)
