"""Long runs of adapters with 16-bit rows that begin on 16 bytes (products on the tensor cores' own memory) against the formulas in 64 bits.

Tolerances by element, as in the other tests of the adapters, but for h's sums: a tile's columns of x go to four accumulators in turn (two above
64 ranks), 16 columns an instruction, so at most I / 64 (I / 32) sums follow one another in one, then the accumulators' and the CTAs' (at most 12), each off by
2^-23 of what it holds (the tensor core cuts off): e_h = (40 + I / 32) 2^-23 H.
"""
import math

import pytest
import torch

from paper_2407_12637_b200 import lbt, lm

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
PART = {torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -20}   # what two 16-bit parts leave of h
TYPES = list(HALF_ULP)


def _make(M, I, O, r, n, dtype, seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    rows = lambda w: randn(M, w + pad).to(dtype)[:, :w]  # noqa: E731
    return {"x": rows(I), "base": rows(O), "a": (randn(n, r, I) * I ** -0.5).to(dtype), "b": (randn(n, r, O) * r ** -0.5).to(dtype),
            "scale": 0.5 + torch.rand(n, generator=g, device="cuda")}


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _check(t, cuts, ids, y, h=None):
    n, rank, I = t["a"].shape
    dtype = t["x"].dtype
    for lo, hi, i in zip(cuts, cuts[1:], ids):
        if i < 0 or i >= n:
            assert torch.equal(y[lo:hi], t["base"][lo:hi])
            continue
        x, a, b, s = t["x"][lo:hi].double(), t["a"][i].double(), t["b"][i].double(), t["scale"][i].double()
        want_h, eh = x @ a.T, (x.abs() @ a.abs().T) * (40 + I / 32) * 2.0 ** -23
        out = t["base"][lo:hi].double() + s * (want_h @ b)
        tol = s * ((eh + want_h.abs() * (PART[dtype] + (rank / 4 + 8) * 2.0 ** -23)) @ b.abs()) + 1.01 * HALF_ULP[dtype] * out.abs() + 2.0 ** -23 * t["base"][lo:hi].double().abs()
        if dtype == torch.float16:
            tol = tol + 2.0 ** -25
        assert ((y[lo:hi].double() - out).abs() <= tol).all(), float(((y[lo:hi].double() - out).abs() / tol).max())
        if h is not None:
            assert ((h[lo:hi].double() - want_h).abs() <= eh + 1e-30).all(), float(((h[lo:hi].double() - want_h).abs() / eh).max())


def _forward(t, cuts=None, ids=None, out=None, adapters=None):
    ad = adapters or lm.Adapters(t["a"], t["b"], t["scale"])
    out = torch.full_like(t["base"], 7.0) if out is None else out
    runs = () if cuts is None else (_i32(cuts), _i32(ids))
    return ad, ad.forward(t["x"], t["base"], *runs, out=out, keep=True)


@pytest.mark.parametrize("M", [1300, 2060, 2600, 3500, 4500, 6000, 9000, 18001, 20000])
@pytest.mark.parametrize("I,O", [(200, 136), (8, 1000)])
@pytest.mark.parametrize("rank,dtype", [(16, torch.bfloat16), (64, torch.float16), (127, torch.bfloat16)])
def test_clusters_of_every_size(rank, dtype, I, O, M):
    """From eight CTAs a tile to one and to more tiles than the device holds; CTAs that have no column of x."""
    t = _make(M, I, O, rank, 1, dtype, seed=M)
    ad, y = _forward(t)
    _check(t, [0, M], [0], y, ad.kept[1])
    ad.check()


@pytest.mark.parametrize("rank", [1, 8, 15, 17, 33, 48, 65, 80, 128])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_ranks_and_runs(dtype, rank):
    """Runs that end anywhere in a tile, one without an adapter, rows ahead of the first run and behind the last one, wider matrices."""
    cuts, ids = [3, 700, 701, 701, 1213, 2000, 2513, 4100], [2, 0, 1, -1, 1, 0, 3]
    t = _make(4200, 264, 392, rank, 3, dtype, seed=rank, pad=24)
    wide = torch.full((4200, 392 + 24), 7.0, device="cuda").to(dtype)
    ad, y = _forward(t, cuts, ids, out=wide[:, :392])
    _check(t, cuts, ids, y)
    assert (wide[:, 392:] == 7.0).all() and (wide[:3] == 7.0).all() and (wide[4100:] == 7.0).all()
    ad.check()


@pytest.mark.parametrize("rank", [64, 128])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_long_rows(dtype, rank):
    t = _make(600, 16384, 4104, rank, 1, dtype, seed=5)
    _, y = _forward(t)
    _check(t, [0, 600], [0], y)


@pytest.mark.parametrize("rank", [20, 100])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_what_is_not_finite_stays_where_it_is(dtype, rank):
    """A tile's copies reach into the next run's rows and a weight's box ends at its rank: neither the neighbour's rows nor the next adapter's weights
    touch a run's outputs."""
    cuts, ids = [0, 1000, 2300], [0, 1]
    t = _make(2300, 136, 200, rank, 3, dtype, seed=9)
    _, want = _forward(t, cuts, ids)
    want = want.clone()
    t["x"][1000:], t["base"][1000:] = math.nan, math.inf
    t["a"][1], t["b"][1], t["a"][2], t["b"][2] = math.nan, math.inf, math.inf, math.nan
    t["x"][17, 3], t["x"][140, 0], t["x"][999, 135] = math.inf, -math.inf, math.nan
    _, y = _forward(t, cuts, ids)
    bad = [17, 140, 999]
    rest = [m for m in range(1000) if m not in bad]
    assert torch.equal(y[rest], want[rest]) and not torch.isfinite(y[bad]).any() and not torch.isfinite(y[1000:]).any()


def test_h_beyond_the_range_of_fp16():
    for size in (3e4, 1e-4):
        t = _make(1500, 64, 48, 16, 1, torch.float16, seed=14)
        t["x"].mul_(size / 100)
        t["a"].mul_(100.0 if size > 1 else 0.01)
        t["b"].mul_(1e-6 / size if size > 1 else 1.0)
        _, y = _forward(t)
        _check(t, [0, 1500], [0], y)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_in_place_captured_and_on_two_streams(dtype):
    """The same bits whichever way it runs."""
    t = _make(2500, 520, 264, 32, 2, dtype, seed=20)
    cuts, ids = [0, 1300, 2500], [1, 0]
    ad, want = _forward(t, cuts, ids)
    runs = (_i32(cuts), _i32(ids))
    base = t["base"].clone()
    assert torch.equal(ad.forward(t["x"], base, *runs), want)
    outs = [torch.empty_like(want) for _ in range(3)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, out in zip(streams, outs):
        with torch.cuda.stream(s):
            for _ in range(4):
                ad.forward(t["x"], t["base"], *runs, out=out)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ad.forward(t["x"], t["base"], *runs, out=outs[2])
    for _ in range(2):
        outs[2].zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for out in outs)
    ad.check()


@pytest.mark.parametrize("rank", [16, 72])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_weight_gradients_alone(dtype, rank):
    """Without dx the second product is left out: dA keeps its bits."""
    t = _make(2500, 264, 136, rank, 2, dtype, seed=22)
    g = torch.Generator(device="cuda").manual_seed(23)
    dy, dbase = (torch.randn(2500, w, generator=g, device="cuda").to(dtype) for w in (136, 264))
    ad, _ = _forward(t, [0, 1100, 1300, 2500], [1, -1, 0])
    all_of_them = ad.backward(dy, dbase, dx=torch.empty_like(dbase))
    alone = ad.backward(dy)
    assert set(alone) == {"da", "db"} and torch.equal(alone["da"], all_of_them["da"]) and torch.equal(alone["db"], all_of_them["db"])
    back = lm.Adapters(t["b"], t["a"], t["scale"])   # dx is the operator with A and B exchanged
    assert torch.equal(back.forward(dy, dbase, _i32([0, 1100, 1300, 2500]), _i32([1, -1, 0]), out=torch.empty_like(dbase)), all_of_them["dx"])
    ad.check()


@pytest.mark.parametrize("M,rank,mute", [(300, 16, 0), (300, 64, 7), (2500, 128, 2), (20000, 40, 0)])
def test_a_lost_signal_stores_nothing(M, rank, mute):
    """One CTA of each cluster that waits in vain: an error code, no output from any CTA of the cluster, and a usable context."""
    t = _make(M, 520, 1032, rank, 1, torch.bfloat16, seed=3)
    ad, want = _forward(t)
    out = torch.full_like(t["base"], 7.0)
    desc = lbt.AdaptersDesc(M=M, I=520, O=1032, runs=0, adapters=1, rank=rank, type=lbt.BF16)
    lbt.selftest_adapters_timeout(desc, t["x"], t["a"], t["b"], t["base"], out, mute, ad.status, 2000)
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    with pytest.raises(lbt.LbtError) as e:
        ad.check()
    assert e.value.status == lbt.ERR_TIMEOUT
    assert torch.equal(_forward(t, adapters=ad)[1], want)
    ad.check()   # (said once)


def test_a_self_test_without_such_rows_is_refused():
    t = _make(8, 60, 64, 8, 1, torch.bfloat16)
    desc = lbt.AdaptersDesc(M=8, I=60, O=64, runs=0, adapters=1, rank=8, type=lbt.BF16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for mute, limit in ((0, 1000), (8, 1000), (0, 0)):   # rows of 120 bytes; no such CTA; no limit
        with pytest.raises(lbt.LbtError):
            lbt.selftest_adapters_timeout(desc, t["x"], t["a"], t["b"], t["base"], t["base"], mute, status, limit)
    assert int(status) == 0
