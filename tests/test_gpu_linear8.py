"""The 8-bit linear layer against its definition: codes bit for bit, products from exact integer sums in 64 bits.

Tolerances.  y = fl(fl(acc) fl(s_x s_w)) + b: three roundings of the product and one of the sum, each within 2^-24 of its
magnitude, then one rounding to the output's type (2^-24, 2^-8, 2^-11; fp16 also 2^-25 absolute below its normal range).
"""
import threading

import numpy as np
import pytest
import torch

from guard import Guard
from paper_2407_12637_b200 import lbt, lm

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _rows8(t):
    """Codes (float64) and scales (fp32) of the rows of an fp32 CPU tensor, by the definition; a bad row has NaN as its scale."""
    most = t.abs().amax(1, keepdim=True) if t.shape[1] else torch.zeros(t.shape[0], 1)
    good = torch.isfinite(t).all(1, keepdim=True)
    live = good & (most > 1e-36)
    factor = torch.where(live, torch.reciprocal(most) * 127.0, 0.0)
    q = torch.where(live, torch.round(torch.nan_to_num(t, 0.0, 0.0, 0.0) * factor), 0.0)
    scale = torch.where(good, torch.where(live, most * (torch.ones(1) / 127.0), 0.0), float("nan"))
    return q.double(), scale.reshape(-1)


def _close(got, acc, scale, bias, name=""):
    """got against acc * scale (+ bias), acc exact, scale [rows, cols] in 64 bits."""
    part = acc * scale
    ref = part + (bias.double() if bias is not None else 0.0)
    tol = 4 * 2.0 ** -24 * (part.abs() + (bias.double().abs() if bias is not None else 0.0)) + 1.01 * HALF_ULP[got.dtype] * ref.abs() + 2.0 ** -25
    if got.dtype != torch.float16:
        tol = tol - 2.0 ** -25 + 1e-37
    d = (got.double().cpu() - ref).abs()
    assert torch.equal(torch.isnan(got.cpu()), torch.isnan(ref)), name
    bad = d > tol
    assert not bad.any(), (name, int(bad.sum()), float(d[bad].max()))


def _make(M, I, O, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, I, generator=g) * std
    x[:, ::17] *= 20
    return x.to(dtype), torch.randn(O, I, generator=g) * 0.05, torch.randn(O, generator=g), torch.randn(M, O, generator=g).pow(3).to(dtype)


SHAPES = [(1, 1, 1), (1, 4096, 256), (2, 100, 17), (3, 16, 33), (8, 129, 130), (16, 2048, 384), (17, 1000, 257), (33, 128, 1024), (64, 515, 129),
          (100, 4096, 128), (128, 2000, 640), (129, 127, 128), (130, 640, 384), (300, 1111, 1000), (511, 513, 77), (1000, 64, 2047), (640, 8192, 96)]


@pytest.mark.parametrize("M,I,O", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
def test_forward_and_backward(M, I, O, dtype):
    x, w, b, dy = _make(M, I, O, dtype, M * 7 + I)
    guard = Guard()
    lin = lm.Linear8(I, O, bias=b.cuda())
    lin.load_weight(w.cuda())
    q_w, s_w = _rows8(w)
    assert torch.equal(lin.q_w.cpu()[:, :I].double(), q_w) and torch.equal(lin.s_w.cpu(), s_w)
    assert not lin.q_w[:, I:].any()
    q_x, s_x = _rows8(x.float())
    y = guard.alloc((M, O), dtype)
    lin.forward(x.cuda(), out=y, keep=True)
    assert torch.equal(lin.kept[0].cpu()[:, :I].double(), q_x) and torch.equal(lin.kept[1].cpu(), s_x)
    _close(y, q_x @ q_w.T, s_x.double()[:, None] * s_w.double(), b, "y")

    dx, dw, db = guard.alloc((M, I), dtype), guard.alloc((O, I), torch.float32), guard.alloc((O,), torch.float32)
    out = lin.backward(dy.cuda(), dx=dx, dw=dw, dbias=db)
    assert out["dx"] is dx and out["dw"] is dw and out["dbias"] is db
    q_r, s_r = _rows8(dy.float() * s_w)
    q_c, s_c = _rows8((dy.float() * s_x[:, None]).T.contiguous())
    _close(dx, q_r @ q_w, s_r.double()[:, None], None, "dx")
    _close(dw, q_c @ q_x, s_c.double()[:, None], None, "dw")
    s = dy.double()
    # a sum of M fp32 values: at most M roundings of partial sums no larger than the sum of magnitudes
    assert ((db.double().cpu() - s.sum(0)).abs() <= M * 2.0 ** -24 * s.abs().sum(0) + 1e-37).all()
    assert int(lin.status) == 0
    guard.check()


@pytest.mark.parametrize("M,I,O", [(2304, 384, 2304), (4096, 2176, 1280), (2500, 130, 2100)])
def test_many_tiles(M, I, O):
    """More tiles than CTA pairs (several per pair), ragged at every edge."""
    x, w, b, dy = (t.cuda() for t in _make(M, I, O, torch.bfloat16, 5))
    lin = lm.Linear8(I, O, weight=w)
    y = lin.forward(x, keep=True)
    out = lin.backward(dy)
    q_x, s_x, q_w, s_w = lin.kept[0][:, :I].double(), lin.kept[1].double(), lin.q_w[:, :I].double(), lin.s_w.double()
    assert torch.equal(lin.q_w.cpu()[:, :I].double(), _rows8(w.cpu())[0])
    q_r, s_r = _rows8(dy.float().cpu() * lin.s_w.cpu())
    q_c, s_c = _rows8((dy.float().cpu() * lin.kept[1].cpu()[:, None]).T.contiguous())
    _close(y.cpu(), (q_x @ q_w.T).cpu(), (s_x[:, None] * s_w).cpu(), None, "y")
    _close(out["dx"].cpu(), (q_r.cuda() @ q_w).cpu(), s_r.double()[:, None], None, "dx")
    _close(out["dw"].cpu(), (q_c.cuda() @ q_x).cpu(), s_c.double()[:, None], None, "dw")
    assert "dbias" not in out


@pytest.mark.parametrize("M", [1, 5, 40, 300])
def test_strides_and_offsets(M):
    """Rows of wider tensors, starting at odd elements; the neighbours stay as they were."""
    I, O = 200, 150
    x, w, b, dy = _make(M, I, O, torch.bfloat16, 3)
    lin = lm.Linear8(I, O, bias=b.cuda(), weight=w.cuda())
    wide = lambda t, off: torch.full((t.shape[0], t.shape[1] + 21), 7.0, dtype=t.dtype, device="cuda")[:, off:off + t.shape[1]]  # noqa: E731
    xs, dys = wide(x, 3), wide(dy, 8)
    xs.copy_(x)
    dys.copy_(dy)
    y, dx, dw = wide(dy, 5), wide(x, 1), wide(w, 8)
    lin.forward(xs, out=y, keep=True)
    lin.backward(dys, dx=dx, dw=dw)
    other = lm.Linear8(I, O, bias=b.cuda(), weight=w.cuda())
    y2 = other.forward(x.cuda(), keep=True)
    want = other.backward(dy.cuda())
    assert torch.equal(y, y2) and torch.equal(dx, want["dx"]) and torch.equal(dw, want["dw"])
    for t in (y, dx, dw):
        base = t._base
        off = t.storage_offset()
        assert (base[:, :off] == 7).all() and (base[:, off + t.shape[1]:] == 7).all()


def test_rows_of_zeros_tiny_values_and_non_finite_values():
    M, I, O = 12, 96, 40
    x, w, _, dy = _make(M, I, O, torch.float32, 9)
    x[1] = 0
    x[2] = 1e-39
    x[3, 5] = float("inf")
    x[4, 95] = float("nan")
    x[5] = 3e38
    w[7] = 0
    q_x, s_x = _rows8(x)
    q_w, s_w = _rows8(w)
    lin = lm.Linear8(I, O, weight=w.cuda())
    y = lin.forward(x.cuda(), keep=True)
    assert torch.equal(lin.kept[0].cpu()[:, :I].double(), q_x) and torch.equal(lin.kept[1].cpu().isnan(), s_x.isnan())
    rows = [i for i in range(M) if i not in (3, 4, 5)]
    _close(y[rows], (q_x @ q_w.T)[rows], s_x.double()[rows, None] * s_w.double(), None)
    assert y[3:5].isnan().all() and not y[1:3].any()
    # a gradient row with an infinity: its dX row is NaN, every column of it is in dW
    lin = lm.Linear8(I, O, weight=w.cuda())
    lin.forward(torch.where(torch.isfinite(x), x, 0.0).clamp(-100, 100).cuda(), keep=True)
    dy[6, 3] = float("-inf")
    out = lin.backward(dy.cuda())
    assert out["dx"][6].isnan().all() and torch.isfinite(out["dx"][[i for i in range(M) if i != 6]]).all()
    assert out["dw"][3].isnan().all() and torch.isfinite(out["dw"][[i for i in range(O) if i != 3]]).all()


def test_zero_tokens_and_single_outputs():
    lin = lm.Linear8(64, 48, bias=torch.ones(48, device="cuda"), weight=torch.randn(48, 64, device="cuda"))
    x = torch.empty(0, 64, device="cuda")
    assert lin.forward(x, keep=True).shape == (0, 48)
    out = lin.backward(torch.empty(0, 48, device="cuda"))
    assert out["dx"].shape == (0, 64) and not out["dw"].any() and not out["dbias"].any()
    x = torch.randn(5, 64, device="cuda")
    lin.forward(x, keep=True)
    dy = torch.randn(5, 48, device="cuda")
    both = lin.backward(dy)
    assert torch.equal(lin.backward(dy, need_dw=False)["dx"], both["dx"]) and torch.equal(lin.backward(dy, need_dx=False)["dw"], both["dw"])
    assert set(lin.backward(dy, need_dw=False)) == {"dx"}


def test_gradient_against_differences():
    """x on its own grid: raising one code by one changes y by exactly s_x W[:, i]; dx is that difference against dy up to the
    gradient's rounding, half a step of s_r for each output channel."""
    M, I, O = 6, 64, 80
    g = torch.Generator().manual_seed(2)
    q = torch.randint(-100, 101, (M, I), generator=g).float()
    q[:, 0] = 127                        # keeps every row's scale
    step = 2.0 ** -5
    w = torch.randn(O, I, generator=g)
    dy = torch.randn(M, O, generator=g)
    lin = lm.Linear8(I, O, weight=w.cuda())
    y0 = lin.forward((q * step).cuda(), keep=True).double()
    dx = lin.backward(dy.cuda())["dx"].double().cpu()
    s_r = _rows8(dy * lin.s_w.cpu())[1].double()
    for i in (1, 7, 63):
        moved = q.clone()
        moved[:, i] += 1
        diff = ((lin.forward((moved * step).cuda()).double() - y0).cpu() * dy.double()).sum(1) / step
        room = 0.51 * s_r * lin.q_w[:, i].double().abs().sum().cpu() + 1e-3 * dy.double().abs().sum(1)
        assert ((dx[:, i] - diff).abs() <= room).all()


def test_another_stream_and_repeats():
    """Work on a side stream; the same call gives the same bits every time, whatever ran between."""
    x, w, b, dy = (t.cuda() for t in _make(70, 300, 200, torch.float16, 4))
    lin = lm.Linear8(300, 200, bias=b, weight=w)
    y0 = lin.forward(x, keep=True)
    g0 = lin.backward(dy)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        lin.forward(torch.randn_like(x), keep=False, stream=side)
        y = lin.forward(x, keep=True, stream=side)
        g = lin.backward(dy, stream=side)
        torch.empty(200, 320, dtype=torch.int8, device="cuda").fill_(99)   # memory that the default stream may be given
    side.synchronize()
    assert torch.equal(y, y0) and all(torch.equal(g[k], g0[k]) for k in g0)


def test_longest_reduction():
    """All codes 127 over the longest sum that is accepted: the accumulator ends 4 072 below 2^31."""
    I = lbt.MAX_REDUCTION8
    lin = lm.Linear8(I, 2, weight=torch.ones(2, I, device="cuda"))
    y = lin.forward(torch.ones(1, I, device="cuda"))
    assert (127 * 127 * I) < 2 ** 31 <= 127 * 127 * (I + 1)
    assert ((y.double() - I).abs() <= 6 * 2.0 ** -24 * I).all()


def test_refusals():
    lin = lm.Linear8(64, 48, weight=torch.randn(48, 64, device="cuda"))
    x = torch.randn(5, 64, device="cuda")
    for bad in (torch.randn(5, 63, device="cuda"), x.double(), x.cpu(), x.t(), torch.randn(64, device="cuda")):
        with pytest.raises((ValueError, IndexError)):
            lin.forward(bad)
    with pytest.raises(lbt.LbtError):   # rows that overlap
        lin.forward(torch.randn(1, 64, device="cuda").expand(5, 64))
    with pytest.raises(ValueError):
        lin.forward(x, out=torch.empty(5, 47, device="cuda"))
    with pytest.raises(ValueError):
        lin.forward(x, out=torch.empty(6, 48, device="cuda"))
    with pytest.raises(RuntimeError):
        lin.backward(torch.randn(5, 48, device="cuda"))
    lin.forward(x, keep=True)
    with pytest.raises(ValueError):
        lin.backward(torch.randn(6, 48, device="cuda"))
    with pytest.raises(ValueError):
        lin.load_weight(torch.randn(64, 48, device="cuda"))
    I = lbt.MAX_REDUCTION8 + 1
    long = lm.Linear8(I, 1)
    with pytest.raises(lbt.LbtError) as e:
        long.forward(torch.ones(1, I, device="cuda"))
    assert e.value.status == lbt.ERR_ACC_RANGE


def test_bias_gradient_alone():
    lin = lm.Linear8(64, 48, bias=torch.ones(48, device="cuda"), weight=torch.randn(48, 64, device="cuda"))
    bare = lm.Linear8(64, 48, weight=torch.randn(48, 64, device="cuda"))
    x, dy = torch.randn(70, 64, device="cuda"), torch.randn(70, 48, device="cuda")
    for layer in (lin, bare):
        layer.forward(x, keep=True)
        want = layer.backward(dy, dbias=torch.full((48,), 7.0, device="cuda"))["dbias"]
        assert ((want.double() - dy.double().sum(0)).abs() <= 70 * 2.0 ** -24 * dy.double().abs().sum(0)).all()
        for need_dx in (True, False):
            db = torch.full((48,), 7.0, device="cuda")
            out = layer.backward(dy, need_dx=need_dx, need_dw=False, dbias=db)
            assert out["dbias"] is db and torch.equal(db, want) and set(out) == {"dbias"} | ({"dx"} if need_dx else set())
    assert set(lin.backward(dy, need_dw=False)) == {"dx"} and set(bare.backward(dy)) == {"dx", "dw"}


def test_two_threads_on_one_stream():
    """Two threads that share a layer and the default stream, each with its own inputs: the bits that each gets alone."""
    lin = lm.Linear8(300, 200, weight=torch.randn(200, 300, device="cuda"))
    xs = [torch.randn(70, 300, device="cuda") * (i + 1) for i in range(2)]
    want = [lin.forward(x) for x in xs]
    got = [[], []]

    def work(i):
        for _ in range(300):
            got[i].append(lin.forward(xs[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(2) for y in got[i])


def test_a_refused_forward_pass_leaves_what_backward_reads():
    lin = lm.Linear8(64, 48, weight=torch.randn(48, 64, device="cuda"))
    x, dy = torch.randn(70, 64, device="cuda"), torch.randn(70, 48, device="cuda")
    lin.forward(x, keep=True)
    want, kept = lin.backward(dy), lin.kept
    wide = torch.randn(1, 64, device="cuda").expand(30, 64)   # rows that overlap
    with pytest.raises(lbt.LbtError):
        lin.forward(wide, keep=True)
    assert lin.kept is kept
    out = lin.backward(dy)
    assert all(torch.equal(out[k], want[k]) for k in want)


def test_graphs_of_several_lengths():
    """Captured passes of growing lengths, with calls outside between them; a graph that is gone takes no other's scratch with it."""
    lin = lm.Linear8(300, 200, bias=torch.randn(200, device="cuda"), weight=torch.randn(200, 300, device="cuda"))
    kept = []
    for M in (70, 9, 400, 33):
        x, dy = torch.randn(M, 300, device="cuda"), torch.randn(M, 200, device="cuda")
        want = lin.forward(x, keep=True)
        grads = lin.backward(dy)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = lin.forward(x)
            y2 = lin.forward(x, keep=True)
            out = lin.backward(dy)
        kept.append((graph, y, y2, out, want, {k: v.clone() for k, v in grads.items()}, x, dy))   # (a graph reads its inputs where they are)
    del kept[2], graph, y, y2, out
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for graph, y, y2, out, want, grads, _, _ in kept:
        for t in (y, y2, *out.values()):
            t.fill_(7)
        lin.forward(torch.randn(500, 300, device="cuda"), keep=True)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(y2, want) and all(torch.equal(out[k], grads[k]) for k in grads)


@pytest.mark.parametrize("M,I,O,rank", [(128, 8192, 256, 0), (128, 8192, 256, 7), (32, 4096, 300, 3), (200, 300, 257, 0)])   # (the last: one slice)
def test_a_lost_signal_stores_nothing(M, I, O, rank):
    """One CTA of a cluster that waits in vain: an error code, no output from the CTAs that would add its part, and a usable context."""
    x, w, _, _ = _make(M, I, O, torch.float32, 13)
    lin = lm.Linear8(I, O, weight=w.cuda())
    want = lin.forward(x.cuda(), keep=True)
    q, s = lin.kept
    y = torch.full((M, O), 7.0, device="cuda")
    lbt.selftest_linear8_timeout(q, s, lin.q_w, lin.s_w, y, I, rank, lin.status, 2000)
    torch.cuda.synchronize()
    assert (y == 7).all()
    with pytest.raises(lbt.LbtError) as e:
        lin.check()
    assert e.value.status == lbt.ERR_TIMEOUT
    lin.check()   # (said once)
    assert torch.equal(lin.forward(x.cuda()), want)
    lin.check()
    with pytest.raises(lbt.LbtError) as e:
        lbt.selftest_linear8_timeout(q, s, lin.q_w, lin.s_w, y, I, 8, lin.status, 2000)
    assert e.value.status == lbt.ERR_UNSUPPORTED


@pytest.mark.parametrize("cols", [1, 100, 128, 1000, 1024, 1030, 9000])
def test_code_rows_of_a_wider_matrix(cols):
    """Rows of codes inside a wider matrix: zeros up to the next multiple of 16 columns, what lies behind them stays as it was."""
    rows, pitch = 5, lbt.pitch8(cols)
    ldq = pitch + 48
    x = torch.randn(rows, cols, device="cuda")
    q, want = torch.full((rows, ldq), 77, dtype=torch.int8, device="cuda"), torch.empty(rows, pitch, dtype=torch.int8, device="cuda")
    s, want_s = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    lbt.rows8_quantize(x, want, want_s)
    assert not want[:, cols:].any()
    for kind in (torch.float32, torch.bfloat16):
        xk = x.to(kind)
        lbt.rows8_quantize(xk, want, want_s)
        q.fill_(77)
        assert lbt.lib().lbt_rows8_quantize(xk.data_ptr(), lbt.TYPES[kind], rows, cols, cols, q.data_ptr(), ldq, s.data_ptr(), None) == lbt.OK
        torch.cuda.synchronize()
        assert torch.equal(q[:, :pitch], want) and torch.equal(s, want_s) and (q[:, pitch:] == 77).all()


@pytest.mark.parametrize("M,I,O", [(1, 50000, 130), (8, 6000, 130), (16, 3000, 257), (9, 4096, 384), (16, 2112, 100), (16, 1920, 384), (3, 13500, 100), (1, 41000, 70)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
def test_few_tokens_with_long_rows(M, I, O, dtype):
    """Codes that fill a multiprocessor's shared memory: blocks of sixteen warps, and the longest of eight."""
    x, w, b, _ = _make(M, I, O, dtype, M + I)
    guard = Guard()
    lin = lm.Linear8(I, O, bias=b.cuda(), weight=w.cuda())
    y = guard.alloc((M, O), dtype)
    lin.forward(x.cuda(), out=y, keep=True)
    q_w, s_w = _rows8(w)
    q_x, s_x = _rows8(x.float())
    assert torch.equal(lin.kept[0].cpu()[:, :I].double(), q_x) and not lin.kept[0][:, I:].any() and torch.equal(lin.kept[1].cpu(), s_x)
    _close(y, q_x @ q_w.T, s_x.double()[:, None] * s_w.double(), b, "y")
    lin.check()
    guard.check()


@pytest.mark.parametrize("M,I,O", [(17, 200, 19100), (32, 256, 19200), (64, 130, 24000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
def test_few_tokens_to_many_channels(M, I, O, dtype):
    """More channels than 74 tiles of 256 columns hold: tiles of 256 rows, few of them tokens."""
    x, w, b, _ = _make(M, I, O, dtype, M + I)
    guard = Guard()
    lin = lm.Linear8(I, O, bias=b.cuda(), weight=w.cuda())
    y = guard.alloc((M, O), dtype)
    lin.forward(x.cuda(), out=y)
    q_w, s_w = _rows8(w)
    q_x, s_x = _rows8(x.float())
    _close(y, q_x @ q_w.T, s_x.double()[:, None] * s_w.double(), b, "y")
    guard.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16], ids=str)
@pytest.mark.parametrize("M,I,O", [(2304, 384, 2304), (2500, 130, 2100)])
def test_many_tiles_with_bias(M, I, O, dtype):
    """The CTA pairs' epilogue with a bias, fp32 and fp16 outputs, a 16-bit dW."""
    x, w, b, dy = (t.cuda() for t in _make(M, I, O, dtype, 6))
    lin = lm.Linear8(I, O, bias=b, weight=w)
    y = lin.forward(x, keep=True)
    out = lin.backward(dy, dw_dtype=torch.bfloat16)
    q_x, s_x, q_w, s_w = lin.kept[0][:, :I].double(), lin.kept[1].double(), lin.q_w[:, :I].double(), lin.s_w.double()
    q_r, s_r = _rows8(dy.float().cpu() * lin.s_w.cpu())
    q_c, s_c = _rows8((dy.float().cpu() * lin.kept[1].cpu()[:, None]).T.contiguous())
    _close(y.cpu(), (q_x @ q_w.T).cpu(), (s_x[:, None] * s_w).cpu(), b.cpu(), "y")
    _close(out["dx"].cpu(), (q_r.cuda() @ q_w).cpu(), s_r.double()[:, None], None, "dx")
    _close(out["dw"].cpu(), (q_c.cuda() @ q_x).cpu(), s_c.double()[:, None], None, "dw")
    s = dy.double()
    assert ((out["dbias"].double() - s.sum(0)).abs() <= M * 2.0 ** -24 * s.abs().sum(0) + 1e-37).all()


@pytest.mark.parametrize("M,I,O", [(0, 64, 48), (1, 200, 150), (16, 200, 150), (40, 130, 77), (300, 515, 150), (2304, 384, 2304)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
def test_from_codes(M, I, O, dtype):
    """A product that starts from codes gives the bits of the one that makes them; rows of a wider output at an odd offset."""
    x, w, b, dy = (t.cuda() for t in _make(M, I, O, dtype, 12))
    lin = lm.Linear8(I, O, bias=b, weight=w)
    y = lin.forward(x, keep=True)
    want = lin.backward(dy)
    served = lm.Linear8.from_codes(lin.q_w, lin.s_w, I, bias=b)
    q, s = (t.clone() for t in lin.kept)
    wide = torch.full((M, O + 21), 7.0, dtype=dtype, device="cuda")
    served.forward_codes(q, s, out=wide[:, 5:5 + O], keep=True)
    assert torch.equal(wide[:, 5:5 + O], y) and (wide[:, :5] == 7).all() and (wide[:, 5 + O:] == 7).all()
    assert torch.equal(served.forward_codes(q, s, dtype=dtype), y)
    got = served.backward(dy)
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_the_binding_gives_the_layers_bits():
    M, I, O = 70, 300, 200
    x, w, b, dy = (t.cuda() for t in _make(M, I, O, torch.bfloat16, 14))
    lin = lm.Linear8(I, O, bias=b, weight=w)
    want = lin.forward(x, keep=True)
    grads = lin.backward(dy)
    q, s, y = torch.empty_like(lin.kept[0]), torch.empty_like(lin.kept[1]), torch.empty_like(want)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lbt.linear8_forward(x, lin.q_w, lin.s_w, y, q, s, b, status)
    assert torch.equal(y, want) and torch.equal(q, lin.kept[0]) and torch.equal(s, lin.kept[1])
    lbt.linear8_matmul(q, s, lin.q_w, lin.s_w, y.zero_(), I, b, status)
    assert torch.equal(y, want)
    dx, dw, db = torch.empty_like(x), torch.empty(O, I, device="cuda"), torch.empty(O, device="cuda")
    lbt.linear8_backward(dy, lin.q_w, lin.s_w, q, s, I, dx, dw, db, dev_status=status)
    assert torch.equal(dx, grads["dx"]) and torch.equal(dw, grads["dw"]) and torch.equal(db, grads["dbias"]) and int(status) == 0
