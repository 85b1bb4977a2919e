"""AdamW over many tensors against the formula in 64 bits.

Tolerances.  A step is about ten fp32 roundings: p, m, v within 16 * 2^-24 of the magnitudes that enter (|p| + |update|, |m| +
|g|, v + g^2), p then rounded to its type.  8-bit moments: the value stored is the nearest e4m3 multiple of the scale, so it
lies within half an e4m3 step of the 64-bit value: 2^-4 of it, or 2^-10 of the scale below the normal range; the smallest
positive code stands for every smaller positive root.
"""
import pytest
import torch

from guard import Guard
from paper_2407_12637_b200 import lbt, lm

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
B1, B2 = 0.9, 0.99


def _formula(p, g, m, v, lr, wd, step, eps):
    m = B1 * m + (1 - B1) * g
    v = B2 * v + (1 - B2) * g * g
    up = lr * (m / (1 - B1 ** step)) / (torch.sqrt(v / (1 - B2 ** step)) + eps)
    return p * (1 - lr * wd) - up, m, v, up


def _tensors(sizes, dtype, gdtype, seed, guard):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ps, gs = [], []
    for n in sizes:
        p, g = guard.alloc((n,), dtype), guard.alloc((n,), gdtype)
        p.copy_(torch.randn(n, generator=gen, device="cuda"))
        g.copy_(torch.randn(n, generator=gen, device="cuda").pow(3) * 0.01)
        ps.append(p)
        gs.append(g)
    return ps, gs


SIZES = [1, 2, 31, 255, 256, 257, 0, 1000, 4096, 70000, 513, 8]


@pytest.mark.parametrize("dtype,gdtype", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16),
                                          (torch.float16, torch.float32)], ids=str)
@pytest.mark.parametrize("bits", [8, 32])
def test_steps(bits, dtype, gdtype):
    guard = Guard()
    ps, gs = _tensors(SIZES, dtype, gdtype, 1, guard)
    lrs, wds = [1e-2 / (i + 1) for i in range(len(SIZES))], [0.1 * (i % 3) for i in range(len(SIZES))]
    state = torch.float32 if bits == 32 else torch.float8_e4m3fn
    make = lambda kind, sizes: [guard.alloc((n,), kind, 0) if kind == torch.float32 else guard.alloc((n,), torch.uint8, 0).view(kind) for n in sizes]  # noqa: E731
    blocks = [-(-n // 256) for n in SIZES]
    scales = {"m_scale": make(torch.float32, blocks), "v_scale": make(torch.float32, blocks)} if bits == 8 else {}
    opt = lm.AdamW(ps, gs, make(state, SIZES), make(state, SIZES), **scales, lr=lrs, betas=(B1, B2), eps=1e-6, weight_decay=wds)
    for step in (1, 2, 3):
        for g in gs:
            g.mul_(0.7).add_(0.001)
        before = [p.double() for p in ps]
        m0, v0 = ([t.double() for t in part] for part in opt.moments())
        opt.step()
        m1, v1 = opt.moments()
        for i, n in enumerate(SIZES):
            if n == 0:
                continue
            g = gs[i].double()
            p, m, v, up = _formula(before[i], g, m0[i], v0[i], lrs[i], wds[i], step, 1e-6)
            # the moments' own roundings: m = b1 m + ..., v up to 4 roundings; the update's magnitude bounds their effect on p
            size_m, size_v = m0[i].abs() + g.abs(), v0[i] + g * g
            shake = lrs[i] / (1 - B1 ** step) * size_m / (torch.sqrt(v / (1 - B2 ** step)) + 1e-6)
            tol = 16 * EPS * (before[i].abs() + up.abs() + shake * (1 + size_v / v.clamp(min=1e-300))) + 1.01 * HALF_ULP[dtype] * p.abs()
            assert ((ps[i].double() - p).abs() <= tol + (2.0 ** -25 if dtype == torch.float16 else 0)).all(), (i, step)
            if bits == 32:
                assert ((m1[i].double() - m).abs() <= 4 * EPS * size_m).all() and ((v1[i].double() - v).abs() <= 4 * EPS * size_v).all()
                continue
            u, b = torch.sqrt(v), torch.arange(n, device="cuda") // 256
            for got, want, scale in ((opt.m[i].double() * opt.m_scale[i].double()[b], m, opt.m_scale[i].double()),
                                     (opt.v[i].double() * opt.v_scale[i].double()[b], u, opt.v_scale[i].double())):
                top = torch.zeros(blocks[i], dtype=torch.float64, device="cuda").index_reduce_(0, b, want.abs(), "amax")
                assert ((scale - top / 448).abs() <= 16 * EPS * top / 448 + 1e-44).all()
                near = want.abs() * 2.0 ** -4 + scale[b] * 2.0 ** -10
                assert ((got - want).abs() <= near * 1.0001 + (scale[b] * 2.0 ** -9 if want is u else 0)).all()
            assert (opt.v[i].double()[u > 0] > 0).all()
    guard.check()


@pytest.mark.parametrize("count", [0, 1, 40, 41, 399, 400, 401, 900])
def test_many_tensors_are_one_step(count):
    """Any number of tensors gives what each alone gives."""
    sizes = [(7 * i) % 300 for i in range(count)]
    ps, gs = _tensors(sizes, torch.float32, torch.float32, 2, Guard())
    alone = [p.clone() for p in ps]
    lm.AdamW(ps, gs, lr=1e-2).step()
    for i in range(0, count, max(1, count // 12)):
        opt = lm.AdamW([alone[i]], [gs[i]], lr=1e-2)
        opt.step()
        assert torch.equal(alone[i], ps[i])


@pytest.mark.parametrize("bits", [8, 32])
def test_unaligned_views_give_the_same_bits(bits):
    g = torch.Generator(device="cuda").manual_seed(4)
    n = 5000
    p, gr = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    want = lm.AdamW([p.clone()], [gr], state_bits=bits)
    shift = lambda t: torch.cat([t.new_zeros(1), t])[1:]  # noqa: E731
    got = lm.AdamW([shift(p)], [shift(gr)], state_bits=bits)
    for _ in range(2):
        want.step()
        got.step()
    assert torch.equal(want.params[0], got.params[0])
    for a, b in ((want.m, got.m), (want.v, got.v)):
        assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8))


@pytest.mark.parametrize("bits", [8, 32])
def test_scale_and_skip(bits):
    ps, gs = _tensors([700], torch.float32, torch.float32, 5, Guard())
    a, b = ps[0].clone(), ps[0].clone()
    scaled = lm.AdamW([a], [gs[0]], state_bits=bits)
    scaled.step(grad_scale=torch.tensor([0.25], device="cuda"))
    plain = lm.AdamW([b], [gs[0] * 0.25], state_bits=bits)
    plain.step()
    assert torch.equal(a, b)
    held = a.clone()
    scaled.step(skip=torch.tensor([1], dtype=torch.int32, device="cuda"))
    assert torch.equal(a, held)
    scaled.step(skip=torch.tensor([0], dtype=torch.int32, device="cuda"))
    assert not torch.equal(a, held)


@pytest.mark.parametrize("bits", [8, 32])
def test_non_finite_gradients_stay_with_their_elements(bits):
    n = 600
    p, g = torch.ones(n, device="cuda"), torch.full((n,), 0.1, device="cuda")
    g[5], g[300] = float("nan"), float("inf")
    opt = lm.AdamW([p], [g], state_bits=bits)
    opt.step()
    rest = [i for i in range(n) if i not in (5, 300)]
    g[5] = g[300] = 0.1
    opt.step()
    m, v = opt.moments()
    for t in (p, m[0], v[0]):
        assert torch.isfinite(t[rest]).all() and not torch.isfinite(t[5]) and not torch.isfinite(t[300])
    assert (p[rest] == p[0]).all()


def test_small_roots_keep_small_steps():
    """Beside a gradient 10^6 times larger an element's root falls below the codes; it must not divide by eps alone."""
    p, g = torch.zeros(256, device="cuda"), torch.full((256,), 1e-6, device="cuda")
    g[0] = 1.0
    opt = lm.AdamW([p], [g], lr=1e-3, weight_decay=0.0, eps=1e-12)
    for _ in range(5):
        opt.step()
    assert p.abs().max() <= 5.1e-3


def test_follows_the_32_bit_states():
    """Twenty steps on a quadratic: the 8-bit states reach the same loss within a tenth."""
    g = torch.Generator(device="cuda").manual_seed(6)
    target, scale = torch.randn(4096, generator=g, device="cuda"), 0.1 + torch.rand(4096, generator=g, device="cuda")
    losses = []
    for bits in (8, 32):
        p, grad = torch.zeros(4096, device="cuda"), torch.zeros(4096, device="cuda")
        opt = lm.AdamW([p], [grad], lr=0.05, weight_decay=0.0, state_bits=bits)
        for _ in range(20):
            grad.copy_(scale * (p - target))
            opt.step()
        losses.append(float((scale * (p - target) ** 2).sum()))
    assert abs(losses[0] - losses[1]) <= 0.1 * losses[1]


def test_more_than_two_to_the_31_elements():
    n = 2 ** 31 + 300
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 255, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 255, n - 1], device="cuda")
    g[at] = 1.0
    opt = lm.AdamW([p], [g], lr=0.5, weight_decay=0.0)
    opt.step()
    assert torch.equal(p[at].float(), torch.full((6,), -0.5, device="cuda"))
    assert int((p != 0).sum()) == 6


def test_refusals():
    p, g = torch.zeros(10, device="cuda"), torch.zeros(10, device="cuda")
    for bad in (([p], []), ([p], [g[:9]]), ([p.double()], [g])):
        with pytest.raises(ValueError):
            lm.AdamW(*bad)
    with pytest.raises(ValueError):
        lm.AdamW([p], [g], state_bits=4)
    with pytest.raises(ValueError):
        lm.AdamW([p], [g], [p.clone()], [p.half()])
    with pytest.raises(ValueError):
        lm.AdamW([p], [g], lr=[1.0, 2.0])
    for betas, eps in (((1.0, 0.9), 1e-8), ((0.9, -0.1), 1e-8), ((0.9, 0.99), -1.0), ((float("nan"), 0.9), 1e-8)):
        with pytest.raises(lbt.LbtError) as e:
            lm.AdamW([p], [g], betas=betas, eps=eps).step()
        assert e.value.status == lbt.ERR_INVALID_ARG


def _state_bits(opt):
    """Everything a step writes, as bytes."""
    parts = opt.params + opt.m + opt.v + [s for s in opt.m_scale + opt.v_scale if s is not None]
    return [t.view(torch.uint8) for t in parts]


@pytest.mark.parametrize("count", [1, 41, 401])   # (401: two launches a step)
@pytest.mark.parametrize("bits", [8, 32])
def test_skipped_steps_do_not_count(bits, count):
    """Steps that were held back leave the bias corrections where they were: what follows is bit for bit an optimizer that never saw them."""
    ps, gs = _tensors([(37 * i) % 600 + 1 for i in range(count)], torch.float32, torch.float32, 7, Guard())
    held, taken = lm.AdamW(ps, gs, lr=1e-2, state_bits=bits), lm.AdamW([p.clone() for p in ps], gs, lr=1e-2, state_bits=bits)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    for skipped in (1, 1, 0, 1, 0, 0, 1, 1, 1, 0):
        for g in gs:
            g.mul_(0.9).add_(0.001)
        flag.fill_(skipped)
        held.step(skip=flag)
        if not skipped:
            taken.step()
        assert all(torch.equal(a, b) for a, b in zip(_state_bits(held), _state_bits(taken)))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_captured_step_counts_its_replays(bits):
    """Replays of a captured step, steps outside of the graph and held-back ones in any order: the bits of the same steps taken one by one."""
    ps, gs = _tensors([700, 33], torch.float32, torch.float32, 9, Guard())
    graphed, plain = lm.AdamW(ps, gs, lr=1e-2, state_bits=bits), lm.AdamW([p.clone() for p in ps], gs, lr=1e-2, state_bits=bits)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    graphed.step(skip=flag)
    plain.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step(skip=flag)
    taken = 1
    for replay, skipped in ((1, 0), (1, 0), (0, 0), (1, 1), (1, 0), (0, 1), (0, 0), (1, 0)):
        for g in gs:
            g.mul_(0.9).add_(0.001)
        flag.fill_(skipped)
        if replay:
            graph.replay()
        else:
            graphed.step(skip=flag)
        if not skipped:
            plain.step()
            taken += 1
        assert all(torch.equal(a, b) for a, b in zip(_state_bits(graphed), _state_bits(plain)))
        assert graphed.taken() == plain.taken() == taken


@pytest.mark.parametrize("bits", [8, 32])
def test_squares_that_overflow(bits):
    """A finite gradient whose square is infinite: v is, the update is 0 by the formula, then and in every later step; only the decay moves p."""
    n, big = 600, [5, 300, 599]
    p, g = torch.ones(n, device="cuda"), torch.full((n,), 0.1, device="cuda")
    opt = lm.AdamW([p], [g], lr=1e-2, weight_decay=0.1, state_bits=bits)
    decay, want = torch.tensor(1 - 1e-2 * 0.1, device="cuda"), torch.ones(3, device="cuda")
    for step in range(3):
        g[big] = torch.tensor([1e20, -3e38, 2e19] if step == 0 else [0.1, 0.0, -0.2], device="cuda")
        opt.step()
        want *= decay
        assert torch.equal(p[big], want) and torch.isfinite(p).all(), step
        assert torch.isfinite(opt.m[0].float()).all() and int((~torch.isfinite(opt.v[0].float())).sum()) == 3


def test_moments_in_codes_need_their_scales():
    p, g = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    codes = lambda: [torch.zeros(300, dtype=torch.float8_e4m3fn, device="cuda")]  # noqa: E731
    scales = [torch.ones(2, device="cuda")]
    for given in ({"m": codes()}, {"m": codes(), "v": codes()}, {"m": codes(), "v": codes(), "m_scale": scales}, {"m": codes(), "v": codes(), "v_scale": scales},
                  {"v": codes()}):
        with pytest.raises(ValueError):
            lm.AdamW([p], [g], **given)
    lm.AdamW([p], [g], codes(), codes(), scales, [scales[0].clone()]).step()


@pytest.mark.parametrize("dtype,gdtype", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float16), (torch.float16, torch.float32)], ids=str)
def test_many_blocks_are_the_same_steps(dtype, gdtype):
    """More than 18 944 blocks of 256 (a warp takes eight at a time): codes, scales and parameters are bit for bit those of the same
    tensors stepped in pieces of few blocks each."""
    sizes = [2_000_003, 256 * 9, 1, 256 * 8 - 1, 3_000_007, 17, 256 * 15 + 3, 700_001]
    assert sum(-(-n // 256) for n in sizes) > 148 * 32 * 4
    gen = torch.Generator(device="cuda").manual_seed(8)
    rand = lambda n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    ps, gs, ms, vs, mss, vss = [], [], [], [], [], []
    for n in sizes:
        b = -(-n // 256)
        ps.append(rand(n).to(dtype))
        gs.append((rand(n).pow(3) * 0.01).to(gdtype))
        ms.append((rand(n) * 100).clamp(-448, 448).to(torch.float8_e4m3fn))
        vs.append((rand(n).abs() * 100 + 0.01).clamp(max=448).to(torch.float8_e4m3fn))
        mss.append(torch.rand(b, generator=gen, device="cuda") * 1e-4)
        vss.append(torch.rand(b, generator=gen, device="cuda") * 1e-3)
    copy = lambda ts: [t.clone() for t in ts]  # noqa: E731
    whole = lm.AdamW(ps, gs, ms, vs, mss, vss, lr=1e-2, step=4)
    apart = [copy(t) for t in (ps, ms, vs, mss, vss)]
    cut = 256 * 1000
    pieces = [(i, at) for i, n in enumerate(sizes) for at in range(0, n, cut)]
    at = lambda ts: [ts[i][a:a + cut] for i, a in pieces]  # noqa: E731
    scales_at = lambda ts: [ts[i][a // 256:a // 256 + 1000] for i, a in pieces]  # noqa: E731
    for step in range(3):
        for g in gs:
            g.mul_(0.8).add_(0.001)
        whole.step()
        parts = [at(apart[0]), at(gs), at(apart[1]), at(apart[2]), scales_at(apart[3]), scales_at(apart[4])]
        for k in range(len(pieces)):
            lm.AdamW(*[[t[k]] for t in parts], lr=1e-2, step=4 + step).step()
        for a, b in zip((ps, ms, vs, mss, vss), apart):
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b)), step


@pytest.mark.parametrize("shift", [0, 1])   # (aligned, and element by element)
def test_a_second_moment_that_is_nan_shows(shift):
    n = 600
    p, m, v = (torch.full((n + shift,), x, device="cuda")[shift:] for x in (1.0, 0.1, 0.01))
    v[7], v[300] = float("nan"), float("inf")
    lm.AdamW([p], [torch.full((n,), 0.1, device="cuda")], [m], [v], step=3).step()
    assert p[7].isnan() and v[7].isnan() and torch.isfinite(p[300]) and torch.isinf(v[300]) and int(p.isnan().sum()) == 1
