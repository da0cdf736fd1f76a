"""AdamW over many tensors against its definition in 64 bits.

Tolerances.  u = 2^-24 is half a step of float32.  m: beta and 1 - beta are rounded (u each), one product and the sum (u
each): 4 u (beta1 |m| + (1 - beta1) |g|); a scaled gradient has u more, and v twice that for the square, one for the
squaring: 8 u (..).  p: lr, the bias corrections (3 u each, computed on the device 4 u more), the root and the reciprocal (1
ulp = 2 u each), v's 8 u halved by the root, m's 5 u, eps, products and sums: below 32 u of the update's parts taken by
magnitude; then p's own rounding, half a step of its type.  Codes of moments are held bit for bit where the arithmetic is
exact: betas of 0.5 and 0.75 and operands of few bits."""
import math

import pytest
import torch

import moments_reference as ref
from paper_2304_14463_amd.moccasin import MoccasinError

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2304_14463_amd import training
    training.lib()
    return training


class Guarded:
    """A contiguous tensor between values that must stay as they are."""

    def __init__(self, x, dtype, lead=3):
        self.n, self.lead = x.numel(), lead
        self.whole = torch.full((lead + self.n + 40,), 77, dtype=dtype, device="cuda")
        self.inner = self.whole[lead:lead + self.n].view(x.shape)
        self.inner.copy_(x)

    def intact(self):
        return bool((self.whole[:self.lead] == 77).all()) and bool((self.whole[self.lead + self.n:] == 77).all())


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


SHAPES = [(1,), (7,), (31,), (33,), (0,), (8, 125), (2048,), (2049,), (5, 1003), (64, 96), (70001,)]


@pytest.mark.parametrize("param", TYPES)
@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("step", [1, 1000])
def test_moments_in_32_bits(tr, param, grad, step):
    g = torch.Generator().manual_seed(len(param) + 10 * len(grad) + step)
    normal = lambda shape, by: torch.randn(shape, generator=g, dtype=torch.float64) * by   # noqa: E731
    P, G = TYPES[param], TYPES[grad]
    p = [normal(s, 0.5).to(P) for s in SHAPES]
    d = [normal(s, 0.01).to(G) for s in SHAPES]
    m = [normal(s, 0.01).float() for s in SHAPES]
    v = [(normal(s, 0.01) ** 2).float() for s in SHAPES]
    decay = [0.1 if len(s) > 1 else 0.0 for s in SHAPES]
    kinds = [None, torch.float16, torch.bfloat16]
    gp, gm, gv = ([Guarded(x, t) for x in xs] for xs, t in ((p, P), (m, torch.float32), (v, torch.float32)))
    gd = [Guarded(x, G, 1) for x in d]
    gc = [Guarded(torch.zeros(s), kinds[i % 3]) if kinds[i % 3] else None for i, s in enumerate(SHAPES)]
    lr, betas, eps, scale = 1e-2, (0.9, 0.999), 1e-8, 0.7
    tr.moc_adamw_step([x.inner for x in gp], [x.inner for x in gd], [tr.Moments(a.inner, b.inner) for a, b in zip(gm, gv)], lr, step, betas, eps, decay,
                      [c and c.inner for c in gc], grad_scale=scale)
    for i in range(len(SHAPES)):
        pd, dd, md, vd = (x[i].double() for x in (p, d, m, v))
        want, wm, wv = ref.adamw(pd, dd, md, vd, lr, step, betas, eps, decay[i], scale)
        mag_m = betas[0] * md.abs() + (1 - betas[0]) * (scale * dd).abs()
        mag = lr * decay[i] * pd.abs() + lr / (1 - betas[0] ** step) * mag_m / (torch.sqrt(wv / (1 - betas[1] ** step)) + eps)
        assert bool(((gm[i].inner.cpu().double() - wm).abs() <= 6 * U * mag_m + tiny(torch.float32)).all())
        assert bool(((gv[i].inner.cpu().double() - wv).abs() <= 8 * U * wv + tiny(torch.float32)).all())
        for got in [gp[i]] + ([gc[i]] if gc[i] else []):
            t = got.inner.dtype
            bound = 32 * U * mag + U * want.abs()
            assert bool(((got.inner.cpu().double() - want).abs() <= bound + half_step(t) * (want.abs() + bound) + tiny(t)).all())
        assert all(x.intact() for x in (gp[i], gd[i], gm[i], gv[i])) and (gc[i] is None or gc[i].intact())
        assert torch.equal(gd[i].inner.cpu(), d[i])


def few_bits(g, shape, bits, low, high):
    """whole numbers of so many bits times 2^low..2^high, signed"""
    e = torch.randint(low, high + 1, shape, generator=g).double()
    return torch.randint(-(1 << bits) + 1, 1 << bits, shape, generator=g).double() * torch.exp2(e)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 1000, 2047, 2049, 70001])
@pytest.mark.parametrize("seed,step", [(0, 1), (2 ** 63 + 12345678901, 77), (5, 2 ** 33 + 9)])
def test_codes_of_moments_are_the_definition_bit_for_bit(tr, n, seed, step):
    """Exact arithmetic: m is a code of 4 bits times 2^k, halved, and the gradient's half; v is 0.75 of a code and a quarter of
    the gradient's square.  All terms lie within 24 bits of each other."""
    g = torch.Generator().manual_seed(n)
    blocks = -(-n // 32)
    mc = torch.randint(0, 2, (n,), generator=g) * 128 + torch.randint(48, 127, (n,), generator=g)      # normal codes of 10 exponents
    vc = torch.randint(150, 255, (n,), generator=g)
    mk, vk = torch.full((blocks,), 120), torch.full((blocks,), 110)                                    # 2^-7, 2^-17
    grad = few_bits(g, (n,), 3, -9, -5)
    grad[torch.rand(n, generator=g) < 0.1] = 0
    gm, gv = Guarded(mc, torch.uint8), Guarded(vc, torch.uint8, 5)
    sm, sv = Guarded(mk, torch.uint8, 1), Guarded(vk, torch.uint8)
    p, d = torch.zeros(n, device="cuda"), grad.float().cuda()
    other = torch.ones(40, device="cuda")
    step_number = 1
    # the tensor's number is its place in the list, empty ones counted
    tr.moc_adamw_step([other, p], [other * 0.5, d], [tr.zero_moments(other), tr.Moments(gm.inner, gv.inner, sm.inner, sv.inner)], 0.01, step, (0.5, 0.75), seed=seed)
    m = 0.5 * ref.values(mc, mk, False) + 0.5 * grad
    v = 0.75 * ref.values(vc, vk, True) + 0.25 * grad * grad
    assert torch.equal(m, m.float().double()) and torch.equal(v, v.float().double())   # the premise
    bits = ref.random_bits(seed, step, step_number, torch.arange(n))
    for got, scales, x, b, second in ((gm, sm, m, bits[0], False), (gv, sv, v, bits[1], True)):
        codes, k = ref.codes_of(x, b, second)
        assert torch.equal(scales.inner.cpu(), k)
        same = codes if second else torch.where(x == 0, codes & 127, codes)
        mine = got.inner.cpu() if second else torch.where(x == 0, got.inner.cpu() & 127, got.inner.cpu())
        assert torch.equal(mine, same)
        assert got.intact() and scales.intact()
    (_, _), (rm, rv) = tr.moc_moments_read([tr.zero_moments(other), tr.Moments(gm.inner, gv.inner, sm.inner, sv.inner)])
    assert torch.equal(rm.cpu().double(), ref.values(gm.inner, sm.inner, False)) and torch.equal(rv.cpu().double(), ref.values(gv.inner, sv.inner, True))


def test_ordinary_betas_round_to_a_neighbour_and_to_the_mean(tr):
    """What is stored is one of the codes around the value, and its mean over the random bits is the value: of N roundings the mean
    of (stored - value) / distance of the codes has a deviation of at most 0.5 / sqrt(N); six are allowed, and 2^-15 for the
    random bits' number.  A code next to the value by less than the arithmetic's error (8 u of the value: 2^-18 of a distance) may
    be the one beyond."""
    g = torch.Generator().manual_seed(3)
    n, times = 4096, 64
    m0, v0 = torch.randn(n, generator=g, dtype=torch.float64), torch.rand(n, generator=g, dtype=torch.float64) + 0.01
    grad = torch.randn(n, generator=g).cuda()
    start = tr.zero_moments(torch.zeros(n, device="cuda"))
    mc, mk = ref.codes_of(m0, torch.full((n,), 1 << 15), False)
    vc, vk = ref.codes_of(v0, torch.full((n,), 1 << 15), True)
    mv, vv = ref.values(mc, mk, False), ref.values(vc, vk, True)
    _, m, v = ref.adamw(torch.zeros(n).double(), grad.cpu().double(), mv, vv, 0, 1, (0.9, 0.999), 1e-8, 0)
    sums = {False: torch.zeros(n).double(), True: torch.zeros(n).double()}
    seen = set()
    for seed in range(times):
        moments = tr.Moments(mc.cuda(), vc.cuda(), mk.cuda(), vk.cuda())
        tr.moc_adamw_step([torch.zeros(n, device="cuda")], [grad], [moments], 0.0, 1000 + seed, seed=seed // 2)
        seen.add(moments.v.cpu().numpy().tobytes())
        for codes, scales, x, second in ((moments.m, moments.m_scales, m, False), (moments.v, moments.v_scales, v, True)):
            low, share, k = ref.neighbours(x, second)
            assert torch.equal(scales.cpu().long(), k + 127)
            up = (codes.cpu().long() & (255 if second else 127)) - low
            assert bool(((up == 0) | (up == 1) | ((share < 2.0 ** -18) & (up == -1)) | ((share > 1 - 2.0 ** -18) & (up == 2))).all())
            sums[second] += up - share
    assert len(seen) == times
    for s in sums.values():
        assert abs(float(s.mean()) / times) < 6 * 0.5 / math.sqrt(n * times) + 2.0 ** -15
        assert float((s / times).abs().max()) < 6 * 0.5 / math.sqrt(times)
    assert start.m.sum() == 0


def test_second_moments_fall_where_nearest_codes_would_not(tr):
    """1000 steps without a gradient leave 0.999^1000 = 0.368 of v; the sum of 65536 values falls with it.  A step's rounding
    has a variance of at most (a code's distance)^2 / 4 with probability of the share 0.001 v / distance: below 0.001 * v *
    0.125 v a step and value, so the sum is off by less than 6 sqrt(1000 * 0.000125 / 65536) = 0.8 %; 1 % is allowed."""
    n = 1 << 16
    p, grad = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    g = torch.Generator().manual_seed(1)
    c, k = ref.codes_of(torch.rand(n, generator=g).double() + 0.5, torch.full((n,), 1 << 15), True)
    zero = tr.zero_moments(p)
    moments = tr.Moments(zero.m, c.cuda(), zero.m_scales, k.cuda())
    before = ref.values(moments.v, moments.v_scales, True).sum()
    for step in range(1, 1001):
        tr.moc_adamw_step([p], [grad], [moments], 1e-3, step, weight_decay=0.0)
    after = ref.values(moments.v, moments.v_scales, True).sum()
    assert abs(float(after / before) / 0.999 ** 1000 - 1) < 0.01
    assert not moments.m.any() and not p.any()


def test_values_that_are_not_finite_and_the_borders(tr):
    n = 200
    grad = torch.zeros(n)
    grad[0], grad[33], grad[70], grad[100], grad[130] = math.nan, math.inf, -math.inf, 1e-30, 3e38
    grad[160:192] = 2.0 ** -60
    grad[160] = 1.0
    p = torch.ones(n, device="cuda")
    moments = tr.zero_moments(p)
    tr.moc_adamw_step([p], [grad.cuda()], [moments], 1e-3, 1, (0.5, 0.5))
    (m, v), = tr.moc_moments_read([moments])
    m, v, c = m.cpu(), v.cpu(), moments.v.cpu()
    assert bool(m[[0, 33, 70]].isnan().all()) and bool(v[[0, 33, 70, 130]].isnan().all())   # 3e38 squared is infinite
    assert m[130] == 1.5 * 2.0 ** 126 or m[130] == 1.625 * 2.0 ** 126 or abs(float(m[130]) / 1.5e38 - 1) <= 0.125
    assert bool((c[161:192] == 1).all()) and float(v[160]) == 0.5   # positive: never code 0
    assert bool((m[161:192].abs() <= 2.0 ** -9 * 0.5).all())
    rest = torch.ones(n, dtype=torch.bool)
    rest[[0, 33, 70, 100, 130]] = False
    rest[160:192] = False
    assert not m[rest].any() and not v[rest].any()
    assert p.cpu()[0].isnan() and bool((p.cpu()[rest] == torch.tensor(1.0) - torch.tensor(1e-3) * torch.tensor(0.01)).all())


def test_many_tensors_of_both_kinds(tr):
    """More tensors than a launch takes, moments in 8 and in 32 bits by turns: each as if it were stepped alone (in 8 bits at its
    number of the list)."""
    g = torch.Generator().manual_seed(9)
    shapes = [(1 + 37 * i % 301,) for i in range(133)] + [(300, 1000)]
    p = [torch.randn(s, generator=g).cuda() for s in shapes]
    d = [torch.randn(s, generator=g).cuda() for s in shapes]
    moments = [tr.zero_moments(x, 8 if i % 3 else 32) for i, x in enumerate(p)]
    single = [x.clone() for x in p]
    alone = [tr.zero_moments(x, 8 if i % 3 else 32) for i, x in enumerate(p)]
    for step in (1, 2):
        tr.moc_adamw_step(p, d, moments, 0.01, step, seed=4)
        for i in range(len(p)):
            skip = [torch.zeros(0, device="cuda")] * i
            tr.moc_adamw_step(skip + [single[i]], skip + [d[i]], [tr.zero_moments(x) for x in skip] + [alone[i]], 0.01, step, seed=4)
    for i in range(len(p)):
        assert torch.equal(p[i], single[i])
        for k in ("m", "v", "m_scales", "v_scales"):
            a, b = getattr(moments[i], k), getattr(alone[i], k)
            assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("bits", [8, 32])
def test_rates_and_steps_on_the_device_and_a_captured_step(tr, bits):
    """A replay reads rate, step and scale where they are then; the same numbers from the host give the same within the
    corrections' roundings (8 u of the update), moments the same bits."""
    g = torch.Generator().manual_seed(bits)
    start, grad = torch.randn(3001, generator=g).cuda(), torch.randn(3001, generator=g).cuda()
    p, moments = start.clone(), tr.zero_moments(start, bits)
    lr, step, scale = torch.tensor([0.01], device="cuda"), torch.tensor([1], device="cuda"), torch.tensor([1.0], device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        tr.moc_adamw_step([p.clone()], [grad], [tr.zero_moments(start, bits)], lr, step, grad_scale=scale)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tr.moc_adamw_step([p], [grad], [moments], lr, step, grad_scale=scale, seed=8)
    q, other = start.clone(), tr.zero_moments(start, bits)
    eager, own = start.clone(), tr.zero_moments(start, bits)
    for t in range(1, 6):
        lr.fill_(0.01 / t)
        step.fill_(t)
        scale.fill_(0.5 + 0.25 * t)
        graph.replay()
        torch.cuda.synchronize()
        before = q.clone()
        tr.moc_adamw_step([eager], [grad], [own], lr, step, grad_scale=scale, seed=8)
        tr.moc_adamw_step([q], [grad], [other], float(lr), t, grad_scale=float(scale), seed=8)
        assert torch.equal(p, eager) and torch.equal(moments.m, own.m) and torch.equal(moments.v, own.v)
        assert torch.equal(moments.m, other.m) and torch.equal(moments.v, other.v)
        moved = (q - before).abs().double() + 0.01
        assert bool(((p.double() - q.double()).abs() <= t * (8 * U * moved + 2 * U * q.abs())).all())
    # a rate alone on the device
    a, b = start.clone(), start.clone()
    tr.moc_adamw_step([a], [grad], [tr.zero_moments(start, bits)], torch.tensor([0.003], device="cuda"), 7)
    tr.moc_adamw_step([b], [grad], [tr.zero_moments(start, bits)], 0.003, 7)
    assert bool(((a - b).abs() <= 8 * U * (0.03 + b.abs())).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_every_code_reads_as_defined(tr, dtype):
    t = TYPES[dtype]
    codes = torch.arange(256, dtype=torch.uint8).repeat(200)
    scales = torch.arange(20, 220, dtype=torch.uint8).repeat_interleave(8)
    (m, v), = tr.moc_moments_read([tr.Moments(codes.cuda(), codes.cuda(), scales.cuda(), scales.cuda())], t)
    for got, second in ((m, False), (v, True)):
        want = ref.values(codes, scales, second).to(t)
        assert got.dtype == t and torch.equal(got.cpu().nan_to_num(3e4), want.nan_to_num(3e4)) and torch.equal(got.cpu().isnan(), want.isnan())
    x = torch.randn(99, device="cuda")
    out = torch.zeros(99, device="cuda", dtype=t), torch.zeros(99, device="cuda", dtype=t)
    got = tr.moc_moments_read([tr.Moments(x, x.abs())], out=[out])
    assert got[0] is out and torch.equal(out[0], x.to(t)) and torch.equal(out[1], x.abs().to(t))


def test_refusals(tr):
    x = lambda *s, **k: torch.ones(*s, device="cuda", **k)   # noqa: E731
    p, g, mo = x(64), x(64), tr.zero_moments(x(64))
    call = lambda ps=None, gs=None, ms=None, **k: tr.moc_adamw_step(ps or [p], gs or [g], ms or [mo], k.pop("lr", 0.01), k.pop("step", 1), **k)   # noqa: E731
    shared = x(100)
    for bad in (lambda: call([x(64, 2)[:, 0]]), lambda: call(gs=[x(63)]), lambda: call(gs=[x(8, 8)]), lambda: call(gs=[g, g]), lambda: call([p.cpu()]), lambda: call([p.double()]), lambda: call([p.int()]),
                lambda: call(ms=[tr.Moments(x(64), x(63))]), lambda: call(ms=[tr.Moments(x(64), mo.v)]), lambda: call(ms=[tr.Moments(mo.m, mo.v, mo.m_scales, mo.v_scales[:1])]),
                lambda: call(ms=[tr.Moments(x(64).half(), x(64).half())]), lambda: call(ms=[tr.Moments(x(64), x(64), mo.m_scales)]), lambda: call(copies=[x(64)]),
                lambda: call(copies=[x(63).half()]), lambda: call(copies=[None, None]), lambda: call(weight_decay=[0.1, 0.2]), lambda: call(weight_decay=-1.0), lambda: call(weight_decay=math.nan),
                lambda: call(weight_decay=math.inf), lambda: call(betas=(1.0, 0.9)), lambda: call(betas=(0.9, -0.1)), lambda: call(eps=0.0), lambda: call(eps=1e-40), lambda: call(step=0), lambda: call(lr=math.inf),
                lambda: call(lr=x(2)), lambda: call(lr=x(1).double()), lambda: call(step=x(1)), lambda: call(grad_scale=math.nan),
                # memory that is written twice, or read and written
                lambda: call([p, p], [g, g], [mo, tr.zero_moments(p)]), lambda: call([p, x(64)], [g, g], [mo, mo]), lambda: call([p], [p]), lambda: call([shared[:64]], [shared[36:]]),
                lambda: call([shared[:64], shared[36:]], [g, g], [mo, tr.zero_moments(p)]), lambda: call(ms=[tr.Moments(mo.m, mo.m, mo.m_scales, mo.v_scales)]),
                lambda: tr.moc_moments_read([mo], out=[(x(64), x(63))]), lambda: tr.moc_moments_read([mo], out=[(p, p)]), lambda: tr.moc_moments_read([mo], torch.int32), lambda: tr.zero_moments(p, 4)):
        with pytest.raises((ValueError, MoccasinError)):
            bad()
    for bad in (lambda: call([3]), lambda: call(ms=[3]), lambda: tr.moc_adamw_step(3, [], [], 0.1, 1), lambda: tr.moc_moments_read(p[0]), lambda: call(lr="x"), lambda: call(step=1.5)):
        with pytest.raises(TypeError):
            bad()
    torch.cuda.synchronize()
    assert bool((p == 1).all()) and not mo.m.any() and not mo.v.any() and bool((shared == 1).all())
    # the gradients of tied parameters, and of a list of nothing
    call([p, x(64)], [g, g], [tr.zero_moments(p), tr.zero_moments(p)])
    tr.moc_adamw_step([], [], [], 0.1, 1)
    assert tr.moc_moments_read([]) == []
    call([x(0)], [x(0)], [tr.zero_moments(x(0))])


def test_another_stream_and_device(tr, monkeypatch):
    p, g = torch.ones(1 << 20, device="cuda"), torch.ones(1 << 20, device="cuda")
    mo = tr.zero_moments(p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tr.moc_adamw_step([p], [g], [mo], 0.5, 1, weight_decay=0.0, stream=side)
    side.synchronize()
    assert bool(((p - 0.5).abs() < 1e-6).all())
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for call in (lambda: tr.moc_adamw_step([p], [g], [mo], 0.5, 1), lambda: tr.moc_moments_read([mo])):
            with pytest.raises(ValueError, match="cuda:0.*cuda:1"):
                call()


def test_lists_may_be_iterators(tr):
    """What an optimizer is given: parameters that can be gone over once."""
    shapes = [(5, 70), (33,), (1,)]
    params, grads = [torch.ones(s, device="cuda") for s in shapes], [torch.full(s, 0.5, device="cuda") for s in shapes]
    moments = [tr.zero_moments(p, 32) for p in params]
    want = [p.clone() for p in params]
    kept = [tr.zero_moments(p, 32) for p in params]
    tr.moc_adamw_step(want, grads, kept, 0.1, 1)
    tr.moc_adamw_step(iter(params), iter(grads), iter(moments), 0.1, 1)
    assert all(torch.equal(a, b) for a, b in zip(params, want)) and bool((params[0] != 1).all())
    read = tr.moc_moments_read(iter(moments))
    assert len(read) == 3 and all(torch.equal(m, k.m) and torch.equal(v, k.v) for (m, v), k in zip(read, kept))
