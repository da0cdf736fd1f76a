"""The training operators against their definitions in 64 bits: 8-bit checkpoints bit for bit, the rest
within what their roundings can add up to.

Tolerances.  u = 2^-24 is half a step of float32.  A sum of n terms in any order is off by at most
(n - 1) u sum |term|; the matrix cores may cut instead of round, so twice that is allowed, n * 2^-23
sum |term|.  exp2 and the reciprocal are off by 1 ulp, their argument by 2^-22 of itself at most: an
activation and its derivative by 2^-18 of max(1, |u|) * |result's scale|.  What is written is off by a
half step of its type besides, half_step(dtype) |value|, or the half of the smallest subnormal."""
import itertools
import math
import zlib

import pytest
import torch

import training_reference as ref
from training_reference import Framed, TYPES, half_step

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2304_14463_amd import training
    training.lib()
    return training


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def normal(g, *shape, by=1.0):
    return torch.randn(*shape, generator=g, dtype=torch.float64) * by


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def near(got, want, bound, dtype=None):
    """|got - want| <= bound + the rounding to dtype, NaN and infinities in the same places"""
    got, want, dtype = got.double().cpu(), want.double().cpu(), dtype or got.dtype
    assert got.shape == want.shape
    nan = want.isnan()
    assert bool((got.isnan() == nan).all()), "NaN in other places"
    allowed = bound + half_step(dtype) * (want.abs() + bound) + tiny(dtype)
    off = torch.where(nan, 0.0, (got - want).abs() - allowed)
    assert float(off.max() if off.numel() else 0.0) <= 0, f"off by {float((got - want).abs().nan_to_num().max())}, {float(off.max())} more than allowed"


def framed_checkpoint(tr, rows, cols, fmt, lead=0, pad=0):
    codes, scales = Framed(rows, cols, torch.uint8, lead, pad), Framed(rows, -(-cols // 32), torch.uint8, lead, pad)
    return tr.Checkpoint(codes.inner, scales.inner, fmt), codes, scales


# ---- checkpoints --------------------------------------------------------------------------------

CHECKPOINT_SIZES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 1000), (7, 1247), (300, 64), (64, 2050), (1, 16385)]


def hard_values(g, rows, cols, dtype):
    """values of all magnitudes, borders between codes, zeros of both signs, what is not finite"""
    x = normal(g, rows, cols) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=g).double())
    x = x.to(dtype).double()
    f = torch.finfo(dtype)
    special = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, f.max, -f.max, f.smallest_normal, tiny(dtype), -tiny(dtype), 448.0, 464.0, 127.0, 127.5, 126.5,
                            1.0625, 1.1875, 0.5, 1.5, 2.5], dtype=torch.float64)
    pick = torch.rand(rows, cols, generator=g) < 0.05
    x = torch.where(pick, special[torch.randint(0, len(special), (rows, cols), generator=g)], x)
    if rows > 2:
        x[1] = 0.0
        x[2] = torch.randint(-130, 131, (cols,), generator=g).double() / 2   # ties of int8
    return x.to(dtype)


@pytest.mark.parametrize("rows,cols", CHECKPOINT_SIZES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_checkpoint_is_the_definition_bit_for_bit(tr, rows, cols, dtype, fmt):
    dtype = TYPES[dtype]
    x = hard_values(gen(rows, cols, str(dtype), fmt), rows, cols, dtype)
    want, scales = ref.keep(x, fmt, dtype)
    for lead, pad in ((0, 0), (1, 3), (8, 24)):
        xin = Framed(rows, cols, dtype, lead, pad)
        xin.of(x)
        kept, fc, fs = framed_checkpoint(tr, rows, cols, fmt, lead, pad)
        got = tr.moc_checkpoint_write(xin.inner, out=kept)
        assert got is kept
        assert ref.same_codes(kept.scales, scales) and ref.same_codes(kept.codes, want)
        assert fc.intact() and fs.intact()
        v = ref.values(want, scales, fmt)
        for to in TYPES.values():
            out = Framed(rows, cols, to, lead, pad)
            tr.moc_checkpoint_read(kept, to, out=out.inner)
            # a rounding once, and none where the type has the value
            assert torch.equal(out.inner.cpu().nan_to_num(3e5), v.to(to).nan_to_num(3e5)) and out.intact()
            if to == dtype:
                assert bool((out.inner.cpu().isfinite() == x.isfinite()).all())


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_read_through_the_activation(tr, act, fmt):
    g = gen(act, fmt)
    u = normal(g, 37, 500) * torch.exp2(torch.randint(-6, 8, (37, 1), generator=g).double())
    u[3, 5] = math.nan
    codes, scales = ref.keep(u, fmt, torch.float32)
    kept = tr.Checkpoint(codes.cuda(), scales.cuda(), fmt)
    v = ref.values(codes, scales, fmt)
    for dtype in TYPES.values():
        near(tr.moc_checkpoint_read(kept, dtype, act=act), ref.act(v, act), 2.0 ** -18 * v.abs().nan_to_num())


def test_every_code_and_scale_reads_as_defined(tr):
    codes = torch.arange(256, dtype=torch.uint8).repeat(234, 1)
    scales = torch.arange(16, 250, dtype=torch.uint8)[:, None].repeat(1, 8)
    for fmt in ("e4m3", "int8"):
        got = tr.moc_checkpoint_read(tr.Checkpoint(codes.cuda(), scales.cuda(), fmt), torch.float32).cpu()
        want = ref.values(codes, scales, fmt).float()
        assert torch.equal(got.nan_to_num(1.5, math.inf, -math.inf), want.nan_to_num(1.5, math.inf, -math.inf))


# ---- layer norm ---------------------------------------------------------------------------------

# one column, odd ones, each of the shapes that the kernels come in, rows that no registers hold
NORM_SIZES = [(1, 1), (3, 2), (5, 31), (9, 512), (6, 513), (4, 1000), (7, 1247), (3, 2050), (2, 4096), (3, 5000), (2, 8200), (3, 16384), (2, 16392), (2, 33001), (2, 40000)]


def norm_inputs(rows, cols, dtype, held):
    g = gen(rows, cols, str(dtype), held)
    x = (normal(g, rows, cols) * torch.exp(0.5 * normal(g, cols)) + 3 * normal(g, rows, 1)).to(dtype)
    gamma, beta = (1 + 0.1 * normal(g, cols)).float(), (0.1 * normal(g, cols)).float()
    if held == "tensor":
        return g, x, x.double(), gamma, beta
    codes, scales = ref.keep(x.double(), held, dtype)
    return g, (codes, scales), ref.values(codes, scales, held), gamma, beta


def norm_bounds(v, gamma, eps):
    """how far mean, rstd and (x - mean) * rstd may be, from the values v"""
    n = v.shape[1]
    size = v.abs().mean(1)
    dmean = (n * 2 * U + 2 * U) * size                                # the sum, the division
    d = v - v.mean(1, keepdim=True)
    var = (d * d).mean(1)
    spread = d.abs().amax(1) * 0 + d.abs().mean(1)
    dvar = 2 * dmean * spread * 0 + dmean * dmean + (n * 2 * U + 6 * U) * var + 4 * U * v.abs().amax(1) * spread
    drel = dvar / (2 * (var + eps)) + 4 * U                           # of rstd, relative
    rstd = (var + eps).rsqrt()
    h = d * rstd[:, None]
    dh = (dmean[:, None] + 2 * U * v.abs() + 2 * U * v.mean(1).abs()[:, None]) * rstd[:, None] + h.abs() * (drel[:, None] + 4 * U)
    return dmean, rstd * drel, h, dh


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("dtype,held", [("fp32", "tensor"), ("fp16", "tensor"), ("bf16", "tensor"), ("bf16", "e4m3"), ("fp16", "int8")])
def test_norm_forward(tr, rows, cols, dtype, held):
    dtype, eps = TYPES[dtype], 1e-5
    g, x, v, gamma, beta = norm_inputs(rows, cols, dtype, held)
    y, mean, rstd = ref.norm(v, gamma, beta, eps)
    dmean, drstd, h, dh = norm_bounds(v, gamma, eps)
    bound = dh * gamma.double().abs() + 4 * U * (h * gamma.double()).abs() + 2 * U * beta.double().abs()
    for lead, pad, fmt, ptype in ((0, 0, "e4m3", torch.float32), (1, 5, "int8", torch.bfloat16)):
        ga, be = gamma.to(ptype).cuda(), beta.to(ptype).cuda()
        if ptype != torch.float32:
            y, mean, rstd = ref.norm(v, ga.cpu(), be.cpu(), eps)
        if held == "tensor":
            xin = Framed(rows, cols, dtype, lead, pad).of(x)
        else:
            xin, _, _ = framed_checkpoint(tr, rows, cols, held, lead, pad)
            xin.codes.copy_(x[0]), xin.scales.copy_(x[1])
        out = Framed(rows, cols, dtype, lead, pad)
        kept, fc, fs = framed_checkpoint(tr, rows, cols, fmt, lead, pad)
        got, gm, gr, gk = tr.moc_norm_forward(xin, ga, be, eps, keep=kept, out=out.inner)
        near(got, y, bound)
        near(gm, mean, dmean)
        near(gr, rstd, drstd)
        assert out.intact() and fc.intact() and fs.intact()
        # the checkpoint is of y before its rounding: a step of the code next to a border, no more
        kv = ref.values(gk.codes, gk.scales, fmt)
        wide = torch.exp2(gk.scales.cpu().double() - 127).repeat_interleave(32, 1)[:, :cols]
        step = torch.maximum(y.abs() * 2.0 ** -4, wide * 2.0 ** -10) if fmt == "e4m3" else wide / 2
        assert bool(((kv - y).abs() <= step * (1 + 2.0 ** -10) + bound).all())
        alone = tr.moc_norm_forward(xin, ga, be, eps, dtype=dtype)
        assert torch.equal(alone[0], got) and alone[3] is None and torch.equal(alone[1], gm) and torch.equal(alone[2], gr)


@pytest.mark.parametrize("rows,cols", NORM_SIZES + [(1000, 64), (2500, 442), (4999, 33)])
@pytest.mark.parametrize("dtype,held", [("fp32", "tensor"), ("fp16", "tensor"), ("bf16", "tensor"), ("bf16", "e4m3"), ("fp16", "int8")])
def test_norm_backward(tr, rows, cols, dtype, held):
    dtype, eps = TYPES[dtype], 1e-5
    g, x, v, gamma, beta = norm_inputs(rows, cols, dtype, held)
    _, mean, rstd = ref.norm(v, gamma, beta, eps)
    mean, rstd = mean.float(), rstd.float()
    dy, res = (0.3 * normal(g, rows, cols)).to(dtype), normal(g, rows, cols).to(dtype)
    for lead, pad, residual in ((0, 0, None), (1, 5, res)):
        dx, dgamma, dbeta = ref.norm_grad(dy, v, gamma, mean, rstd, residual)
        h = (v - mean.double()[:, None]) * rstd.double()[:, None]
        dh = 4 * U * (v.abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]
        p = (dy.double() * gamma.double()).abs()
        m1, m2 = p.mean(1, keepdim=True), (p * h.abs()).mean(1, keepdim=True)
        part = (cols * 2 * U + 8 * U) * (m1 + h.abs() * m2) + h.abs() * (p * dh).mean(1, keepdim=True) + dh * m2 + 8 * U * p
        bound = rstd.double()[:, None] * part + (4 * U * residual.double().abs() if residual is not None else 0.0)
        if held == "tensor":
            xin = Framed(rows, cols, dtype, lead, pad).of(x)
        else:
            xin, _, _ = framed_checkpoint(tr, rows, cols, held, lead, pad)
            xin.codes.copy_(x[0]), xin.scales.copy_(x[1])
        out = Framed(rows, cols, dtype, lead, pad)
        rin = None if residual is None else Framed(rows, cols, dtype, lead, pad).of(residual)
        din = Framed(rows, cols, dtype, lead, pad).of(dy)
        got, gg, gb = tr.moc_norm_backward(din, xin, gamma.cuda(), mean.cuda(), rstd.cuda(), residual=rin, out=out.inner)
        near(got, dx, bound)
        near(gg, dgamma, (rows * 2 * U + 4 * U) * (dy.double() * h).abs().sum(0) + (dy.double().abs() * dh).sum(0))
        near(gb, dbeta, rows * 2 * U * dy.double().abs().sum(0))
        assert out.intact()
        again, none, nothing = tr.moc_norm_backward(din, xin, gamma.cuda(), mean.cuda(), rstd.cuda(), residual=rin, want_params=False)
        assert torch.equal(again, got) and none is None and nothing is None


def test_norm_without_parameters_and_in_place(tr):
    g = gen("in place")
    x, dy = normal(g, 40, 700).float().cuda(), normal(g, 40, 700).float().cuda()
    one, zero = torch.ones(700, device="cuda"), torch.zeros(700, device="cuda")
    y, mean, rstd, _ = tr.moc_norm_forward(x, one, zero)
    bare = tr.moc_norm_forward(x)
    assert torch.equal(bare[0], y)
    dx = tr.moc_norm_backward(dy, x, one, mean, rstd, residual=x)[0]
    assert torch.equal(tr.moc_norm_backward(dy, x, None, mean, rstd, residual=x)[0], dx)
    over = dy.clone()
    tr.moc_norm_backward(over, x, one, mean, rstd, residual=x, out=over)
    assert torch.equal(over, dx)
    over = x.clone()
    assert torch.equal(tr.moc_norm_forward(over, one, zero, out=over)[0], y) and torch.equal(over, y)


def test_norm_of_no_rows_and_of_what_is_not_finite(tr):
    dx, dg, db = tr.moc_norm_backward(torch.empty(0, 33, device="cuda"), torch.empty(0, 33, device="cuda"), None, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"))
    assert dx.shape == (0, 33) and not dg.any() and not db.any() and dg.shape == (33,)
    assert tr.moc_norm_forward(torch.empty(0, 33, device="cuda"))[0].shape == (0, 33)
    x = torch.randn(4, 300, device="cuda")
    x[1, 7], x[2, 9] = math.nan, math.inf
    y, mean, rstd, kept = tr.moc_norm_forward(x, keep="int8")
    assert y[1].isnan().all() and y[2].isnan().all() and y[0].isfinite().all() and y[3].isfinite().all()
    back = tr.moc_checkpoint_read(kept, torch.float32)
    assert torch.equal(back.isnan(), y.isnan())
    same = torch.full((2, 100), 3.0, device="cuda")   # no variance
    y, mean, rstd, _ = tr.moc_norm_forward(same)
    assert not y.any() and (mean == 3).all() and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)


def test_norm_gradient_is_that_of_differences(tr):
    """dx against central differences of the definition, in 64 bits"""
    g = gen("differences")
    x, gamma, beta, dy = normal(g, 3, 40), 1 + 0.1 * normal(g, 40), 0.1 * normal(g, 40), normal(g, 3, 40)
    f = lambda x, ga, be: (ref.norm(x, ga, be, 1e-5)[0] * dy).sum()   # noqa: E731
    step = 1e-5
    _, mean, rstd = ref.norm(x.float(), gamma.float(), beta.float(), 1e-5)
    dx, dg, db = tr.moc_norm_backward(dy.float().cuda(), x.float().cuda(), gamma.float().cuda(), mean.float().cuda(), rstd.float().cuda())
    for got, i, j in [(dx[r, c], r, c) for r, c in itertools.product(range(3), (0, 1, 17, 39))]:
        e = torch.zeros_like(x)
        e[i, j] = step
        assert abs(float((f(x + e, gamma, beta) - f(x - e, gamma, beta)) / (2 * step)) - float(got)) < 1e-4
    for j in (0, 5, 39):
        e = torch.zeros(40, dtype=torch.float64)
        e[j] = step
        assert abs(float((f(x, gamma + e, beta) - f(x, gamma - e, beta)) / (2 * step)) - float(dg[j])) < 1e-4
        assert abs(float((f(x, gamma, beta + e) - f(x, gamma, beta - e)) / (2 * step)) - float(db[j])) < 1e-4


# ---- linear -------------------------------------------------------------------------------------

# rows, cin, cout: one of each; below, at and above the tiles' sizes; sizes that go through registers;
# few tiles over a long sum (which is cut); enough tiles for the large kernel
LINEAR_SIZES = [(1, 1, 1), (1, 8, 8), (1, 64, 40), (3, 65, 31), (2, 4096, 136), (31, 72, 264), (32, 128, 128), (33, 63, 129), (64, 1000, 72), (127, 200, 513), (130, 442, 100),
                (129, 3000, 128), (256, 64, 256), (257, 136, 520), (300, 1247, 33), (5, 2500, 7), (40, 24, 2056)]
LAYOUTS = [(0, 0), (8, 16), (1, 3)]   # aligned; aligned inside a larger matrix; aligned to the element only


def framed(x, lead, pad):
    return Framed(*x.shape, x.dtype, lead, pad).of(x)


def sum_bound(a, b, n):
    """of a sum of n products"""
    return n * 2 * U * (a.double().abs() @ b.double().abs())


@pytest.mark.parametrize("rows,cin,cout", LINEAR_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act,residual,fmt", [("none", None, None), ("gelu", "same", "e4m3"), ("relu", "fp32", "int8"), ("silu", "same", None)])
def test_linear_forward(tr, rows, cin, cout, dtype, act, residual, fmt):
    dtype = TYPES[dtype]
    g = gen(rows, cin, cout, act)
    x, w, bias = normal(g, rows, cin).to(dtype), normal(g, cout, cin, by=cin ** -0.5).to(dtype), (0.3 * normal(g, cout)).float()
    res = None if residual is None else normal(g, rows, cout).to(dtype if residual == "same" else torch.float32)
    u = x.double() @ w.double().t() + bias.double()
    ub = sum_bound(x, w.t(), cin + 1) + 2 * U * u.abs() + 2 * U * bias.double().abs()
    y = ref.act(u, act) + (0 if res is None else res.double())
    bound = 1.2 * ub + 2.0 ** -18 * u.abs() * (act not in ("none", "relu")) + 2 * U * y.abs()
    first = None
    for lead, pad in LAYOUTS:
        out, kept = Framed(rows, cout, torch.float32 if residual == "fp32" else dtype, lead, pad), None
        if fmt:
            kept, fc, fs = framed_checkpoint(tr, rows, cout, fmt, lead, pad)
        got, k = tr.moc_linear_forward(framed(x, lead, pad), framed(w, lead, pad), bias.cuda() if act != "silu" else bias.to(dtype).cuda(), act=act,
                                       residual=None if res is None else framed(res, lead, pad), keep=kept, out=out.inner)
        if act == "silu":
            b2 = bias.to(dtype).double()
            u2 = x.double() @ w.double().t() + b2
            near(got, ref.act(u2, act) + (0 if res is None else res.double()), bound + 4 * U)
        else:
            near(got, y, bound)
        assert out.intact()
        if fmt:
            assert fc.intact() and fs.intact()
            kv = ref.values(k.codes, k.scales, fmt)
            wide = torch.exp2(k.scales.cpu().double() - 127).repeat_interleave(32, 1)[:, :cout]
            step = torch.maximum(u.abs() * 2.0 ** -4, wide * 2.0 ** -10) if fmt == "e4m3" else wide / 2
            assert bool(((kv - u).abs() <= step * (1 + 2.0 ** -10) + 1.2 * ub).all())
            peak = torch.nn.functional.pad(u.abs(), (0, -cout % 32)).view(rows, -1, 32).amax(2)
            top = torch.exp2(k.scales.cpu().double() - 127) * (448 if fmt == "e4m3" else 127)
            slack = torch.nn.functional.pad(ub, (0, -cout % 32)).view(rows, -1, 32).amax(2)
            assert bool((peak <= top + slack).all()) and bool((2 * (peak + slack) >= top * (1 - 2.0 ** -10)).all())
        if lead == 0:
            first = got
            assert torch.equal(tr.moc_linear_forward(x.cuda(), w.cuda(), bias.cuda() if act != "silu" else bias.to(dtype).cuda(), act=act,
                                                     residual=None if res is None else res.cuda(), dtype=got.dtype)[0], got)   # the checkpoint changes nothing, nor does another run


@pytest.mark.parametrize("rows,cin,cout", LINEAR_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act,held", [("none", None), ("relu", "tensor"), ("gelu", "int8"), ("silu", "e4m3"), ("gelu", "fp32")])
def test_linear_backward_input(tr, rows, cin, cout, dtype, act, held):
    dtype = TYPES[dtype]
    g = gen(rows, cin, cout, act, held)
    dy, w = (0.1 * normal(g, rows, cout)).to(dtype), normal(g, cout, cin, by=cout ** -0.5).to(dtype)
    u = (2 * normal(g, rows, cin)).to(torch.float32 if held == "fp32" else dtype)
    if rows > 2:
        u[1, 0], u[2, -1] = math.nan, 0.0
    pre, v = u, u.double()
    if held in ("int8", "e4m3"):
        pre = ref.keep(u.double(), held, dtype)
        v = ref.values(*pre, held)
    d = dy.double() @ w.double()
    want = d if held is None else d * ref.slope(v, act)
    bound = 1.2 * sum_bound(dy, w, cout) + 2.0 ** -18 * d.abs() * (1 + v.abs().nan_to_num())
    for lead, pad in LAYOUTS:
        if held is None:
            p = None
        elif held in ("int8", "e4m3"):
            p, _, _ = framed_checkpoint(tr, rows, cin, held, lead, pad)
            p.codes.copy_(pre[0]), p.scales.copy_(pre[1])
        else:
            p = framed(pre, lead, pad)
        out = Framed(rows, cin, dtype if act != "silu" else torch.float32, lead, pad)
        got = tr.moc_linear_backward_input(framed(dy, lead, pad), framed(w, lead, pad), act=act, pre=p, out=out.inner)
        near(got, want, bound)
        assert out.intact()


@pytest.mark.parametrize("rows,cin,cout", LINEAR_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("held,narrow", [("tensor", False), ("tensor", True), ("e4m3", False), ("int8", False)])
def test_linear_backward_weight(tr, rows, cin, cout, dtype, held, narrow):
    dtype = TYPES[dtype]
    g = gen(rows, cin, cout, held)
    dy, x = (0.1 * normal(g, rows, cout)).to(dtype), normal(g, rows, cin).to(dtype)
    v = x.double()
    if held != "tensor":
        kept = ref.keep(x.double(), held, dtype)
        v = ref.values(*kept, held).to(dtype).double()
    want = dy.double().t() @ v
    for lead, pad in LAYOUTS:
        if held == "tensor":
            xin = framed(x, lead, pad)
        else:
            xin, _, _ = framed_checkpoint(tr, rows, cin, held, lead, pad)
            xin.codes.copy_(kept[0]), xin.scales.copy_(kept[1])
        out = Framed(cout, cin, dtype if narrow else torch.float32, lead, pad)
        dw, db = tr.moc_linear_backward_weight(framed(dy, lead, pad), xin, out=out.inner)
        near(dw, want, sum_bound(dy.t(), v, rows))
        near(db, dy.double().sum(0), rows * 2 * U * dy.double().abs().sum(0))
        assert out.intact()
        assert tr.moc_linear_backward_weight(framed(dy, lead, pad), xin, want_bias=False)[1] is None


@pytest.mark.parametrize("rows,cin,cout", [(70, 48, 64), (515, 336, 264), (64, 2064, 8), (129, 16, 1032)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_weight_gradient_from_whole_blocks(tr, rows, cin, cout, dtype, fmt):
    """Sizes whose checkpoints are read 16 codes at a time, half blocks at the rows' ends among them."""
    dtype = TYPES[dtype]
    g = gen("blocks", rows, cin, cout, fmt)
    dy, x = (0.1 * normal(g, rows, cout)).to(dtype), (normal(g, rows, cin) * torch.exp(normal(g, cin))).to(dtype)
    x[rows // 2, cin // 2] = math.nan
    codes, scales = ref.keep(x.double(), fmt, dtype)
    v = ref.values(codes, scales, fmt).to(dtype).double()
    for pad in (0, 16):
        kept, _, _ = framed_checkpoint(tr, rows, cin, fmt, 16 - (cin + pad) % 16, pad)
        kept.codes.copy_(codes), kept.scales.copy_(scales)
        out = Framed(cout, cin, torch.float32)
        dw, _ = tr.moc_linear_backward_weight(framed(dy, 0, 0), kept, out=out.inner)
        near(dw, dy.double().t() @ v, sum_bound(dy.t(), v.nan_to_num(), rows))
        assert out.intact()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_every_code_in_a_product(tr, fmt, dtype):
    """one row times 1: the product gives every code's value with every scale that the type can hold"""
    dtype = TYPES[dtype]
    bytes_ = torch.arange(16, 250) if dtype == torch.bfloat16 else torch.arange(103, 136)
    codes = torch.arange(256, dtype=torch.uint8).repeat(len(bytes_))[None]
    scales = bytes_.to(torch.uint8).repeat_interleave(8)[None]
    kept = tr.Checkpoint(codes.cuda(), scales.cuda(), fmt)
    one = torch.zeros(1, 8, dtype=dtype, device="cuda")
    one[0, 3] = 1
    want = tr.moc_checkpoint_read(kept, dtype).float()[0]
    assert torch.equal(want.cpu().nan_to_num(1.5, math.inf, -math.inf), ref.values(codes, scales, fmt)[0].to(dtype).float().nan_to_num(1.5, math.inf, -math.inf))
    dw, _ = tr.moc_linear_backward_weight(one, kept)
    assert torch.equal(dw[3].nan_to_num(1.5, math.inf, -math.inf), want.nan_to_num(1.5, math.inf, -math.inf))
    assert not dw[0].nan_to_num(0, 0, 0).any()


@pytest.mark.parametrize("rows,cin,cout", [(4096, 4096, 3840), (3850, 4160, 4104)])
def test_the_large_tiles(tr, rows, cin, cout):
    """Sizes whose outputs are many tiles of 256 x 256, whole ones and not; sampled rows in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cin, generator=g, device="cuda").bfloat16()
    w = (torch.randn(cout, cin, generator=g, device="cuda") * cin ** -0.5).bfloat16()
    dy = (torch.randn(rows, cout, generator=g, device="cuda") * 0.1).bfloat16()
    some = torch.randint(0, rows, (64,), generator=g, device="cuda")
    some[0], some[1] = 0, rows - 1
    y, kept = tr.moc_linear_forward(x, w, None, act="gelu", keep="int8", dtype=torch.float32)
    u = x[some].double() @ w.double().t()
    ub = cin * 2 * U * (x[some].double().abs() @ w.double().abs().t())
    near(y[some], ref.act(u, "gelu"), (1.2 * ub + 2.0 ** -18 * u.abs()).cpu())
    kv = ref.values(kept.codes[some], kept.scales[some], "int8")
    wide = torch.exp2(kept.scales[some].cpu().double() - 127).repeat_interleave(32, 1)[:, :cout]
    assert bool(((kv - u.cpu()).abs() <= wide / 2 * (1 + 2.0 ** -10) + ub.cpu()).all())
    dx = tr.moc_linear_backward_input(dy, w, dtype=torch.float32)
    near(dx[some], dy[some].double() @ w.double(), (cout * 2 * U * (dy[some].double().abs() @ w.double().abs())).cpu())
    cols = torch.randint(0, cout, (64,), generator=g, device="cuda")
    cols[0], cols[1] = 0, cout - 1
    for fmt in (None, "e4m3", "int8"):
        xin = x if fmt is None else tr.moc_checkpoint_write(x, fmt)
        v = x if fmt is None else tr.moc_checkpoint_read(xin, torch.bfloat16)
        dw, _ = tr.moc_linear_backward_weight(dy, xin)
        part = dy[:, cols].double().t()
        near(dw[cols], part @ v.double(), (rows * 2 * U * (part.abs() @ v.double().abs())).cpu())


def test_whole_numbers_are_exact(tr):
    """Products and sums of small whole numbers have no rounding at all, whatever the tiles and splits."""
    g = gen("whole")
    for rows, cin, cout in ((5, 3000, 40), (200, 520, 300), (1, 4096, 1000), (333, 77, 65)):
        x, w = (torch.randint(-4, 5, s, generator=g).to(torch.bfloat16) for s in ((rows, cin), (cout, cin)))
        dy = torch.randint(-4, 5, (rows, cout), generator=g).to(torch.bfloat16)
        assert torch.equal(tr.moc_linear_forward(x.cuda(), w.cuda(), dtype=torch.float32)[0].cpu(), (x.double() @ w.double().t()).float())
        assert torch.equal(tr.moc_linear_backward_input(dy.cuda(), w.cuda(), dtype=torch.float32).cpu(), (dy.double() @ w.double()).float())
        dw, db = tr.moc_linear_backward_weight(dy.cuda(), x.cuda())
        assert torch.equal(dw.cpu(), (dy.double().t() @ x.double()).float()) and torch.equal(db.cpu(), dy.double().sum(0).float())


def test_linear_of_nothing(tr):
    e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    bias = torch.randn(40, device="cuda")
    y, kept = tr.moc_linear_forward(e(3, 0), e(40, 0), bias, act="relu", keep="int8", dtype=torch.float32)
    assert torch.equal(y, bias.clamp(min=0).repeat(3, 1))
    want = ref.keep(bias.double().repeat(3, 1), "int8", torch.bfloat16)
    assert ref.same_codes(kept.codes, want[0]) and ref.same_codes(kept.scales, want[1])
    assert tr.moc_linear_forward(e(0, 8), e(40, 8), bias)[0].shape == (0, 40)
    assert tr.moc_linear_forward(e(2, 8), e(0, 8))[0].shape == (2, 0)
    assert not tr.moc_linear_backward_input(e(4, 0), e(0, 17)).any()
    dw, db = tr.moc_linear_backward_weight(e(0, 40), e(0, 24))
    assert dw.shape == (40, 24) and not dw.any() and not db.any()
    dw, db = tr.moc_linear_backward_weight(e(5, 40).fill_(1), e(5, 0))
    assert dw.shape == (40, 0) and (db == 5).all()


def test_what_is_not_finite_stays_in_its_row(tr):
    x, w = torch.randn(70, 96, device="cuda").bfloat16(), torch.randn(50, 96, device="cuda").bfloat16()
    clean = tr.moc_linear_forward(x, w, act="gelu")[0]
    x[3, 5], x[60, 95] = math.nan, math.inf
    y, kept = tr.moc_linear_forward(x, w, act="gelu", keep="e4m3")
    good = torch.ones(70, dtype=torch.bool, device="cuda")
    good[3] = good[60] = False
    assert torch.equal(y[good], clean[good]) and y[3].isnan().all() and not y[60][w[:, 95] > 0].isfinite().any()
    back = tr.moc_checkpoint_read(kept, torch.float32)
    assert back[~good].isnan().all() and back[good].isfinite().all()


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_linear_gradients_are_those_of_differences(tr, act):
    """f(u, w) = sum of dy * (act(u) w^T), differences of the definition in 64 bits."""
    g = gen("linear differences", act)
    u, w, dy = (normal(g, *s).to(torch.float16) for s in ((4, 24), (16, 24), (4, 16)))
    h = ref.act(u.double(), act).to(torch.float16)
    du = tr.moc_linear_backward_input(dy.cuda(), w.cuda(), act=act, pre=u.cuda(), dtype=torch.float32).cpu()
    dw, db = tr.moc_linear_backward_weight(dy.cuda(), h.cuda())
    step = 1e-6
    f = lambda u: (dy.double() * (ref.act(u, act) @ w.double().t())).sum()   # noqa: E731
    for i, j in itertools.product((0, 3), (0, 7, 23)):
        e = torch.zeros(4, 24, dtype=torch.float64)
        e[i, j] = step
        assert abs(float((f(u.double() + e) - f(u.double() - e)) / (2 * step)) - float(du[i, j])) < 1e-3
    f = lambda w, b: (dy.double() * (h.double() @ w.t() + b)).sum()   # noqa: E731
    for i, j in itertools.product((0, 15), (0, 23)):
        e, b = torch.zeros(16, 24, dtype=torch.float64), torch.zeros(16, dtype=torch.float64)
        e[i, j] = step
        assert abs(float((f(w.double() + e, b) - f(w.double() - e, b)) / (2 * step)) - float(dw.cpu()[i, j])) < 1e-3
        b[i] = step
        assert abs(float((f(w.double(), b) - f(w.double(), -b)) / (2 * step)) - float(db.cpu()[i])) < 1e-3


def test_slope_at_the_ends(tr):
    """the activations' derivatives at arguments whose squares overflow, at 0 and at what is not finite"""
    u = torch.tensor([[0.0, -0.0, 3e38, -3e38, 1e20, -1e20, 17.0, -17.0, 1e-30, math.nan]], dtype=torch.float32)
    dy, w = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda"), torch.ones(1, 10, dtype=torch.bfloat16, device="cuda")
    for act, want in (("relu", [0, 0, 1, 0, 1, 0, 1, 0, 1]), ("gelu", [0.5, 0.5, 1, 0, 1, 0, 1, 0, 0.5]), ("silu", [0.5, 0.5, 1, 0, 1, 0, 1, 0, 0.5])):
        got = tr.moc_linear_backward_input(dy, w, act=act, pre=u.cuda(), dtype=torch.float32).cpu()[0]
        assert torch.allclose(got[:9], torch.tensor(want, dtype=torch.float32), rtol=2.0 ** -18, atol=2e-6) and got[9].isnan()


# ---- as a step of a program ---------------------------------------------------------------------

def block(tr, x, p, dy, work=None, stream=None):
    """A residual block forward and backward, kept in 8 bits."""
    n, mean, rstd, kept = tr.moc_norm_forward(x, p["g"], p["b"], keep="int8", stream=stream)
    h, u = tr.moc_linear_forward(n, p["w1"], p["b1"], act="gelu", keep="e4m3", stream=stream)
    y, _ = tr.moc_linear_forward(h, p["w2"], p["b2"], residual=x, stream=stream)
    du = tr.moc_linear_backward_input(dy, p["w2"], act="gelu", pre=u, stream=stream)
    dw2, db2 = tr.moc_linear_backward_weight(dy, tr.moc_checkpoint_read(u, x.dtype, act="gelu", stream=stream), stream=stream)
    dn = tr.moc_linear_backward_input(du, p["w1"], stream=stream)
    dw1, db1 = tr.moc_linear_backward_weight(du, kept, stream=stream)
    dx, dg, db = tr.moc_norm_backward(dn, x, p["g"], mean, rstd, residual=dy, stream=stream)
    return [y, dx, dg, db, dw1, db1, dw2, db2]


def block_inputs(seed, rows=260, width=256, inner=512):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, by=1.0: (torch.randn(*s, generator=g, device="cuda") * by)   # noqa: E731
    p = dict(g=1 + r(width, by=0.1), b=r(width, by=0.1), w1=r(inner, width, by=width ** -0.5).bfloat16(), b1=r(inner, by=0.1), w2=r(width, inner, by=inner ** -0.5).bfloat16(),
             b2=r(width, by=0.1))
    return r(rows, width).bfloat16(), p, r(rows, width, by=0.02).bfloat16()


def test_a_block_in_a_graph(tr):
    x, p, dy = block_inputs(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(tr, x, p, dy)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(tr, x, p, dy)
    for seed in (2, 3, 4):
        x2, _, dy2 = block_inputs(seed)
        x.copy_(x2), dy.copy_(dy2)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, block(tr, x, p, dy)):
            assert torch.equal(got, want)
        torch.cuda.synchronize()


def test_a_block_on_another_stream_gives_the_same_bits(tr):
    x, p, dy = block_inputs(5)
    want = block(tr, x, p, dy)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = block(tr, x, p, dy, stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_refusals_with_tensors(tr):
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    x, w, v = bf(4, 64), bf(32, 64), torch.zeros(64, device="cuda")
    k = tr.empty_checkpoint(4, 64, "int8", "cuda")
    for call in (lambda: tr.moc_linear_forward(x, bf(32, 65)), lambda: tr.moc_linear_forward(x.t(), w), lambda: tr.moc_linear_forward(x.cpu(), w),
                 lambda: tr.moc_linear_forward(x, w, act="tanh"), lambda: tr.moc_linear_forward(x, w, bias=v), lambda: tr.moc_linear_forward(x, w, residual=bf(4, 33)),
                 lambda: tr.moc_linear_forward(x, w, out=bf(4, 31)), lambda: tr.moc_linear_forward(x, w, keep="e5m2"), lambda: tr.moc_linear_forward(x[0], w),
                 lambda: tr.moc_linear_backward_input(x, bf(32, 64)), lambda: tr.moc_linear_backward_weight(x, bf(5, 64)), lambda: tr.moc_checkpoint_read(x, torch.float32),
                 lambda: tr.moc_checkpoint_write(x.double()), lambda: tr.moc_checkpoint_write(x.expand(4, 64).as_strided((4, 64), (0, 1))),
                 lambda: tr.moc_norm_forward(x, v[:3]), lambda: tr.moc_norm_backward(x, x, v, v[:4], v[:3]), lambda: tr.moc_norm_backward(x, x, v, v[:4].half(), v[:4]),
                 lambda: tr.moc_norm_forward(x, v, v.half()), lambda: tr.moc_checkpoint_read(tr.Checkpoint(k.codes, k.scales[:, :1], "int8"), torch.float32)):
        with pytest.raises(ValueError):
            call()
    from paper_2304_14463_amd.moccasin import MoccasinError
    for call in (lambda: tr.moc_linear_forward(x.float(), w.float()), lambda: tr.moc_linear_forward(x, w.half()), lambda: tr.moc_linear_backward_input(x, bf(64, 8), act="relu"),
                 lambda: tr.moc_linear_forward(x, w, dtype=torch.float16), lambda: tr.moc_linear_forward(x, w, residual=bf(4, 32).half()),
                 lambda: tr.moc_linear_backward_weight(x, x.half()), lambda: tr.moc_norm_forward(x, eps=-1.0), lambda: tr.moc_norm_forward(bf(4, 0)),
                 lambda: tr.moc_linear_forward(bf(1, 8192), bf(64, 8192), work=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(MoccasinError) as err:
            call()
        assert err.value.code == -1
