"""The products whose operands go straight into LDS: from checkpoints (codes of NaN, scales whose values overflow on their way, rows that end
in half a block), with a residual, through a derivative, and with the sum cut.  Which kernel a size takes is asked for, so that a
test stays with the kernel it is for.

Small whole numbers, powers of two of them: no order of sums rounds, and results are equal bit for bit.  Through gelu and silu
the bound is that of their exp2 and reciprocal, 1 ulp each with an argument off by 2^-22 of itself: 2^-18 of the argument (of the
gradient: 1 and more), and half a step of the output's type."""
import math

import pytest
import torch

import training_reference as ref
from training_reference import TYPES, Framed, half_step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    from paper_2304_14463_amd import training
    training.lib()
    return training


def whole(g, *shape, dtype, most=4):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dtype)


def seeded(*key):
    return torch.Generator(device="cuda").manual_seed(sum((i + 1) * int(v) for i, v in enumerate(key)))


def same(got, want):
    """equal, NaN in the same places"""
    return got.shape == want.shape and torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.5, math.inf, -math.inf), want.nan_to_num(0.5, math.inf, -math.inf))


def planned(tr, product, sizes, tile, parts):
    p = tr.moc_linear_parts(product, *sizes)
    assert p.direct and p.tile == tile and (p.parts > 1) == parts, p


# rows, cin, cout, tile, whether the sum is cut: whole tiles and not, whole blocks and halves, odd and even steps, a step in part
WEIGHT_SIZES = [(200, 2032, 2048, 128, False), (203, 2032, 2040, 128, False), (512, 2048, 2048, 128, False), (264, 2032, 4104, 256, False), (333, 4112, 2064, 256, False),
                (64, 2032, 4104, 256, False), (8200, 2032, 1536, 256, True), (8203, 2064, 1544, 256, True)]


@pytest.mark.parametrize("rows,cin,cout,tile,parts", WEIGHT_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_weight_gradient_from_a_checkpoint(tr, rows, cin, cout, tile, parts, dtype, fmt):
    planned(tr, "backward_weight", (rows, cin, cout), tile, parts)
    dtype = TYPES[dtype]
    g = seeded(rows, cin, cout)
    v, dy = whole(g, rows, cin, dtype=torch.float32), whole(g, rows, cout, dtype=dtype, most=2)
    blocks = -(-cin // 32)
    scales = torch.randint(126, 129, (rows, blocks), generator=g, device="cuda").to(torch.uint8)
    codes = v.to(torch.float8_e4m3fn).view(torch.uint8) if fmt == "e4m3" else v.to(torch.int8).view(torch.uint8)
    # codes of NaN: in the first row, in the last block of the last one
    nan = 0x7F if fmt == "e4m3" else 0x80
    codes[0, 5] = codes[rows - 1, cin - 1] = codes[rows // 2, 40] = nan
    # values up to 2^123, whose row is the only one that counts for column 3 of dy
    codes[7, 64:96] = codes[7, 64:96].where(codes[7, 64:96] != nan, 0)
    scales[7, 2] = 248
    dy[:, 3] = 0
    dy[7] = 0
    dy[7, 3] = 1
    kept = tr.Checkpoint(codes, scales, fmt)
    x = ref.values(codes, scales, fmt).to(dtype).double().cuda()   # in float16 2^123 is infinite
    want = (dy.double().t() @ x).float()
    assert int(want.isnan().any(0).sum()) >= 3 and bool((want[3, 64:96].abs() >= 2.0 ** 121).any())
    out = Framed(cout, cin, torch.float32, 0, 8)
    _, db = tr.moc_linear_backward_weight(dy, kept, out=out.inner)
    assert same(out.inner, want) and out.intact() and torch.equal(db, dy.double().sum(0).float())
    narrow, _ = tr.moc_linear_backward_weight(dy, kept, dtype=dtype)
    assert same(narrow, want.to(dtype))
    # the same codes inside larger matrices, aligned all the same
    fc, fs = Framed(rows, cin, torch.uint8, 16 - (cin + 16) % 16, 16), Framed(rows, blocks, torch.uint8, 1, 3)
    again, _ = tr.moc_linear_backward_weight(dy, tr.Checkpoint(fc.of(codes), fs.of(scales), fmt))
    assert same(again, want)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,cin,cout,tile", [(200, 2048, 2048, 128), (264, 2048, 4104, 256)])
def test_every_code_and_scale_straight_into_lds(tr, fmt, dtype, rows, cin, cout, tile):
    """Each row of dy is 1 in a place of its own: the product gives the values of every code with every scale."""
    planned(tr, "backward_weight", (rows, cin, cout), tile, False)
    dtype = TYPES[dtype]
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(rows, cin // 256)
    nan = (codes == 0x80) if fmt == "int8" else (codes & 0x7F) == 0x7F
    codes = codes.masked_fill(nan, 0)   # it would be all of a column
    # scales with which the type holds every code's value
    first, last = (103, 134) if dtype == torch.float16 else (16, 248 if fmt == "int8" else 246)
    scales = (first + torch.arange(rows * (cin // 32), device="cuda").view(rows, -1) % (last - first + 1)).to(torch.uint8)
    kept = tr.Checkpoint(codes, scales, fmt)
    dy = torch.zeros(rows, cout, dtype=dtype, device="cuda")
    at = (torch.arange(rows, device="cuda") * 13) % cout
    dy[torch.arange(rows, device="cuda"), at] = 1
    x = ref.values(codes, scales, fmt).to(dtype).cuda()
    dw, _ = tr.moc_linear_backward_weight(dy, kept)
    assert bool(x.isfinite().all()) and torch.equal(dw[at], x.float())


# rows, cin, cout
FORWARD_SIZES = [(1536, 256, 2056, 128, False), (200, 16392, 1032, 128, True), (8200, 264, 1536, 256, False), (1032, 16384, 2032, 256, True)]


@pytest.mark.parametrize("rows,cin,cout,tile,parts", FORWARD_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("residual,fmt", [("same", "int8"), ("fp32", "e4m3"), (None, None)])
def test_forward_with_a_residual(tr, rows, cin, cout, tile, parts, dtype, residual, fmt):
    planned(tr, "forward", (rows, cin, cout), tile, parts)
    dtype = TYPES[dtype]
    g = seeded(rows, cin, cout)
    x, w = whole(g, rows, cin, dtype=dtype, most=2), whole(g, cout, cin, dtype=dtype, most=2)
    bias = whole(g, cout, dtype=torch.float32)
    res = None if residual is None else whole(g, rows, cout, dtype=dtype if residual == "same" else torch.float32)
    u = x.double() @ w.double().t() + bias.double()
    add = 0.0 if res is None else res.double()
    for act, y in (("none", u), ("relu", u.clamp(min=0))):
        out = Framed(rows, cout, torch.float32, 4, 8)
        _, kept = tr.moc_linear_forward(x, w, bias, act=act, residual=res, keep=fmt, out=out.inner)
        assert torch.equal(out.inner, (y + add).float()) and out.intact()
        if fmt:
            k = tr.moc_checkpoint_write(u.float(), fmt)
            assert torch.equal(kept.codes, k.codes) and torch.equal(kept.scales, k.scales)
        narrow, _ = tr.moc_linear_forward(x, w, bias, act=act, residual=res)
        assert torch.equal(narrow, (y + add).to(dtype))
    if residual == "same":   # in the residual's own memory
        over = res.clone()
        tr.moc_linear_forward(x, w, bias, residual=over, out=over)
        assert torch.equal(over, (u + add).to(dtype))
    w = w / 16   # arguments that the activations bend
    u = x.double() @ w.double().t() + bias.double()
    for act in ("gelu", "silu"):
        y = tr.moc_linear_forward(x, w, bias, act=act, residual=res, dtype=torch.float32)[0].double()
        want = ref.act(u, act) + add
        assert bool(((y - want).abs() <= 2.0 ** -18 * u.abs() + half_step(torch.float32) * 2 * want.abs() + 2.0 ** -100).all())


BACKWARD_SIZES = [(1536, 2032, 256, 128, False), (200, 4112, 4104, 128, True), (8200, 1536, 264, 256, False), (1032, 2032, 16384, 256, True)]


@pytest.mark.parametrize("rows,cin,cout,tile,parts", BACKWARD_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("held", ["same", "fp32", "e4m3", "int8"])
def test_input_gradient_through_a_derivative(tr, rows, cin, cout, tile, parts, dtype, held):
    planned(tr, "backward_input", (rows, cin, cout), tile, parts)
    dtype = TYPES[dtype]
    g = seeded(rows, cin, cout)
    dy, w = whole(g, rows, cout, dtype=dtype, most=2), whole(g, cout, cin, dtype=dtype, most=2)
    v = whole(g, rows, cin, dtype=torch.float32) / 2
    v[1, 0] = v[rows - 1, cin - 1] = math.nan
    pre = v.to(dtype) if held == "same" else v if held == "fp32" else tr.moc_checkpoint_write(v, held)   # halves up to 2: exact in all
    d = dy.double() @ w.double()
    out = Framed(rows, cin, torch.float32, 4, 8)
    tr.moc_linear_backward_input(dy, w, act="relu", pre=pre, out=out.inner)
    assert same(out.inner, torch.where(v.isnan(), v, torch.where(v > 0, d.float(), 0.0))) and out.intact()
    for act in ("gelu", "silu"):
        got = tr.moc_linear_backward_input(dy, w, act=act, pre=pre, dtype=torch.float32).double()
        want = d * ref.slope(v.double(), act)
        assert torch.equal(got.isnan(), v.isnan())
        off = (got - want).abs() - 2.0 ** -18 * d.abs() * (1 + v.double().abs()) - 2 * half_step(torch.float32) * want.abs()
        assert bool((off.nan_to_num(0.0) <= 0).all())
