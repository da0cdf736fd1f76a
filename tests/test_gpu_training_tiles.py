"""Products in every kind of tile, with the sum whole and cut: small whole numbers, which no order of sums rounds."""
import pytest
import torch

from training_reference import TYPES, Framed

pytestmark = pytest.mark.gpu

# 128 x 128 and 256 x 256 straight into LDS, their last tiles in part; 256 x 256 through registers, whole sums and cut ones, by
# rows and columns of every alignment; 64 x 64; operands with rows of fewer than eight values on either side
SIZES = [(2050, 2056, 2064), (1800, 4104, 1800), (700, 8200, 2000), (3001, 1500, 3005), (2501, 3005, 2509), (4000, 1001, 4001), (3000, 6001, 1501), (1400, 1400, 1400), (700, 3, 900),
         (900, 700, 3), (3, 700, 900), (2600, 5, 2600), (65, 7, 7), (64, 9, 8), (1000, 70, 9)]


def whole(g, *shape, dtype):
    return torch.randint(-4, 5, shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("rows,cin,cout", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_whole_numbers_in_every_tile(rows, cin, cout, dtype):
    from paper_2304_14463_amd import training as tr
    dtype = TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(rows + cin + cout)
    x, w, dy, bias = whole(g, rows, cin, dtype=dtype), whole(g, cout, cin, dtype=dtype), whole(g, rows, cout, dtype=dtype), whole(g, cout, dtype=torch.float32)
    out = Framed(rows, cout, torch.float32, 4, 8)
    tr.moc_linear_forward(x, w, bias, out=out.inner)
    assert torch.equal(out.inner, (x.double() @ w.double().t() + bias.double()).float()) and out.intact()
    out = Framed(rows, cin, torch.float32, 1, 3)
    tr.moc_linear_backward_input(dy, w, out=out.inner)
    assert torch.equal(out.inner, (dy.double() @ w.double()).float()) and out.intact()
    want, sums = (dy.double().t() @ x.double()).float(), dy.double().sum(0).float()
    for xin in (x, tr.moc_checkpoint_write(x, "int8"), tr.moc_checkpoint_write(x, "e4m3")):
        out = Framed(cout, cin, torch.float32, 0, 1)
        _, db = tr.moc_linear_backward_weight(dy, xin, out=out.inner)
        assert torch.equal(out.inner, want) and torch.equal(db, sums) and out.intact()


@pytest.mark.parametrize("rows,cin,cout", [(1400, 1400, 1400), (2501, 3005, 2509), (2050, 2056, 2064), (700, 3, 900)])
def test_what_lies_beside_an_operand_is_not_used(rows, cin, cout):
    """Operands inside larger matrices of NaN."""
    from paper_2304_14463_amd import training as tr
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, w, dy = (whole(g, *s, dtype=torch.bfloat16) for s in ((rows, cin), (cout, cin), (rows, cout)))

    def inside(v):
        room = torch.full((v.shape[0] + 2, v.shape[1] + 16), float("nan"), dtype=v.dtype, device="cuda")
        room[1:-1, 8:-8] = v
        return room[1:-1, 8:-8]

    a, b, d = inside(x), inside(w), inside(dy)
    assert torch.equal(tr.moc_linear_forward(a, b, dtype=torch.float32)[0], (x.double() @ w.double().t()).float())
    assert torch.equal(tr.moc_linear_backward_input(d, b, dtype=torch.float32), (dy.double() @ w.double()).float())
    dw, db = tr.moc_linear_backward_weight(d, a)
    assert torch.equal(dw, (dy.double().t() @ x.double()).float()) and torch.equal(db, dy.double().sum(0).float())
    kept = tr.moc_checkpoint_write(a, "int8")
    assert torch.equal(tr.moc_linear_backward_weight(d, kept)[0], dw)


@pytest.mark.parametrize("cols", [9, 31, 33, 519, 1001, 1025, 1033, 2047, 2049, 4095, 4097, 8191, 8193, 16383])
@pytest.mark.parametrize("held", ["bf16", "fp32", "e4m3", "int8"])
def test_rows_of_norms_that_end_in_a_run(cols, held):
    """dbeta is a sum of whole numbers; rows of a constant have no difference from their mean, whatever lies beside them."""
    from paper_2304_14463_amd import training as tr
    rows, dtype = 5, torch.float32 if held == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(cols)
    room = torch.full((rows, cols + 8), float("nan"), dtype=dtype, device="cuda")
    x, dy = room[:, :cols], whole(g, rows, cols, dtype=dtype)
    x.copy_(torch.tensor([[1.0], [-2.0], [0.5], [4.0], [0.0]], device="cuda").expand(rows, cols))
    xin = x if held in ("bf16", "fp32") else tr.moc_checkpoint_write(x, held)
    beta = whole(g, cols, dtype=torch.float32)
    y, mean, rstd, kept = tr.moc_norm_forward(xin, None, beta, keep="int8", dtype=torch.float32)
    assert torch.equal(mean, x[:, 0].float()) and torch.equal(y, beta.expand(rows, cols))
    assert torch.equal(tr.moc_checkpoint_read(kept, torch.float32), y)
    dx, dgamma, dbeta = tr.moc_norm_backward(dy, xin, None, mean, rstd, residual=dy)
    assert torch.equal(dbeta, dy.double().sum(0).float()) and not dgamma.any() and dx.isfinite().all()
    # dx = rstd (dy - mean(dy)) + dy, rstd = 1 / sqrt(1e-5): four roundings, the sum's n, and dx's own
    want = (dy.double() - dy.double().mean(1, keepdim=True)) * rstd.double()[:, None] + dy.double()
    size = (dy.double().abs() + dy.double().abs().mean(1, keepdim=True)) * rstd.double()[:, None] + dy.double().abs()
    assert bool(((dx.double() - want).abs() <= (6 + cols) * 2.0 ** -24 * size + torch.finfo(dtype).eps / 2 * (want.abs() + size * 2.0 ** -8)).all())
