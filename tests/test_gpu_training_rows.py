"""Layer norm over so many rows that every workgroup goes over several, the last time not all of them, for each shape that the kernels come in.

A row's result does not depend on the rows beside it: the whole call gives the bits of calls of 200 rows, of which a
workgroup has one turn.  The backward pass gets mean 0, rstd 1 and whole numbers, which no order of sums rounds: dgamma and
dbeta are exact; dx = rstd (p - mean(p) - h mean(p h)) + residual has ten roundings at most, each half a step of the largest
of its terms, and dx's own, of a subnormal value half of the smallest one."""
import pytest
import torch

from training_reference import Framed, half_step

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
PIECE = 200
# rows, cols: a wave a row with one run and with two, 256 threads with one and two, 512, 1024, and rows that no registers hold
SIZES = [(25001, 64), (25003, 441), (20001, 1000), (17000, 1024), (5001, 1247), (5000, 2048), (3101, 4095), (1601, 5000), (801, 16384), (790, 9001), (601, 16392), (600, 20003)]
HELD = ["bf16", "fp16", "fp32", "e4m3", "int8"]
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.bfloat16, "int8": torch.float16}


@pytest.fixture(scope="module")
def tr():
    from paper_2304_14463_amd import training
    training.lib()
    return training


def part(tr, x, at):
    return tr.Checkpoint(x.codes[at], x.scales[at], x.fmt) if isinstance(x, tr.Checkpoint) else x[at]


def pieces(rows):
    return [slice(i, min(i + PIECE, rows)) for i in range(0, rows, PIECE)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("held", HELD)
def test_forward(tr, rows, cols, held):
    dtype = DTYPES[held]
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda")) + torch.randn(rows, 1, generator=g, device="cuda")).to(dtype)
    if held in ("e4m3", "int8"):
        x = tr.moc_checkpoint_write(x, held)
    gamma, beta = (torch.randn(cols, generator=g, device="cuda") for _ in range(2))
    keep = "e4m3" if held == "int8" else "int8"
    out = Framed(rows, cols, dtype, 0, 8)
    y, mean, rstd, kept = tr.moc_norm_forward(x, gamma, beta, keep=keep, out=out.inner)
    assert out.intact()
    for at in pieces(rows):
        y2, mean2, rstd2, kept2 = tr.moc_norm_forward(part(tr, x, at), gamma, beta, keep=keep, dtype=dtype)
        assert torch.equal(y[at], y2) and torch.equal(mean[at], mean2) and torch.equal(rstd[at], rstd2)
        assert torch.equal(kept.codes[at], kept2.codes) and torch.equal(kept.scales[at], kept2.scales)
    v = tr.moc_checkpoint_read(x, torch.float32) if isinstance(x, tr.Checkpoint) else x
    want = v.double().mean(1)
    assert bool(((mean.double() - want).abs() <= (cols + 2) * 2 * U * v.double().abs().mean(1)).all())
    if not isinstance(x, tr.Checkpoint):
        over = x.clone()
        assert torch.equal(tr.moc_norm_forward(over, gamma, beta, out=over)[0], y) and torch.equal(over, y)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("held", HELD)
def test_backward(tr, rows, cols, held):
    dtype = DTYPES[held]
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    whole = lambda most, *s: torch.randint(-most, most + 1, s, generator=g, device="cuda").float()   # noqa: E731
    values, dy, residual = whole(4, rows, cols).to(dtype), whole(2, rows, cols).to(dtype), whole(4, rows, cols).to(dtype)
    x = tr.moc_checkpoint_write(values, held) if held in ("e4m3", "int8") else values   # exact
    gamma, mean, rstd = 1 + whole(4, cols) / 8, torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    out = Framed(rows, cols, dtype, 0, 8)
    dx, dgamma, dbeta = tr.moc_norm_backward(dy, x, gamma, mean, rstd, residual=residual, out=out.inner)
    assert out.intact()
    h, d = values.double(), dy.double()
    assert torch.equal(dgamma, (d * h).sum(0).float()) and torch.equal(dbeta, d.sum(0).float())
    p = d * gamma.double()
    a, b = p.mean(1, keepdim=True), (p * h).mean(1, keepdim=True)
    want = p - a - h * b + residual.double()
    size = p.abs() + a.abs() + (h * b).abs() + residual.double().abs()
    assert bool(((dx.double() - want).abs() <= 10 * U * size + half_step(dtype) * (want.abs() + 10 * U * size + torch.finfo(dtype).smallest_normal)).all())
    for at in pieces(rows):
        again, _, _ = tr.moc_norm_backward(dy[at], part(tr, x, at), gamma, mean[at], rstd[at], residual=residual[at])
        assert torch.equal(dx[at], again)
    for which in ("dy", "residual"):   # in the memory of an input
        ins = dict(dy=dy.clone(), residual=residual.clone())
        over, dgamma2, dbeta2 = tr.moc_norm_backward(ins["dy"], x, gamma, mean, rstd, residual=ins["residual"], out=ins[which])
        assert torch.equal(over, dx) and torch.equal(dgamma2, dgamma) and torch.equal(dbeta2, dbeta)
