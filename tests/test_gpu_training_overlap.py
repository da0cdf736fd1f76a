"""Outputs in the memory of an input: refused where a result would be written over what is still read, right where it may be."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    from paper_2304_14463_amd import training
    training.lib()
    return training


def bf(*s):
    return torch.randn(*s, device="cuda").bfloat16()


def test_refused(tr):
    x, w, dy = bf(64, 64), bf(64, 64), bf(64, 64)
    mean, rstd = torch.zeros(64, device="cuda"), torch.ones(64, device="cuda")
    room = bf(65, 64)
    up, down = room[:64], room[1:]
    k = tr.moc_checkpoint_write(x, "int8")
    over = lambda t: tr.Checkpoint(t.view(torch.uint8)[:, :64], k.scales, "int8")   # noqa: E731
    before = [t.clone() for t in (x, w, dy, room, k.codes, k.scales)]
    for call in (lambda: tr.moc_linear_forward(x, w, out=x), lambda: tr.moc_linear_forward(x, w, out=w), lambda: tr.moc_linear_forward(x, w, residual=up, out=down),
                 lambda: tr.moc_linear_forward(x, w, keep=over(x)), lambda: tr.moc_linear_forward(x, w, keep=over(w)), lambda: tr.moc_linear_forward(x, w, residual=up, keep=over(up)),
                 lambda: tr.moc_linear_forward(x, w, out=up, keep=over(up)), lambda: tr.moc_linear_backward_input(dy, w, out=dy), lambda: tr.moc_linear_backward_input(dy, w, out=w),
                 lambda: tr.moc_linear_backward_input(dy, w, act="relu", pre=up, out=down), lambda: tr.moc_linear_backward_weight(dy, x, out=dy),
                 lambda: tr.moc_linear_backward_weight(dy, x, out=x), lambda: tr.moc_linear_backward_weight(dy, over(x), out=x), lambda: tr.moc_checkpoint_write(x, out=over(x)),
                 lambda: tr.moc_checkpoint_read(over(x), torch.bfloat16, out=x), lambda: tr.moc_norm_forward(up, out=down), lambda: tr.moc_norm_forward(x, keep=over(x)),
                 lambda: tr.moc_norm_forward(x, keep=over(up), out=up), lambda: tr.moc_norm_forward(over(x), out=x), lambda: tr.moc_norm_forward(k, keep=k),
                 lambda: tr.moc_norm_backward(up, x, None, mean, rstd, out=down), lambda: tr.moc_norm_backward(dy, up, None, mean, rstd, out=down),
                 lambda: tr.moc_norm_backward(dy, x, None, mean, rstd, residual=up, out=down), lambda: tr.moc_norm_backward(dy, over(x), None, mean, rstd, out=x),
                 lambda: tr.moc_linear_backward_input(dy, w, act="relu", pre=over(x), out=x)):
        with pytest.raises(ValueError, match="shares memory"):
            call()
    torch.cuda.synchronize()
    for t, b in zip((x, w, dy, room, k.codes, k.scales), before):
        assert torch.equal(t.view(torch.uint8), b.view(torch.uint8))


def test_parts_of_one_matrix_are_apart(tr):
    """Columns beside each other, and rows, of a fused buffer."""
    x, w = bf(100, 64), bf(48, 64)
    room = torch.zeros(100, 64 + 48 + 48, dtype=torch.bfloat16, device="cuda")
    room[:, :64] = x
    want, _ = tr.moc_linear_forward(x, w, act="relu")
    got, _ = tr.moc_linear_forward(room[:, :64], w, act="relu", out=room[:, 64:112])
    assert torch.equal(got, want) and not room[:, 112:].any()
    y = tr.moc_norm_forward(room[:, 64:112], out=room[:, 112:])[0]
    assert torch.equal(y, tr.moc_norm_forward(want)[0])
    rows = bf(200, 64)
    want = tr.moc_norm_forward(rows[:100].clone())[0]
    assert torch.equal(tr.moc_norm_forward(rows[:100], out=rows[100:])[0], want)


@pytest.mark.parametrize("rows,cols", [(3000, 64), (3001, 441), (2000, 1000), (700, 1247), (700, 4096), (600, 5001), (300, 9001), (300, 20003)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_gradient_in_the_memory_of_x(tr, rows, cols, dtype):
    x, dy, residual = (torch.randn(rows, cols, device="cuda").to(dtype) for _ in range(3))
    gamma = torch.randn(cols, device="cuda")
    _, mean, rstd, _ = tr.moc_norm_forward(x)
    want = tr.moc_norm_backward(dy, x, gamma, mean, rstd, residual=residual)
    over = x.clone()
    got = tr.moc_norm_backward(dy, over, gamma, mean, rstd, residual=residual, out=over)
    assert got[0] is over and all(torch.equal(a, b) for a, b in zip(got, want))


# few tiles, a cut sum, ragged ones, straight into LDS in 128 and 256
@pytest.mark.parametrize("rows,cin,cout", [(65, 72, 96), (3, 64, 8192), (2501, 3005, 500), (700, 5, 900), (1536, 2032, 256), (200, 4112, 4104), (8200, 1536, 264), (1032, 2032, 16384)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_input_gradient_in_the_memory_of_the_argument(tr, rows, cin, cout, out):
    dy, w = bf(rows, cout), bf(cout, cin)
    pre = torch.randn(rows, cin, device="cuda").to(out)
    want = tr.moc_linear_backward_input(dy, w, act="gelu", pre=pre, dtype=out)
    over = pre.clone()
    assert torch.equal(tr.moc_linear_backward_input(dy, w, act="gelu", pre=over, out=over), want)
