"""The training operators at the limits that their header gives."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [None, "int8"])
def test_weight_gradient_of_the_most_rows(fmt):
    """The sum over rows is cut, and the last part ends next to 2^31: rows that are not zero at every part's ends, whole numbers."""
    from paper_2304_14463_amd import training as tr
    rows = 2147483136
    p = tr.moc_linear_parts("backward_weight", rows, 1, 1)
    assert p.parts > 1
    at = [r for i in range(p.parts) for r in (i * p.terms, i * p.terms + p.terms // 2, min((i + 1) * p.terms, rows) - 1)]
    dy, x = (torch.zeros(rows, 1, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for n, r in enumerate(at):
        dy[r] = 1 + n % 5
        x[r] = 2 + n % 3
    if fmt:
        x = tr.Checkpoint(x[:, 0].to(torch.int8).view(torch.uint8)[:, None], torch.full((rows, 1), 127, dtype=torch.uint8, device="cuda"), fmt)
    dw, db = tr.moc_linear_backward_weight(dy, x)
    assert float(dw) == sum((1 + n % 5) * (2 + n % 3) for n in range(len(at))) and float(db) == sum(1 + n % 5 for n in range(len(at)))
