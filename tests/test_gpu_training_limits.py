"""The training operators at the limits that their header gives."""
import math

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


@pytest.mark.parametrize("call,rows,cin,cout,needs", [("weight", 512, 2048, 2048, 4 * 2048 * 2), ("weight", 300, 72, 40, 0), ("weight", 5000, 40, 72, 1), ("forward", 1, 8192, 64, 1), ("input", 1, 64, 8192, 1)])
def test_refused_for_its_workspace_nothing_is_queued(call, rows, cin, cout, needs):
    """A workspace that the product, or the bias's gradient beside it, has no room in: the outputs stay as they are."""
    from paper_2304_14463_amd import training as tr
    from paper_2304_14463_amd.moccasin import MoccasinError
    x, w, dy = (torch.ones(*s, dtype=torch.bfloat16, device="cuda") for s in ((rows, cin), (cout, cin), (rows, cout)))
    out = torch.full({"weight": (cout, cin), "forward": (rows, cout), "input": (rows, cin)}[call], math.nan, dtype=torch.float32, device="cuda")
    small = torch.empty(max(16, needs - 16), dtype=torch.uint8, device="cuda")

    def run(work):
        if call == "weight":
            return tr.moc_linear_backward_weight(dy, x, out=out, work=work)
        return tr.moc_linear_forward(x, w, out=out, work=work) if call == "forward" else tr.moc_linear_backward_input(dy, w, out=out, work=work)
    if call == "weight" and rows == 512:   # the product needs none of it: only the bias's gradient does
        p = tr.moc_linear_parts("backward_weight", rows, cin, cout)
        assert p.parts == 1 and p.tile > 64
    if needs:
        with pytest.raises(MoccasinError) as err:
            run(small)
        assert err.value.code == -1
        torch.cuda.synchronize()
        assert bool(out.isnan().all())
    run(torch.empty(tr.lib().moc_linear_work(rows, cin, cout), dtype=torch.uint8, device="cuda"))
    assert bool((out == {"weight": rows, "forward": cin, "input": cout}[call]).all())
