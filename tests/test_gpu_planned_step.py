"""A training step run as a plan says (examples/planned_step.py)."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("planned_step", os.path.join(ROOT, "examples", "planned_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("blocks,rows,width,share", [(8, 200, 64, 0.6), (5, 77, 96, 0.8), (1, 33, 40, 1.0)])
def test_a_plan_gives_the_gradients_of_the_plain_schedule(example, blocks, rows, width, share):
    inner = 4 * width
    step, p = example.Step(blocks, rows, width, inner), example.make_parameters(blocks, width, inner)
    g = torch.Generator(device="cuda").manual_seed(blocks)
    x, dy = (torch.randn(rows, width, generator=g, device="cuda").bfloat16() for _ in range(2))
    sequence, peak, plain = step.plan(share)
    assert set(sequence) == set(range(2 * blocks)) and peak <= plain
    if share < 1:
        assert len(sequence) > 2 * blocks and peak <= share * plain
    y, dx, grads = step.run(sequence, x, dy, p)
    y2, dx2, grads2 = step.run(step.plain(), x, dy, p)
    assert torch.equal(y, y2) and torch.equal(dx, dx2)
    for a, b in zip(grads, grads2):
        assert a.keys() == b.keys() == p[0].keys() and all(torch.equal(a[k], b[k]) for k in a)
        assert all(a[k].isfinite().all() and a[k].shape == p[0][k].shape for k in a)


def test_the_only_block_against_64_bits(example):
    """db2 is a sum of dy.  dw2 = dy^T h with h = gelu of the kept argument, which is off by 2^-4 of itself (e4m3) or by 2^-10 of its
    block's scale, below 2^-9 of the row's largest; before that by the roundings of n (bf16, 2^-8) and of the sums (2^-16 is
    plenty); gelu's slope is below 1.13; h is rounded to bf16 (2^-8)."""
    rows, width, inner = 64, 64, 256
    step, p = example.Step(1, rows, width, inner), example.make_parameters(1, width, inner)
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(rows, width, generator=g, device="cuda").bfloat16() for _ in range(2))
    _, _, grads = step.run(step.plain(), x, dy, p)
    x, dy, q = x.double(), dy.double(), {k: v.double() for k, v in p[0].items()}
    n = torch.nn.functional.layer_norm(x, (width,), q["gamma"], q["beta"])
    u = n @ q["w1"].t() + q["b1"]
    h = torch.nn.functional.gelu(u, approximate="tanh")
    du = (2.0 ** -8 + 2.0 ** -16) * (n.abs() @ q["w1"].abs().t() + q["b1"].abs())
    du = du + 2.0 ** -4 * (u.abs() + du) + 2.0 ** -9 * (u.abs() + du).amax(1, keepdim=True)
    dh = 1.13 * du
    dh = dh + 2.0 ** -8 * (h.abs() + dh)
    bound = dy.abs().t() @ dh + 2.0 ** -16 * (dy.abs().t() @ (h.abs() + dh))
    assert bool(((grads[0]["w2"].double() - dy.t() @ h).abs() <= bound).all())
    assert bool(((grads[0]["b2"].double() - dy.sum(0)).abs() <= 2.0 ** -16 * dy.abs().sum(0)).all())
