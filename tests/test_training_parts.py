"""How a linear layer's products are cut up: by the library's own arithmetic, without a device."""
import random

import pytest

UNITS = 256


@pytest.fixture(scope="module")
def tr():
    from paper_2304_14463_amd import training
    training.lib()
    return training


def sizes():
    """Ordinary sizes, and rows up to the largest with few columns, whose sums are cut into most parts."""
    rng = random.Random(1)
    out = [(rows, cin, cout) for rows in (2147483136, 2147482625, 2147482624, 2147418112, (1 << 30) + 1) for cin, cout in ((1, 1), (8, 8), (64, 64), (7, 300), (200, 16))]
    out += [(rng.randint(0, 40000), rng.randint(0, 20000), rng.randint(0, 20000)) for _ in range(200)]
    return out + [(0, 8, 8), (1, 1, 1), (1, 4194240, 8), (8, 8, 4194240)]


@pytest.mark.parametrize("product", ["forward", "backward_input", "backward_weight"])
@pytest.mark.parametrize("aligned", [True, False])
def test_the_parts_of_a_sum_are_the_whole(tr, product, aligned):
    for rows, cin, cout in sizes():
        for units in (UNITS, 1, 304):
            p = tr.moc_linear_parts(product, rows, cin, cout, aligned, units)
            terms = {"forward": cin, "backward_input": cout, "backward_weight": rows}[product]
            assert (p.parts - 1) * p.terms + p.last == terms, (rows, cin, cout, units, p)
            assert p.parts >= 1 and p.terms % 64 == 0 and (0 < p.last <= p.terms or terms == 0)
            assert p.tile in (64, 128, 256) and not (p.direct and not aligned)


def test_refusals(tr):
    from paper_2304_14463_amd.moccasin import MoccasinError
    with pytest.raises(ValueError):
        tr.moc_linear_parts("backward", 1, 1, 1, units=UNITS)
    for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, -1), (1 << 31, 1, 1), (1, 1 << 23, 1), (1, 1, 1 << 23)):
        with pytest.raises(MoccasinError):
            tr.moc_linear_parts("forward", *bad, units=UNITS)
    with pytest.raises(MoccasinError):
        tr.moc_linear_parts("forward", 1, 1, 1, units=-1)
    assert tr.lib().moc_linear_parts(3, 1, 1, 1, 1, UNITS, None) == -1 and tr.lib().moc_linear_parts(0, 1, 1, 1, 1, UNITS, None) == -1
