"""Whether two matrices share memory, as the binding of the training operators tells it, against a count of all bytes.  No GPU."""
import random

import pytest


@pytest.fixture(scope="module")
def native():
    from paper_2304_14463_amd import training
    return training._bound()


def bytes_of(at, rows, width, step):
    return {at + r * step + b for r in range(rows) for b in range(width)}


def test_against_all_bytes(native):
    rng = random.Random(3)
    seen = [0, 0]
    for _ in range(30000):
        spans = []
        for _ in range(2):
            width = rng.randint(0, 7)
            spans.append((1000 + rng.randint(0, 60), rng.choice([0, 1, 1, 2, 3, 5, 9]), width, max(1, width) + rng.randint(0, 9)))
        if rng.random() < 0.5:   # the two with one step, as slices of one matrix have it
            step = max(spans[0][3], spans[1][3])
            spans = [s[:3] + (step,) for s in spans]
        want = bool(bytes_of(*spans[0]) & bytes_of(*spans[1]))
        assert native.shares(*spans[0], *spans[1]) is want, spans
        seen[want] += 1
    assert min(seen) > 3000


def test_large_matrices(native):
    step, rows = 1 << 23, 2147483136
    at = 1 << 40
    assert native.shares(at, rows, 4096, step, at + 4095, rows, 4096, step)
    assert not native.shares(at, rows, 4096, step, at + 4096, rows, 4096, step)
    assert native.shares(at, rows, 4096, step, at + (rows - 1) * step + 4095, rows, 1, step)
    assert not native.shares(at, rows, 4096, step, at + (rows - 1) * step + 4096, rows, 1, step)
    assert not native.shares(at, rows, 4096, step, at - step + 4096, 2, 4096, step)


def test_refusals(native):
    for bad in ((), (1,) * 7, (0, 1, 1, 0, 0, 1, 1, 1), (0, 1, 1, 1, 0, 1, 1, 0), ("x",) * 8):
        with pytest.raises((TypeError, ValueError)):
            native.shares(*bad)
