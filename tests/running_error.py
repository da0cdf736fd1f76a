"""Numbers in 64 bits beside how far the same computation in 32 bits may be from them: each operation adds half a step of float32,
u = 2^-24, of its result to what its operands' errors make of it.  Tolerances of tests come from the formula alone."""
import torch

U = 2.0 ** -24


class Near:
    def __init__(self, value, off=None):
        self.v = value.double() if isinstance(value, torch.Tensor) else torch.tensor(float(value), dtype=torch.float64)
        self.e = torch.zeros_like(self.v) if off is None else off

    def _of(self, v, e):
        return Near(v, e + U * (v.abs() + e))

    def __add__(self, o):
        return self._of(self.v + o.v, self.e + o.e)

    def __sub__(self, o):
        return self._of(self.v - o.v, self.e + o.e)

    def __mul__(self, o):
        return self._of(self.v * o.v, self.v.abs() * o.e + o.v.abs() * self.e + self.e * o.e)

    def sum(self, dim, deep):
        """`deep` additions one after the other at most"""
        return Near(self.v.sum(dim), self.e.sum(dim) + deep * U * (self.v.abs() + self.e).sum(dim))

    def col(self):
        return Near(self.v[:, None], self.e[:, None])

    def over(self, n):
        return self._of(self.v / n, self.e / n)

    def inverse_root(self):
        """1 / sqrt: within two steps of float32 of that of its argument"""
        low = (self.v - self.e).clamp(min=1e-300)
        v = self.v ** -0.5
        return Near(v, torch.maximum(low ** -0.5 - v, v - (self.v + self.e) ** -0.5) + 4 * U * v)


def check(got, near, dtype=None):
    """`got` is the value within its error and the rounding to its type, NaN and infinities in the same places"""
    got = got.cpu()
    t = dtype or got.dtype
    f = torch.finfo(t)
    want, off = near.v, near.e
    assert got.shape == want.shape
    assert bool((got.double().isnan() == want.isnan()).all()), "NaN in other places"
    over = want.abs() >= f.max
    allowed = off + f.eps / 2 * (want.abs() + off) + f.smallest_normal * f.eps
    far = torch.where(want.isnan() | over, 0.0, (got.double() - want).abs() - allowed)
    assert float(far.max() if far.numel() else 0.0) <= 0, f"off by {float((got.double() - want).abs().nan_to_num().max())}, {float(far.max())} more than allowed"
