"""Log probabilities, entropies and gradients of rows that are masked by finite numbers or lie far from 0, against the definition in 64
bits.

Tolerances, beside those of test_gpu_logprob.py.  u = 2^-24 is half a step of float32, V the columns, d a logit's distance from the row's
largest times the scale.  Every term of a row's sums goes by differences, or by differences from a number within a quarter of a power
of two of the largest logit, so what the entropy is off by does not grow with the logits: a term's exponent by 3 u |d| (the difference,
the scale, their product), the sums by (V / 512 + 64) u of themselves, the logarithm and the quotient by a few u more, which is
(V / 512 + 68) u (2 + sum p |log p| + H); exponents that are off by e_i move the entropy by sum p_i e_i (log p_i + H) and the second
sum's own factor by sum p_i e_i: 4 u sum p |d| (1 + |log p| + H)."""
import math

import pytest
import torch

from test_gpu_logprob import U, check_forward, close, definition, gen, tiny, tr   # noqa: F401
from training_reference import Framed, TYPES, half_step

pytestmark = pytest.mark.gpu

MASKS = [-1e4, -1e9, -2e9, -4e9, -1e10, -1e30, -2.0 ** 64, -2.0 ** 120, -2.0 ** 127, -math.inf]
OFFSETS = [1e3, -1e5, 1e5, -3e6, 1e7, -1e7, 1e9, -1e12, 1e30]
SCALES = [0.25, 0.5, 0.7, 0.9, 1.0, 1.25, 1 / 0.6, 5.0]


def far_rows(vocab, dtype):
    """Five rows for each mask (what the type does not hold is its lowest value) and one for each offset."""
    f, g = torch.finfo(dtype), gen("far", vocab, str(dtype))
    rows = []
    for mask in MASKS:
        mask = max(mask, f.min)
        x = torch.randn(5, vocab, generator=g).to(dtype)
        x[0] = mask
        some = torch.randperm(vocab, generator=g)[:20]
        x[1] = torch.full((vocab,), mask).to(dtype).index_copy_(0, some, x[1, some])
        x[2, :vocab // 2] = mask
        x[3, vocab // 2:] = mask
        x[4, :-1] = mask
        rows.append(x)
    for offset in OFFSETS:
        offset = max(min(offset, f.max / 2), f.min / 2)
        rows.append((torch.randn(1, vocab, generator=g).double() * 3 + offset).to(dtype))
    return torch.cat(rows)


def entropy_bound(want, vocab):
    logs, h = torch.where(want["p"] > 0, want["logs"], 0.0), want["entropy"]
    d = logs - torch.where(want["p"] > 0, want["logs"], -math.inf).amax(1, keepdim=True).nan_to_num(neginf=0.0)
    moved = (want["p"] * d.abs() * (1 + logs.abs() + h[:, None])).sum(1)
    return (vocab / 512 + 68) * U * (2 + want["far"] + h) + 4 * U * moved


@pytest.mark.parametrize("vocab", [1000, 9000, 32003])
@pytest.mark.parametrize("dtype", TYPES)
def test_forward_of_rows_far_from_0(tr, vocab, dtype):   # noqa: F811
    """In parts and, where there are many rows, each by one workgroup."""
    x = far_rows(vocab, TYPES[dtype])
    tokens = (torch.arange(len(x)) * 331) % vocab
    many = -(-1100 // len(x))
    for scale in SCALES:
        want = definition(x.double(), tokens, scale, 5)
        for repeat in (1, many):
            got = tr.moc_logprob_forward(x.cuda().repeat(repeat, 1), tokens.cuda().repeat(repeat), scale=scale, top=5)
            first = type(got)(*(t[:len(x)] for t in got))
            check_forward(first, want, vocab, scale)
            close(first.entropy, want["entropy"], entropy_bound(want, vocab))
            for t in got:   # rows that are alike lie alike only where a row's size is a multiple of 16 bytes
                if vocab % 8 == 0:
                    assert torch.equal(t, t[:len(x)].repeat(repeat, *[1] * (t.dim() - 1)))


def check_far_gradient(got, x, want, tokens, dlogp, dentropy, scale, vocab):
    """Against the gradient by 64-bit logits alone.  A probability is off by u (4 |z - lse| + 8) of itself as in
    test_gpu_logprob.py, and by what lse is off by: as check_forward allows, or, beyond 1024 either way, where the row's own sum is
    taken again by differences from its largest, by that sum's (V / 512 + 64) u and the rounding of its logarithm.  The entropy's part is
    off by the same, times p, and by what the entropy is off by."""
    scale, n = float(torch.tensor(scale)), (vocab / 512 + 64) * U
    p, t, h = want["p"], torch.where(want["p"] > 0, want["logs"], 0.0), want["entropy"][:, None]
    lse = want["lse"].abs().nan_to_num(posinf=math.inf)
    e = torch.where(lse > 1024, n + 4 * U * (1 + math.log(vocab)), n + 4 * U * (want["near"] + lse))[:, None]
    one = (torch.arange(vocab)[None] == tokens[:, None]).double()
    dl, dh = torch.where(tokens < 0, 0.0, dlogp.double())[:, None], dentropy.double()[:, None]
    rel, gone = U * (4 * t.abs() + 8) + e, torch.full_like(p, 2.0 ** -126)
    value = dl * (one - p) - dh * p * (t + h)
    bound = dl.abs() * (p * rel + gone + 2 * U * (one - p).abs() + U * one)
    bound = bound + dh.abs() * ((p * (rel + 8 * U) + gone) * (t.abs() + h) + p * (e + entropy_bound(want, vocab)[:, None])) + 4 * U * value.abs()
    nothing = (want["lse"] == -math.inf)[:, None]   # by the definition: all of the row's logits are -infinity
    value, bound = torch.where(nothing, 0.0, scale * value), scale * bound + 4 * U * (scale * value).abs()
    close(got, value, bound + half_step(got.dtype) * (value.abs() + bound) + tiny(got.dtype) + 2.0 ** -125)


@pytest.mark.parametrize("vocab", [1, 1000, 9000, 32003])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_of_rows_far_from_0(tr, vocab, dtype):   # noqa: F811
    dtype = TYPES[dtype]
    x = far_rows(vocab, dtype) if vocab > 1 else torch.tensor([[3.0], [-6e4], [1e4], [-math.inf], [torch.finfo(dtype).min]]).to(dtype)
    tokens = (torch.arange(len(x)) * 331) % vocab
    tokens[1::7] = -1
    g = gen("far gradient", vocab)
    dlogp, dh = torch.randn(len(x), generator=g), torch.randn(len(x), generator=g)
    for scale in (0.5, 1.0, 1.25, 5.0):
        want = definition(x.double(), tokens, scale, 0)
        f = tr.moc_logprob_forward(x.cuda(), tokens.cuda(), scale=scale)
        for out_type in {dtype, torch.float32}:
            d = tr.moc_logprob_backward(x.cuda(), f.lse, tokens.cuda(), dlogp.cuda(), f.entropy, dh.cuda(), scale, dtype=out_type)
            check_far_gradient(d.cpu(), x, want, tokens, dlogp, dh, scale, vocab)
        only = tr.moc_logprob_backward(x.cuda(), f.lse, tokens.cuda(), dlogp.cuda(), scale=scale)
        check_far_gradient(only.cpu(), x, want, tokens, dlogp, torch.zeros(len(x)), scale, vocab)
        assert not only[1::7].any()
        logits = x.cuda()
        assert torch.equal(tr.moc_logprob_backward(logits, f.lse, tokens.cuda(), dlogp.cuda(), f.entropy, dh.cuda(), scale, out=logits),
                           tr.moc_logprob_backward(x.cuda(), f.lse, tokens.cuda(), dlogp.cuda(), f.entropy, dh.cuda(), scale))


def test_gradient_of_an_odd_matrix_far_from_0(tr):   # noqa: F811
    """Rows at odd addresses in a larger matrix, more columns than a workgroup takes, written over the logits: far rows beside others,
    nothing outside them."""
    for dtype in TYPES.values():
        rows, vocab = 6, 20001
        x = (torch.randn(rows, vocab, generator=gen("odd", str(dtype))) * 2).to(dtype)
        x[1] = torch.finfo(dtype).min
        x[2] = 2000.0
        x[4, 5:] = -3e4
        x[4, :5] = -2e4
        framed = Framed(rows, vocab, dtype, 3, 5)
        framed.of(x)
        tokens, ones = torch.arange(rows) * 4, torch.ones(rows)
        want = definition(x.double(), tokens, 1.0, 0)
        f = tr.moc_logprob_forward(framed.inner, tokens.cuda())
        tr.moc_logprob_backward(framed.inner, f.lse, tokens.cuda(), ones.cuda(), f.entropy, ones.cuda(), out=framed.inner)
        check_far_gradient(framed.inner.cpu(), x, want, tokens, ones, ones, 1.0, vocab)
        assert framed.intact()
