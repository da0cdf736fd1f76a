"""Log probabilities, entropies, alternatives and their gradient against the definition in 64 bits.

Tolerances.  u = 2^-24 is half a step of float32.  A term 2^t of a row's sums is off by exp2's ulp (2 u), by t's rounding (u |t|) and by
scale / ln 2 being rounded (u |z|); terms are added by a lane one after the other, V / 512 of them in each of two sums at most
where a lane has V / 256, and over lanes, waves and parts in some forty steps more, each with u of the sum and the factors that join
them: (V / 512 + 64) u for the logarithm of the sum, and 4 u of the magnitudes of z that have a share in it.  The
entropy's second sum is off by as much of sum p |t|, and by u times the variance of z for the scale's rounding.  In the gradient a
probability is off by u (4 |z - lse| + 8) of itself.  What is written is off by half a step of its type besides."""
import math
import zlib

import pytest
import torch

from paper_2304_14463_amd.moccasin import MoccasinError
from training_reference import Framed, TYPES, half_step

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2304_14463_amd import training
    training.lib()
    return training


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def definition(x, tokens, scale, top):
    """of float64 logits with no NaN and no +infinity; the scale is the float that the call takes"""
    z = x * float(torch.tensor(scale))
    m = z.amax(1, keepdim=True)
    d = z - torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(d)
    s = e.sum(1)
    lse = torch.where(m[:, 0] == -math.inf, -math.inf, m[:, 0] + torch.log(s))
    p = torch.where(s[:, None] > 0, e / s[:, None], 0.0)
    logs = torch.where(m == -math.inf, -math.inf, d - torch.log(s)[:, None])
    entropy = -(p * torch.where(p > 0, logs, 0.0)).sum(1)
    at = tokens.clamp(0, x.shape[1] - 1).long()
    logp = logs.gather(1, at[:, None])[:, 0]
    logp = torch.where(tokens < 0, 0.0, torch.where(tokens >= x.shape[1], math.nan, logp))
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    # magnitudes of z with a share in the sum
    near = torch.where(p > 2.0 ** -40, z.abs(), 0.0).amax(1)
    far = torch.where(p > 0, p * logs.abs(), 0.0).sum(1)
    centre = (p * torch.where(p > 0, z, 0.0)).sum(1, keepdim=True)
    spread = (p * torch.where(p > 0, z - centre, 0.0) ** 2).sum(1)
    return dict(lse=lse, entropy=entropy, logp=logp, ids=ids, top=logs.gather(1, ids), p=p, logs=logs, near=near, far=far, spread=spread)


def close(got, want, bound):
    got, want = got.double().cpu(), want.double().cpu()
    want = torch.where(want.abs() > torch.finfo(torch.float32).max, want.sign() * math.inf, want)   # a difference that float32 does not have
    assert got.shape == want.shape
    assert bool((got.isnan() == want.isnan()).all())
    same = got == want
    off = torch.where(same | want.isnan(), 0.0, (got - want).abs() - bound)
    assert float(off.max() if off.numel() else 0.0) <= 0, (float((got - want).abs().nan_to_num(posinf=0).max()), float(off.max()))


def check_forward(got, want, vocab, scale):
    n = (vocab / 512 + 64) * U
    bound = n + 4 * U * (want["near"] + want["lse"].abs().nan_to_num(posinf=0.0))
    close(got.lse, want["lse"], bound)
    if got.logp is not None:
        close(got.logp, want["logp"], bound + 4 * U * want["logp"].abs().nan_to_num(posinf=0.0))
    close(got.entropy, want["entropy"], n * (1 + want["far"]) + 4 * U * want["near"] + U * want["spread"] + 4 * U * want["entropy"])
    if got.top_tokens is not None:
        assert torch.equal(got.top_tokens.cpu(), want["ids"])
        close(got.top_logp, want["top"], bound[:, None] + 4 * U * want["top"].abs().nan_to_num(posinf=0.0))


SIZES = [(1, 1), (3, 2), (5, 7), (2, 63), (4, 64), (3, 65), (300, 130), (2, 1000), (7, 2047), (3, 8192), (2, 8193), (5, 32003), (1, 131072), (2, 300001)]


def inputs(rows, vocab, dtype, *more):
    g = gen(rows, vocab, str(dtype), *more)
    x = torch.randn(rows, vocab, generator=g, dtype=torch.float64) * torch.exp(torch.randn(rows, 1, generator=g, dtype=torch.float64))
    x[torch.rand(rows, vocab, generator=g) < 0.1] = -math.inf
    x[:, 0] = 0.5
    tokens = torch.randint(-1, vocab, (rows,), generator=g)
    return g, x.to(dtype), tokens


@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lead,pad", [(0, 0), (1, 3)])
def test_forward(tr, rows, vocab, dtype, lead, pad):
    g, x, tokens = inputs(rows, vocab, TYPES[dtype])
    framed = Framed(rows, vocab, TYPES[dtype], lead, pad)
    framed.of(x)
    for scale, top, kind in ((1.0, min(20, vocab), torch.int64), (0.3, 0, torch.int32), (4.0, min(64, vocab), torch.int32), (1.5, 1, None)):
        got = tr.moc_logprob_forward(framed.inner, None if kind is None else tokens.to(kind).cuda(), scale=scale, top=top)
        assert (got.logp is None) == (kind is None) and (got.top_tokens is None) == (top == 0)
        check_forward(got, definition(x.double(), tokens, scale, top), vocab, scale)
    assert framed.intact() and torch.equal(framed.inner.cpu(), x)
    again = tr.moc_logprob_forward(framed.inner, None, scale=1.5, top=1)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, again))


def hard_rows(vocab, dtype):
    """rows that masks and orders make hard, without NaN and +infinity"""
    f = torch.finfo(dtype)
    low, high = f.min, f.max
    g = gen(vocab, str(dtype))
    x = torch.randn(20, vocab, generator=g).to(dtype)
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, vocab // 2] = 3.0
    x[2] = low                                           # a mask of the lowest value that leaves nothing
    x[3] = low
    x[3, vocab - 1] = -1.0
    x[4] = torch.linspace(-10, 10, vocab).to(dtype)      # every one better than those before
    x[5] = torch.linspace(10, -10, vocab).to(dtype)
    x[6] = 0.0
    x[6, ::2] = -0.0                                     # all equal
    x[7] = high
    x[8] = low
    x[8, vocab // 3] = high
    x[9] = torch.randn(vocab, generator=g).to(dtype) * (high / 8)
    x[10, : vocab // 2] = -math.inf
    x[11, vocab // 2:] = low
    x[12] = -math.inf
    x[12, ::2] = low
    x[13] = torch.randint(-2, 3, (vocab,), generator=g).to(dtype)   # five values
    x[14, :] = -math.inf
    x[14, -1] = low
    x[15] = tiny(dtype)
    x[16] = 60.0
    x[16, vocab // 4] = 61.0
    x[17] = high
    x[17, ::3] = -math.inf
    x[18] = -high / 2
    return x


@pytest.mark.parametrize("vocab", [1, 2, 64, 100, 2048, 9000, 70001])
@pytest.mark.parametrize("dtype", TYPES)
def test_masks_and_orders(tr, vocab, dtype):
    """Where values are within a step of the largest float32, z and lse have its steps: bounds go by |z|."""
    dtype = TYPES[dtype]
    x = hard_rows(vocab, dtype)
    tokens = torch.arange(20) % vocab
    got = tr.moc_logprob_forward(x.cuda(), tokens.cuda(), top=min(vocab, 64))
    want = definition(x.double(), tokens, 1.0, min(vocab, 64))
    check_forward(got, want, vocab, 1.0)
    assert float(got.entropy[0]) == 0 and float(got.lse[0]) == -math.inf and float(got.logp[0]) == -math.inf
    dlogp, dh = torch.full((20,), 0.5), torch.full((20,), 0.25)
    d = tr.moc_logprob_backward(x.cuda(), got.lse, tokens.cuda(), dlogp.cuda(), got.entropy, dh.cuda(), dtype=torch.float32).cpu()
    assert bool(d.isfinite().all()) and not d[0].any()
    ok = (x.double().abs().nan_to_num(posinf=0.0).amax(1) < 1000) & (got.lse.cpu() > -math.inf)   # nothing left: 0, as the header says
    assert not d[got.lse.cpu() == -math.inf].any()
    check_gradient(d[ok], x[ok], tokens[ok], got.lse[ok.cuda()], got.entropy[ok.cuda()], dlogp[ok], dh[ok], 1.0)


@pytest.mark.parametrize("rows,vocab", [(1100, 70001), (64, 300001)])
def test_alternatives_that_lie_close_together(tr, rows, vocab):
    """More logits above what many lanes reach than there is room for: whole runs of a few lanes, over all of a row or of a part; and
    rows with more equal ones than that."""
    g = gen(rows, vocab)
    x = torch.randn(rows, vocab, generator=g).half()
    run = torch.arange(vocab) // 8 % 256
    some = [0, 7, rows // 2, rows - 1]
    x[0] = torch.where(run < 20, 100 + torch.rand(vocab, generator=g) * 50, -1.0).half()
    x[7] = torch.where(run % 37 == 5, 3.0, -torch.rand(vocab, generator=g)).half()
    x[rows // 2] = torch.where(run == 255, torch.arange(vocab) / 8.0, -math.inf).half()
    x[rows - 1] = torch.where((run < 2) | (torch.arange(vocab) > vocab - 3000), 5.0, 0.0).half()
    for top in (1, 5, 20, 64):
        got = tr.moc_logprob_forward(x.cuda(), top=top)
        want = definition(x[some].double(), torch.zeros(4, dtype=torch.int64), 1.0, top)
        assert torch.equal(got.top_tokens.cpu()[some], want["ids"])
        check_forward(type(got)(None, *(None if t is None else t[some] for t in got[1:])), want, vocab, 1.0)


def test_values_that_are_no_logits(tr):
    """NaN and +infinity anywhere, in every kind of row, leave a row's results NaN and no alternatives; other rows keep theirs."""
    for dtype in TYPES.values():
        for vocab in (1, 70, 3000, 40000):
            for odd in (math.nan, math.inf):
                x = hard_rows(vocab, dtype)
                bad = torch.zeros(20, dtype=torch.bool)
                bad[1::2] = True
                for r in range(1, 20, 2):
                    x[r, (r * 997) % vocab] = odd
                tokens = torch.arange(20) % vocab
                got = tr.moc_logprob_forward(x.cuda(), tokens.cuda(), top=min(5, vocab))
                for r in (got.lse, got.entropy, got.logp, got.top_logp):
                    assert bool(r.cpu()[bad].isnan().all()) and not bool(r.cpu()[~bad].isnan().any())
                assert bool((got.top_tokens.cpu()[bad] == -1).all()) and bool((got.top_tokens.cpu()[~bad] >= 0).all())
                d = tr.moc_logprob_backward(x.cuda(), got.lse, tokens.cuda(), torch.ones(20, device="cuda"))
                assert bool(d.cpu()[bad].isnan().all()) and not bool(d.cpu()[~bad].isnan().any())


def test_tokens_out_of_range(tr):
    x = torch.randn(6, 50, device="cuda")
    for kind in (torch.int32, torch.int64):
        tokens = torch.tensor([-1, -100, 49, 50, 2 ** 31 - 1, 0], dtype=kind, device="cuda")
        if kind == torch.int64:
            tokens[4] = 2 ** 40 + 3
            tokens[1] = -2 ** 40 + 3
        got = tr.moc_logprob_forward(x, tokens)
        assert bool((got.logp[:2] == 0).all()) and bool(got.logp[3:5].isnan().all()) and bool(got.logp[[2, 5]].isfinite().all())
        d = tr.moc_logprob_backward(x, got.lse, tokens, torch.full((6,), math.nan, device="cuda").index_fill_(0, torch.tensor([2, 3, 4, 5], device="cuda"), 1.0))
        assert not d[:2].any() and bool(d[3:5].isnan().all()) and bool(d[[2, 5]].isfinite().all())


def check_gradient(got, x, tokens, lse, entropy, dlogp, dentropy, scale):
    x, lse, dlogp, tokens, scale = x.double(), lse.double().cpu(), dlogp.double(), tokens.cpu(), float(torch.tensor(scale))
    t = x * scale - lse[:, None]
    p = torch.exp(t)
    t = torch.where(p > 0, t, 0.0)
    one = (torch.arange(x.shape[1])[None] == tokens[:, None]).double()
    dl = torch.where(tokens < 0, 0.0, dlogp)[:, None]
    rel = U * (4 * t.abs() + 8)
    # exp2 has no results below float32's smallest normal number: such a probability is 0, whatever it is multiplied by
    gone = torch.full_like(p, 2.0 ** -126)
    want, bound = dl * (one - p), dl.abs() * (p * rel + gone + 2 * U * (one - p).abs() + U * one)
    if dentropy is not None:
        h, dh = entropy.double().cpu()[:, None], dentropy.double()[:, None]
        want = want - dh * p * (t + h)
        bound = bound + dh.abs() * (p * (rel + 8 * U) + gone) * (t.abs() + h) + 4 * U * want.abs()
    want, bound = scale * want, scale * bound + 4 * U * (scale * want).abs()
    close(got, want, bound + half_step(got.dtype) * (want.abs() + bound) + tiny(got.dtype) + 2.0 ** -125)


@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lead,pad", [(0, 0), (1, 3)])
def test_gradient(tr, rows, vocab, dtype, lead, pad):
    g, x, tokens = inputs(rows, vocab, TYPES[dtype], "gradient")
    dlogp, dh = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    framed = Framed(rows, vocab, TYPES[dtype], lead, pad)
    framed.of(x)
    for scale in (1.0, 0.4):
        f = tr.moc_logprob_forward(framed.inner, tokens.cuda(), scale=scale)
        for out_type in {TYPES[dtype], torch.float32}:
            out = Framed(rows, vocab, out_type, lead, pad)
            assert tr.moc_logprob_backward(framed.inner, f.lse, tokens.int().cuda(), dlogp.cuda(), f.entropy, dh.cuda(), scale, out=out.inner) is out.inner
            check_gradient(out.inner.cpu(), x, tokens, f.lse, f.entropy, dlogp, dh, scale)
            assert out.intact()
        check_gradient(tr.moc_logprob_backward(framed.inner, f.lse, tokens.cuda(), dlogp.cuda(), scale=scale).cpu(), x, tokens, f.lse, None, dlogp, None, scale)
        only = tr.moc_logprob_backward(framed.inner, f.lse, entropy=f.entropy, dentropy=dh.cuda(), scale=scale).cpu()
        check_gradient(only, x, torch.full_like(tokens, -1), f.lse, f.entropy, dlogp, dh, scale)
    want = tr.moc_logprob_backward(framed.inner, f.lse, tokens.cuda(), dlogp.cuda(), f.entropy, dh.cuda(), scale)
    assert tr.moc_logprob_backward(framed.inner, f.lse, tokens.cuda(), dlogp.cuda(), f.entropy, dh.cuda(), scale, out=framed.inner) is framed.inner
    assert torch.equal(framed.inner, want) and framed.intact()
    assert not tr.moc_logprob_backward(x.cuda(), f.lse, scale=scale).any()   # no gradient at all


def test_gradient_against_differences(tr):
    """Central differences of the definition in 64 bits, h = 1e-5: their error is some h^2 of third derivatives, all below 2, and
    2^-52 / h of rounding: 1e-9; the kernel's is below 1e-5 here."""
    g = gen("differences")
    x, tokens, scale = torch.randn(3, 40, generator=g).float(), torch.tensor([4, -1, 39]), 0.7
    dlogp, dh = torch.randn(3, generator=g), torch.randn(3, generator=g)
    f = tr.moc_logprob_forward(x.cuda(), tokens.cuda(), scale=scale)
    got = tr.moc_logprob_backward(x.cuda(), f.lse, tokens.cuda(), dlogp.cuda(), f.entropy, dh.cuda(), scale).cpu().double()

    def value(x):
        w = definition(x, tokens, scale, 0)
        return (w["logp"] * dlogp.double() + w["entropy"] * dh.double()).sum()

    for r in range(3):
        for c in range(40):
            step = torch.zeros(3, 40, dtype=torch.float64)
            step[r, c] = 1e-5
            slope = (value(x.double() + step) - value(x.double() - step)) / 2e-5
            assert abs(float(slope - got[r, c])) < 2e-5


@pytest.mark.parametrize("rows,vocab", [(1, 50000), (37, 4099)])
def test_captured_and_on_another_stream(tr, rows, vocab):
    g, x, tokens = inputs(rows, vocab, torch.bfloat16, "captured")
    x, t, d = x.cuda(), tokens.cuda(), torch.ones(rows, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first = tr.moc_logprob_forward(x, t, top=20, stream=side)
    side.synchronize()
    graphs = []
    for _ in range(2):   # two graphs, each with its own workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f = tr.moc_logprob_forward(x, t, top=20)
            out = tr.moc_logprob_backward(x, f.lse, t, d, f.entropy, d)
        graphs.append((graph, f, out))
    for turn in range(3):
        x.copy_(torch.randn(rows, vocab, generator=g))
        for graph, _, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        f = tr.moc_logprob_forward(x, t, top=20)
        out = tr.moc_logprob_backward(x, f.lse, t, d, f.entropy, d)
        for _, other, other_out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(f, other)) and torch.equal(out, other_out)
    assert first.top_tokens.shape == (rows, 20)


def test_offsets_beyond_32_bits(tr):
    """rows of a matrix whose last one begins past 2^32 bytes and 2^31 values"""
    rows, vocab = 17000, 131072
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    x[-1, 77], x[-1, -1] = 9.0, 8.0
    t = torch.full((rows,), 77, device="cuda")
    f = tr.moc_logprob_forward(x, t, top=2)
    w = definition(x[-1:].double().cpu(), t[-1:].cpu(), 1.0, 2)
    assert f.top_tokens[-1].tolist() == [77, vocab - 1] and abs(float(f.logp[-1]) - float(w["logp"])) < 1e-3
    assert bool((f.lse[:-1] == f.lse[0]).all()) and abs(float(f.lse[0]) - math.log(vocab)) < 1e-3
    d = tr.moc_logprob_backward(x, f.lse, t, torch.ones(rows, device="cuda"), out=x)
    assert abs(float(d[-1, 77]) - (1 - math.exp(float(w["logp"])))) < 0.01 and abs(float(d[-1, -1]) + math.exp(float(w["top"][0, 1]))) < 0.01
    assert float(d[0, 77]) == 1.0 and bool((d[:-1, 78] == d[0, 78]).all())


def test_refusals(tr):
    x, t, v = torch.zeros(4, 64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    same = torch.zeros(4 * 64 + 4, device="cuda")
    for bad in (lambda: tr.moc_logprob_forward(x.t()), lambda: tr.moc_logprob_forward(x[0]), lambda: tr.moc_logprob_forward(x.double()), lambda: tr.moc_logprob_forward(tr.moc_checkpoint_write(x)),
                lambda: tr.moc_logprob_forward(x, t[:3]), lambda: tr.moc_logprob_forward(x, v), lambda: tr.moc_logprob_forward(x, t.cpu()), lambda: tr.moc_logprob_forward(x, t[:, None]),
                lambda: tr.moc_logprob_forward(x, top=65), lambda: tr.moc_logprob_forward(x, top=-1), lambda: tr.moc_logprob_forward(x[:, :3], top=4), lambda: tr.moc_logprob_forward(x, scale=0.0),
                lambda: tr.moc_logprob_forward(x, scale=-1.0), lambda: tr.moc_logprob_forward(x, scale=math.nan), lambda: tr.moc_logprob_forward(x[:, :0]),
                lambda: tr.moc_logprob_backward(x, v[:3]), lambda: tr.moc_logprob_backward(x, v.double()), lambda: tr.moc_logprob_backward(x, v, None, v), lambda: tr.moc_logprob_backward(x, v, t, v, None, v),
                lambda: tr.moc_logprob_backward(x, v, dtype=torch.float16), lambda: tr.moc_logprob_backward(x, v, out=x[:3]), lambda: tr.moc_logprob_backward(x, v, t, v, out=x.double()),
                lambda: tr.moc_logprob_backward(same[:256].view(4, 64), v, out=same[4:].view(4, 64)), lambda: tr.moc_logprob_backward(x, same[:4], out=same[:256].view(4, 64)),
                lambda: tr.moc_logprob_backward(x, v, t, same[252:256], out=same[:256].view(4, 64))):
        with pytest.raises((ValueError, MoccasinError)):
            bad()
    none = tr.moc_logprob_forward(x[:0], t[:0], top=3)
    assert none.logp.shape == (0,) and none.top_tokens.shape == (0, 3) and tr.moc_logprob_backward(x[:0], v[:0]).shape == (0, 64)


def test_every_call_asks_for_the_device_of_its_tensors(tr, monkeypatch):
    x, v = torch.zeros(4, 64, device="cuda"), torch.zeros(4, device="cuda")
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for call in (lambda: tr.moc_logprob_forward(x), lambda: tr.moc_logprob_backward(x, v)):
            with pytest.raises(ValueError, match="cuda:0.*cuda:1"):
                call()


@pytest.mark.parametrize("rows", [1, 600])
@pytest.mark.parametrize("vocab", [4999, 32003, 131072])
def test_alternatives_among_many_candidates(tr, rows, vocab):
    """Rows that rise or fall by single float32 steps, so that whatever was gathered first is not the best; and 1 .. 1025 distinct or
    equal logits above the others, in order or not, in every place or in few lanes, with more that equal the last."""
    g = gen(vocab)
    steps = 1.0 + torch.arange(vocab) * 2.0 ** -23
    cases = [steps, steps.flip(0), -steps, steps[torch.randperm(vocab, generator=g)], steps.half().float(), torch.full((vocab,), -2.5)]
    for many in (1, 63, 64, 65, 127, 128, 129, 512, 959, 960, 961, 1023, 1024, 1025):
        for equal in (True, False):
            for at in (torch.arange(many) + (vocab - many) // 2, torch.randperm(vocab, generator=g)[:many]):
                x = torch.zeros(vocab)
                x[at] = 3.0 if equal else 3.0 + torch.randperm(many, generator=g) * 2.0 ** -20
                cases.append(x)
        x = torch.where(torch.arange(vocab) % 64 < 8, 1.0, -math.inf)
        x[torch.randperm(vocab, generator=g)[:many]] = 2.0
        cases.append(x)
    x = torch.stack(cases)
    tokens = torch.zeros(len(x), dtype=torch.int64)
    for top in (1, 2, 20, 64):
        want = definition(x.double(), tokens, 1.0, top)
        calls = x.cuda().repeat(-(-rows // len(x)), 1) if rows > 1 else x.cuda()
        got = [tr.moc_logprob_forward(calls, top=top)] if rows > 1 else [tr.moc_logprob_forward(calls[i:i + 1], top=top) for i in range(len(x))]
        tops = torch.cat([f.top_tokens for f in got]).cpu()
        assert torch.equal(tops, want["ids"].repeat(len(tops) // len(x), 1))
        for f in got if rows > 1 else []:
            check_forward(type(f)(None, *(None if t is None else t[:len(x)] for t in f[1:])), want, vocab, 1.0)


def test_rows_without_a_token_have_no_gradient_whatever_they_hold(tr):
    """Padding that was never written: NaN, infinities; the gradient of an entropy there is what its row is."""
    for dtype in TYPES.values():
        for vocab in (1, 70, 9001):
            x = torch.randn(6, vocab, generator=gen(vocab)).to(dtype)
            x[1], x[2, vocab // 2], x[3], x[4, 0] = math.nan, math.nan, math.inf, math.inf
            x[5] = -math.inf
            tokens = torch.tensor([0, -1, -1, -100, -1, -1])
            got = tr.moc_logprob_forward(x.cuda(), tokens.cuda())
            assert not got.logp.cpu()[1:].any() and bool(got.lse.cpu()[1:5].isnan().all())
            d = tr.moc_logprob_backward(x.cuda(), got.lse, tokens.cuda(), torch.full((6,), math.nan, device="cuda").index_fill_(0, torch.tensor([0], device="cuda"), 1.0))
            assert not d.cpu()[1:].any() and bool(d.cpu()[0].isfinite().all())
            d = tr.moc_logprob_backward(x.cuda(), got.lse, tokens.cuda(), torch.ones(6, device="cuda"), got.entropy, torch.ones(6, device="cuda")).cpu()
            assert bool(d[1:5].isnan().all()) and bool(d[0].isfinite().all()) and not d[5].any()
