"""Whole training steps of a small stack by the training operators, as they are used together: residual connections between linear
layers, the loss from log probabilities and the entropy, all gradients, AdamW; against torch's autograd and the update's definition
in 64 bits.

The model: e = rows of a table (given), r0 = e; block i: n = before(r), u = n w1^T + b1, b = gelu(u) w2^T + b2, r' = s r + gate after(b);
logits = last(r) wl^T.  The loss is -sum of weight logp - 0.01 sum of the entropies."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2304_14463_amd import training
    training.lib()
    return training


ROWS, WIDTH, INNER, VOCAB, BLOCKS, GROUPS, SCALE, BONUS = 96, 64, 160, 500, 3, 4, 0.9, 0.01


def parameters(dtype):
    g = torch.Generator().manual_seed(11)
    normal = lambda *s, by=1.0: (torch.randn(*s, generator=g) * by).cuda()   # noqa: E731
    p = {}
    for i in range(BLOCKS):
        p.update({f"before{i}": 1 + normal(WIDTH, by=0.1), f"beta{i}": normal(WIDTH, by=0.1), f"w1{i}": normal(INNER, WIDTH, by=WIDTH ** -0.5), f"b1{i}": normal(INNER, by=0.1),
                  f"w2{i}": normal(WIDTH, INNER, by=INNER ** -0.5), f"b2{i}": normal(WIDTH, by=0.1), f"after{i}": 1 + normal(WIDTH, by=0.1), f"gate{i}": 0.5 + normal(GROUPS, WIDTH, by=0.2)})
    p["last"], p["out"] = 1 + normal(WIDTH, by=0.1), normal(VOCAB, WIDTH, by=WIDTH ** -0.5)
    e, tokens, weight = normal(ROWS, WIDTH).to(dtype), torch.randint(-1, VOCAB, (ROWS,), generator=g).cuda(), torch.rand(ROWS, generator=g).cuda()
    return p, e, tokens, weight


def is_matrix(name):
    return name.startswith(("w1", "w2")) or name == "out"


def step(tr, p, low, e, tokens, weight, keep):
    """(loss, gradients by name, e's gradient): parameters in 32 bits and the matrices' copies `low`"""
    norm = [tr.Norm("layer", p[f"before{i}"], p[f"beta{i}"]) for i in range(BLOCKS)] + [tr.Norm("rms", p["last"])]
    after = [tr.Norm("rms", p[f"after{i}"]) for i in range(BLOCKS)]
    first = tr.moc_residual_forward(None, e, before=norm[0], want_stream=False, keep=keep)
    streams, forwards, inner = [e], [first], []
    for i in range(BLOCKS):
        u, _ = tr.moc_linear_forward(forwards[i].n, low[f"w1{i}"], p[f"b1{i}"])
        a = torch.nn.functional.gelu(u.float(), approximate="tanh").to(u.dtype)
        b, _ = tr.moc_linear_forward(a, low[f"w2{i}"], p[f"b2{i}"])
        f = tr.moc_residual_forward(streams[i], b, p[f"gate{i}"], SCALE, after[i], norm[i + 1], keep=keep if i < BLOCKS - 1 else None)
        inner.append((u, a, b))
        streams.append(f.r)
        forwards.append(f)
    logits, _ = tr.moc_linear_forward(forwards[-1].n, low["out"], dtype=torch.float32)
    f = tr.moc_logprob_forward(logits, tokens, top=3)
    loss = -(weight * f.logp).sum() - BONUS * f.entropy.sum()
    grads = {}
    dlogits = tr.moc_logprob_backward(logits, f.lse, tokens, -weight, f.entropy, torch.full_like(weight, -BONUS), out=logits).to(e.dtype)
    grads["out"], _ = tr.moc_linear_backward_weight(dlogits, forwards[-1].n, want_bias=False)
    dn, dr = tr.moc_linear_backward_input(dlogits, low["out"]), None
    for i in reversed(range(BLOCKS)):
        u, a, b = inner[i]
        d = tr.moc_residual_backward(dr, dn, streams[i + 1], b, p[f"gate{i}"], SCALE, after[i], forwards[i + 1].after, norm[i + 1], forwards[i + 1].before)
        last = i == BLOCKS - 1
        grads["last" if last else f"before{i + 1}"] = d.before_gamma
        if not last:
            grads[f"beta{i + 1}"] = d.before_beta
        grads[f"after{i}"], grads[f"gate{i}"] = d.after_gamma, d.gate
        grads[f"w2{i}"], grads[f"b2{i}"] = tr.moc_linear_backward_weight(d.dblock, a)
        du = tr.moc_linear_backward_input(d.dblock, low[f"w2{i}"], act="gelu", pre=u)
        x = forwards[i].kept if keep else forwards[i].n
        grads[f"w1{i}"], grads[f"b1{i}"] = tr.moc_linear_backward_weight(du, x)
        dn, dr = tr.moc_linear_backward_input(du, low[f"w1{i}"]), d.dx
    d = tr.moc_residual_backward(None, dn, e, before=norm[0], before_stats=forwards[0].before, want_x=False)
    grads["before0"], grads["beta0"] = d.before_gamma, d.before_beta
    return loss, grads, d.dblock.float() + dr.float()


def definition(p, e, tokens, weight):
    p = {k: v.detach().double().requires_grad_() for k, v in p.items()}
    e = e.double().requires_grad_()
    rms = lambda x, g: x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * g   # noqa: E731
    r = e
    for i in range(BLOCKS):
        n = torch.nn.functional.layer_norm(r, (WIDTH,), p[f"before{i}"], p[f"beta{i}"])
        b = torch.nn.functional.gelu(n @ p[f"w1{i}"].t() + p[f"b1{i}"], approximate="tanh") @ p[f"w2{i}"].t() + p[f"b2{i}"]
        r = SCALE * r + p[f"gate{i}"].repeat_interleave(ROWS // GROUPS, 0) * rms(b, p[f"after{i}"])
    logs = torch.log_softmax(rms(r, p["last"]) @ p["out"].t(), 1)
    logp = torch.where(tokens < 0, 0.0, logs.gather(1, tokens.clamp(min=0)[:, None])[:, 0])
    loss = -(weight.double() * logp).sum() + BONUS * (logs.exp() * logs).sum()
    names = list(p)
    grads = torch.autograd.grad(loss, [p[k] for k in names] + [e])
    return loss.detach(), dict(zip(names, grads)), grads[-1]


@pytest.mark.parametrize("dtype,keep", [(torch.bfloat16, None), (torch.float16, None), (torch.float16, "int8")])
def test_gradients_of_a_stack(tr, dtype, keep):
    """A gradient passes some 4 roundings of activations a block, half a step of the type each (2^-9 of the value in the mean, as
    they are spread evenly), and as many of its own: of a whole tensor, taken by its norm, they add up as errors of
    independent signs do, 8 (BLOCKS + 1) of them to below 6 * half a step; twice that is allowed, and for inputs kept in 8
    bits by int8 the 1 / 254 of a block's largest, three times its values' root mean square."""
    p, e, tokens, weight = parameters(dtype)
    low = {k: v.to(dtype) for k, v in p.items() if is_matrix(k)}
    exact = {k: (low[k].float() if k in low else v) for k, v in p.items()}
    loss, grads, de = step(tr, p, low, e, tokens, weight, keep)
    want_loss, want, want_e = definition(exact, e, tokens, weight)
    half = torch.finfo(dtype).eps / 2
    bound = 12 * half + (3 / 254 if keep else 0.0)
    assert abs(float(loss) / float(want_loss) - 1) < bound
    assert set(grads) == set(p)
    for k in p:
        off = float((grads[k].double() - want[k]).norm() / want[k].norm())
        assert grads[k].shape == p[k].shape and off < bound, (k, off)
    assert float((de.double() - want_e).norm() / want_e.norm()) < bound


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_and_their_replay(tr, bits):
    """Eager steps and a captured one, replayed with the step's number on the device, give the same bits; copies are the rounded
    parameters; the first update is the definition's."""
    p, e, tokens, weight = parameters(torch.bfloat16)
    names = list(p)
    copies = lambda q: {k: q[k].bfloat16() for k in names if is_matrix(k)}   # noqa: E731

    def state():
        q = {k: v.clone() for k, v in p.items()}
        return q, copies(q), [tr.zero_moments(q[k], bits) for k in names]

    decay = [0.01 if is_matrix(k) else 0.0 for k in names]

    def train(q, low, moments, number):
        loss, grads, _ = step(tr, q, low, e, tokens, weight, "int8")
        tr.moc_adamw_step([q[k] for k in names], [grads[k] for k in names], moments, 3e-3, number, weight_decay=decay, copies=[low.get(k) for k in names], seed=7)
        return loss, grads

    number = torch.ones(1, dtype=torch.int64, device="cuda")
    eager = state()
    before = {k: v.clone() for k, v in eager[0].items()}
    losses, first = [], None
    for t in range(1, 5):
        number.fill_(t)
        loss, grads = train(*eager, number)
        losses.append(float(loss))
        if t == 1:   # m / (1 - beta1) = g and v / (1 - beta2) = g^2: the sign of g, less what eps takes, and the decay
            for k, d in zip(names, decay):
                g = grads[k].double()
                want = before[k].double() * (1 - 3e-3 * d) - 3e-3 * g / (g.abs() + 1e-8)
                # lr and the corrections to 2^-21 of the update (32 half steps), the parameter's own rounding; where g is below 1e-15 its square leaves float32's range
                bound = 2.0 ** -19 * 3e-3 + 2.0 ** -23 * want.abs()
                assert bool((((eager[0][k].double() - want).abs() <= bound) | (g.abs() < 1e-15)).all()), k
    assert all(torch.equal(eager[1][k], eager[0][k].bfloat16()) for k in eager[1])
    assert all(math.isfinite(v) for v in losses)
    replayed = state()
    train(*[x if isinstance(x, list) else dict(x) for x in state()], number)   # whatever is loaded on first use
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, _ = train(*replayed, number)
    for t in range(1, 5):
        number.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert float(loss) == losses[t - 1]
    assert all(torch.equal(replayed[0][k], eager[0][k]) for k in names)
    for a, b in zip(replayed[2], eager[2]):
        assert torch.equal(a.m, b.m) and torch.equal(a.v, b.v)
