"""The operators that make a whole training step out of a plan's layers, as they are measured.

Three families, each in a plain form of elementary torch operations and through the public calls of
`paper_2304_14463_amd.training`:

* the residual connection: the norm behind a block, its gate, the scale of the stream and the norm before the next
  block in one pass, r = scale * x + gate * after(block), n = before(r), and the gradients of all of it;
* log probabilities of given tokens from a matrix of logits, with the entropy and the most likely alternatives, and
  the gradient with regard to the logits;
* a step of AdamW over many tensors, with moments in 32 bits or in 8.

`own` says which of the two `run` takes.  Moments in 8 bits are returned as the values they stand for.

Moments in 8 bits: 32 consecutive values of a tensor share the scale 2^k, held as the byte k + 127; k is the smallest
whole number, at least -111, for which the block's largest finite magnitude is at most 448 * 2^k.  First moments: a sign
and 4 exponent and 3 fraction bits (normal from 2^-6 on).  Second moments: 5 exponent and 3 fraction bits (normal from
2^-22 on).  The largest code of each is 448, the one above it NaN.  A value between two codes goes to the upper with a
probability of its distance from the lower, by 16 bits of a hash of the seed, the step, the tensor's number and the
value's place; a positive second moment takes no code below 1.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5
BLOCK = 32
MIN_EXP = -111
BETAS, ADAM_EPS, LR, DECAY = (0.9, 0.999), 1e-8, 3e-5, 0.01


def listed():
    return [
        # a token on its way through a deep model: the norm before the next block, all latency
        dict(name="residual 1x1000", op="residual_forward", rows=1, cols=1000, dtype="fp16", stream="fp16", gates=0, after="none", before="rms", scale=1.0, keep="none"),
        # a training batch between two blocks, everything on, the norm kept in 8 bits for the next layer's weight gradient
        dict(name="residual 32768x4096", op="residual_forward", rows=32768, cols=4096, dtype="bf16", stream="bf16", gates=1, after="rms", before="layer", scale=0.9, keep="e4m3"),
        # odd sizes, 17 sequences with a gate each, the block's output kept in 8 bits
        dict(name="residual grad 4998x1247 int8", op="residual_backward", rows=4998, cols=1247, dtype="fp16", stream="fp16", gates=17, after="layer", before="layer", scale=1.0, held="int8"),
        # a large batch of wide rows with a stream in full precision
        dict(name="residual grad 16384x8192", op="residual_backward", rows=16384, cols=8192, dtype="bf16", stream="fp32", gates=1, after="none", before="rms", scale=1.0, held="tensor"),
        # the next token's probabilities with the alternatives that an interface shows
        dict(name="logprob 1x131072 top 20", op="logprob_forward", rows=1, vocab=131072, dtype="bf16", top=20, scale=1.25),
        # a batch of scored tokens over an odd vocabulary
        dict(name="logprob 4999x32003 top 5", op="logprob_forward", rows=4999, vocab=32003, dtype="fp16", top=5, scale=1.0),
        # the loss of a training batch
        dict(name="logprob 8192x131072", op="logprob_forward", rows=8192, vocab=131072, dtype="bf16", top=0, scale=1.0),
        # the gradient of a small batch in full precision, with a bonus on the entropy
        dict(name="logprob grad 1247x32003", op="logprob_backward", rows=1247, vocab=32003, dtype="fp32", scale=0.8, entropy=True),
        # the gradient of a training batch
        dict(name="logprob grad 8192x131072", op="logprob_backward", rows=8192, vocab=131072, dtype="bf16", scale=1.0, entropy=False),
        # two tiny blocks: launches and little else
        dict(name="adamw 2 blocks of 64", op="adamw", blocks=2, width=64, inner=256, param="fp32", grad="fp32", copies=False, bits=32),
        # an ordinary model with odd sizes, parameters in 32 bits and their copies for the products
        dict(name="adamw 12 blocks of 1247", op="adamw", blocks=12, width=1247, inner=4999, param="fp32", grad="fp32", copies=True, bits=32),
        # a large model whose moments take 2 bytes a parameter instead of 8
        dict(name="adamw 16 blocks of 2048 8 bits", op="adamw", blocks=16, width=2048, inner=8192, param="fp32", grad="bf16", copies=True, bits=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _even(rng, value):
    """Half of all sizes as drawn, half as layers have them."""
    return value if rng.random() < 0.5 else max(64, value // 64 * 64)


def draw(rng):
    op = rng.choice(["residual_forward", "residual_backward", "logprob_forward", "logprob_backward", "adamw"])
    case = dict(op=op)
    if op.startswith("residual"):
        cols = _even(rng, _log(rng, 32, 16384))
        gates = rng.choice([0, 1, 1, 8, -1])   # -1: a gate for every row
        rows = _log(rng, 1, min(32768, (1 << 27) // cols))
        rows = -(-rows // 8) * 8 if gates == 8 else rows
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        case.update(rows=rows, cols=cols, dtype=dtype, stream=rng.choice([dtype, dtype, "fp32"]), gates=gates, after=rng.choice(["none", "none", "rms", "layer"]),
                    before=rng.choice(["rms", "layer", "layer"]), scale=rng.choice([1.0, 0.8125]))
        if op == "residual_forward":
            case.update(keep=rng.choice(["none", "e4m3", "int8"]))
        else:
            case.update(held=rng.choice(["tensor", "e4m3", "int8"]))
    elif op.startswith("logprob"):
        vocab = _even(rng, _log(rng, 1000, 262144))
        case.update(rows=_log(rng, 1, min(16384, (1 << 30) // vocab)), vocab=vocab, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), scale=rng.choice([1.0, 0.7, 1.5]))
        if op == "logprob_forward":
            case.update(top=rng.choice([0, 1, 5, 20, 64]))
        else:
            case.update(entropy=rng.random() < 0.5)
    else:
        width = _even(rng, _log(rng, 32, 4096))
        case.update(blocks=rng.randint(1, max(1, min(24, (1 << 29) // (8 * width * width)))), width=width, inner=_even(rng, 4 * width), param=rng.choice(["fp32", "fp32", "bf16"]),
                    grad=rng.choice(["fp32", "bf16", "fp16"]), bits=rng.choice([8, 8, 32]))
        case.update(copies=case["param"] == "fp32" and rng.random() < 0.7)
    return case


# ---- the plain form: the residual connection --------------------------------------------------------------------------


def _keep(x, fmt, dtype):
    """the float32 values that an 8-bit checkpoint of float32 values stands for, and its codes and scales"""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    padded = torch.nn.functional.pad(x, (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    m, e = torch.frexp(padded.abs().amax(2))          # magnitude = m * 2^e, 0.5 <= m < 1
    k = e - 9 + (m > 0.875).int() if fmt == "e4m3" else e - 7 + (m > 127 / 128).int()
    k = torch.where(m == 0, MIN_EXP, k).clamp(min=MIN_EXP).int()
    scale = _power(k)[:, :, None]
    q = padded / scale
    q = q.to(torch.float8_e4m3fn) if fmt == "e4m3" else torch.round(q).to(torch.int8)
    values = (q.float() * scale).view(rows, blocks * BLOCK)[:, :cols]
    return values, q.view(torch.uint8).view(rows, blocks * BLOCK)[:, :cols].contiguous(), (k + 127).to(torch.uint8)


def _power(k):
    """2^k of int32 exponents in -126..127, exactly"""
    return ((k + 127) << 23).view(torch.float32)


def _norm(x, kind, gamma, beta):
    """(norm of the rows, mean, 1 / deviation) in x's precision"""
    mean = x.sum(1) / x.shape[1] if kind == "layer" else None
    d = x - mean[:, None] if kind == "layer" else x
    rstd = 1 / torch.sqrt((d * d).sum(1) / x.shape[1] + EPS)
    h = d * rstd[:, None]
    return h * gamma + beta if beta is not None else h * gamma, mean, rstd


def _norm_grad(dy, x, kind, gamma, mean, rstd):
    """(dx, dgamma, dbeta)"""
    h = (x - mean[:, None] if kind == "layer" else x) * rstd[:, None]
    p = dy * gamma
    out = p - h * ((p * h).sum(1) / x.shape[1])[:, None]
    if kind == "layer":
        out = out - (p.sum(1) / x.shape[1])[:, None]
    return out * rstd[:, None], (dy * h).sum(0), dy.sum(0) if kind == "layer" else None


def _each_row(gate, rows):
    return gate.repeat_interleave(rows // gate.shape[0], 0) if gate.shape[0] > 1 else gate


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _stream(g, rows, cols, dtype):
    """activations as a residual stream has them: channels of different sizes, a few of them far larger"""
    wide = torch.exp(torch.randn(cols, generator=g, device="cuda") * 0.5)
    wide = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.004, 24.0, wide)
    shift = torch.randn(cols, generator=g, device="cuda") * 0.2 + 0.1
    return torch.randn(rows, cols, generator=g, device="cuda").mul_(wide).add_(shift).to(dtype)


def _normal(g, *shape, by=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda").mul_(by).to(dtype)


def _norm_parameters(g, kind, cols):
    if kind == "none":
        return None
    return dict(kind=kind, gamma=1 + _normal(g, cols, by=0.1), beta=_normal(g, cols, by=0.1) if kind == "layer" else None)


def _prepare_residual(s, g):
    rows, cols, dtype, stream = s["rows"], s["cols"], TYPES[s["dtype"]], TYPES[s["stream"]]
    s["block"] = _stream(g, rows, cols, dtype)
    gates = rows if s["gates"] < 0 else s["gates"]
    s["gate"] = 0.5 + _normal(g, gates, cols, by=0.3, dtype=torch.float32 if gates == 1 else dtype) if gates else None
    s["norms"] = {k: _norm_parameters(g, s[k], cols) for k in ("after", "before")}
    s["x"] = _stream(g, rows, cols, stream)
    if s["op"] == "residual_forward":
        return
    # what a forward pass has left: the block's output, as a tensor or in 8 bits, the stream and the statistics
    h = s["block"].float()
    s["kept"] = None
    if s["held"] != "tensor":
        h, codes, scales = _keep(h, s["held"], dtype)
        s["kept"] = (codes, scales)
    s["stats"] = {"after": None, "before": None}
    if s["norms"]["after"]:
        h, mean, rstd = _norm(h.double(), **s["norms"]["after"])
        s["stats"]["after"] = (None if mean is None else mean.float(), rstd.float())
    r = s["scale"] * s["x"].double() + (h if s["gate"] is None else _each_row(s["gate"], rows).double() * h)
    s["r"] = r.to(stream)
    _, mean, rstd = _norm(s["r"].double(), **s["norms"]["before"])
    s["stats"]["before"] = (None if mean is None else mean.float(), rstd.float())
    s["dr"], s["dn"] = _normal(g, rows, cols, by=0.02, dtype=stream), _normal(g, rows, cols, by=0.02, dtype=dtype)
    del s["x"]


def _prepare_logits(s, g):
    rows, vocab, dtype = s["rows"], s["vocab"], TYPES[s["dtype"]]
    wide = 1.5 + torch.rand(rows, 1, generator=g, device="cuda") * 2
    s["logits"] = torch.randn(rows, vocab, generator=g, device="cuda").mul_(wide).to(dtype)
    # some tokens are ruled out everywhere (a vocabulary padded to a round size), some in a row
    s["logits"][:, vocab - vocab // 100:] = -math.inf
    at = torch.randint(0, vocab - vocab // 100, (rows, 64), generator=g, device="cuda")
    s["logits"].scatter_(1, at[:, :32], -math.inf)
    tokens = at[:, 40].clone()
    s["logits"].scatter_(1, tokens[:, None], (torch.rand(rows, 1, generator=g, device="cuda") * 18 - 2).to(dtype))
    s["tokens"] = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.05, -1, tokens) if rows > 1 else tokens
    if s["op"] == "logprob_backward":
        x = s["logits"].float() * s["scale"]
        s["lse"] = torch.logsumexp(x, 1)
        p = torch.exp(x - s["lse"][:, None])
        s["entropy_of"] = s["lse"] - torch.where(p > 0, p * x, 0.0).sum(1, dtype=torch.float64).float() if s["entropy"] else None
        s["dlogp"] = _normal(g, rows)
        s["dentropy"] = _normal(g, rows, by=0.1) if s["entropy"] else None


def _shapes(s):
    w, inner = s["width"], s["inner"]
    return [(w,), (w,), (inner, w), (inner,), (w, inner), (w,)] * s["blocks"]


def _views(flat, shapes, at):
    return [flat[a:a + math.prod(shape)].view(shape) for a, shape in zip(at, shapes)]


def _prepare_adamw(s, g):
    """tensors as views of one buffer a kind: matrices and vectors of each block"""
    s["shapes"] = shapes = _shapes(s)
    s["ids"] = list(range(len(shapes)))
    s["step"], s["seed"] = 1000, int(torch.randint(0, 1 << 30, (1,), generator=g, device="cuda"))
    s["clip"] = 0.5 + 0.5 * torch.rand(1, generator=g, device="cuda")
    s["decay"] = [DECAY if len(shape) == 2 else 0.0 for shape in shapes]
    matrix, starts = [len(shape) == 2 for shape in shapes], {}
    room = {True: 0, False: 0}   # matrices and vectors apart, each tensor from a multiple of 32 values on
    for i, shape in enumerate(shapes):
        starts[i] = room[matrix[i]]
        room[matrix[i]] += -(-math.prod(shape) // BLOCK) * BLOCK

    def buffers(dtype, vector_dtype=torch.float32, per=1):
        return {kind: torch.zeros(room[kind] // per, dtype=dtype if kind else vector_dtype, device="cuda") for kind in (True, False)}

    def views(flat, per=1):
        return [_views(flat[matrix[i]], [shape], [starts[i]])[0] if per == 1 else flat[matrix[i]][starts[i] // per:starts[i] // per + -(-math.prod(shape) // per)]
                for i, shape in enumerate(shapes)]

    s["p"] = buffers(TYPES[s["param"]])
    s["params"] = views(s["p"])
    s["grads"] = views(buffers(TYPES[s["grad"]]))
    s["copy"] = buffers(torch.bfloat16, torch.bfloat16) if s["copies"] else None
    s["copied"] = [c if two else None for c, two in zip(views(s["copy"]), matrix)] if s["copies"] else None
    kind = torch.float32 if s["bits"] == 32 else torch.uint8
    s["m"], s["v"] = buffers(kind, kind), buffers(kind, kind)
    s["ms"], s["vs"] = views(s["m"]), views(s["v"])
    if s["bits"] == 8:
        s["msc"], s["vsc"] = views(buffers(torch.uint8, torch.uint8, BLOCK), BLOCK), views(buffers(torch.uint8, torch.uint8, BLOCK), BLOCK)
        s["m_values"], s["v_values"] = buffers(torch.bfloat16, torch.bfloat16), buffers(torch.bfloat16, torch.bfloat16)
        s["mv"], s["vv"] = views(s["m_values"]), views(s["v_values"])
    for i, shape in enumerate(shapes):
        wide = torch.exp(torch.randn(shape[-1], generator=g, device="cuda")) * 1e-3
        s["params"][i].copy_(_normal(g, *shape, by=0.03) if matrix[i] else 1 + _normal(g, *shape, by=0.1))
        grad = torch.randn(shape, generator=g, device="cuda").mul_(wide)
        s["grads"][i].copy_(grad)
        m, v = _normal(g, *shape, by=0.3).mul_(wide), (0.5 + torch.rand(shape, generator=g, device="cuda")).mul_(wide).mul_(wide)
        if s["bits"] == 32:
            s["ms"][i].copy_(m)
            s["vs"][i].copy_(v)
        else:
            half = torch.full((), 1 << 15, dtype=torch.int64, device="cuda")
            _store_moment(m.view(-1), half, s["ms"][i], s["msc"][i], False)
            _store_moment(v.view(-1), half, s["vs"][i], s["vsc"][i], True)


def prepare(case, seed):
    g, s = _gen(seed), dict(case)
    if case["op"].startswith("residual"):
        _prepare_residual(s, g)
    elif case["op"].startswith("logprob"):
        _prepare_logits(s, g)
    else:
        _prepare_adamw(s, g)
    return s


# ---- the plain form: moments in 8 bits --------------------------------------------------------------------------------


def _mix(h):
    """32 bits of an int64 tensor or number, well mixed"""
    h = h ^ (h >> 16)
    h = (h * 0xF704BB15) & 0xFFFFFFFF
    h = h ^ (h >> 15)
    h = (h * 0x371E2E67) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _random(seed, step, tensor, n):
    """the 32 random bits of each of n values"""
    key = _mix(_mix(_mix(_mix(seed & 0xFFFFFFFF) ^ (seed >> 32)) ^ (step & 0xFFFFFFFF)) ^ tensor)
    place = torch.arange(n, device="cuda")
    return _mix((place & 0xFFFFFFFF) ^ _mix((place >> 32) ^ key))


def _moment_table(second):
    """the values of the 256 codes"""
    c = torch.arange(256, device="cuda")
    low = c if second else c & 127
    first = -22 if second else -6
    v = torch.where(low < 8, low * 2.0 ** (first - 3), (8 + (low & 7)) * torch.exp2(((low >> 3) - 1 + first - 3).float()))
    v = torch.where(low == (255 if second else 127), math.nan, v)
    return v if second else torch.where(c >= 128, -v, v)


def _moment(codes, scales, second):
    return _moment_table(second)[codes.view(-1).long()] * _power(scales.int() - 127).repeat_interleave(BLOCK)[:codes.numel()]


def _store_moment(x, r, codes, scales, second):
    """float32 values, rounded by the random bits r (16 of them a value), into codes and scales"""
    n = x.numel()
    blocks = scales.numel()
    good = torch.isfinite(x)
    mag = torch.where(good, x.abs(), 0.0).clamp(max=1.875 * 2.0 ** 127)
    m, e = torch.frexp(torch.nn.functional.pad(mag, (0, blocks * BLOCK - n)).view(blocks, BLOCK).amax(1))
    k = torch.where(m == 0, MIN_EXP, e - 9 + (m > 0.875).int()).clamp(min=MIN_EXP).int()
    q = mag * _power(-k).repeat_interleave(BLOCK)[:n]
    first = -22 if second else -6
    small = q < 2.0 ** first
    bits = torch.where(small, q + 2.0 ** first, q).view(torch.int32).long() + (r * 16 + 8)
    c = (bits >> 20) - ((first + 127) << 3) + torch.where(small, 0, 8)
    if second:
        c = torch.where((x > 0) & (c < 1), 1, c)
    else:
        c = c + torch.where(torch.signbit(x), 128, 0)
    codes.view(-1).copy_(torch.where(good, c, 255 if second else 127))
    scales.copy_(k + 127)


def _adamw_tensor(s, i):
    p, grad = s["params"][i], s["grads"][i].float().view(-1) * s["clip"]
    m, v = (s["ms"][i].view(-1), s["vs"][i].view(-1)) if s["bits"] == 32 else (_moment(s["ms"][i], s["msc"][i], False), _moment(s["vs"][i], s["vsc"][i], True))
    m = BETAS[0] * m + (1 - BETAS[0]) * grad
    v = BETAS[1] * v + (1 - BETAS[1]) * (grad * grad)
    away = LR / (1 - BETAS[0] ** s["step"]) * m / (torch.sqrt(v / (1 - BETAS[1] ** s["step"])) + ADAM_EPS)
    old = p.float().view(-1)
    new = (old - (LR * s["decay"][i] * old + away)).view(p.shape)
    p.copy_(new)
    if s["copies"] and s["copied"][i] is not None:
        s["copied"][i].copy_(new)
    if s["bits"] == 32:
        s["ms"][i].view(-1).copy_(m)
        s["vs"][i].view(-1).copy_(v)
    else:
        r = _random(s["seed"], s["step"], i, m.numel())
        _store_moment(m, r & 0xFFFF, s["ms"][i], s["msc"][i], False)
        _store_moment(v, r >> 16, s["vs"][i], s["vsc"][i], True)
        s["mv"][i].view(-1).copy_(_moment(s["ms"][i], s["msc"][i], False))
        s["vv"][i].view(-1).copy_(_moment(s["vs"][i], s["vsc"][i], True))


def _adamw_outputs(s):
    out = dict(matrices=s["p"][True], vectors=s["p"][False])
    if s["copies"]:
        out["copies"] = s["copy"][True]
    m, v = (s["m"], s["v"]) if s["bits"] == 32 else (s["m_values"], s["v_values"])
    out.update(m=m[True], m_vectors=m[False], v=v[True], v_vectors=v[False])
    return out


# ---- one pass ---------------------------------------------------------------------------------------------------------


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    op = s["op"]
    if op == "residual_forward":
        dtype, out = TYPES[s["dtype"]], {}
        h = s["block"].float()
        if s["norms"]["after"]:
            h, out["after_mean"], out["after_rstd"] = _norm(h, **s["norms"]["after"])
        r = s["scale"] * s["x"].float() + (h if s["gate"] is None else _each_row(s["gate"].float(), s["rows"]) * h)
        n, out["before_mean"], out["before_rstd"] = _norm(r, **s["norms"]["before"])
        out.update(r=r.to(s["x"].dtype), n=n.to(dtype))
        if s["keep"] != "none":
            out["kept"] = _keep(n, s["keep"], dtype)[0].to(dtype)
        return out
    if op == "residual_backward":
        dtype, rows, out = TYPES[s["dtype"]], s["rows"], {}
        block = s["block"].float() if s["kept"] is None else _values(s)
        norm = s["norms"]["before"]
        d, out["before_gamma"], out["before_beta"] = _norm_grad(s["dn"].float(), s["r"].float(), norm["kind"], norm["gamma"], *s["stats"]["before"])
        d = d + s["dr"].float()
        h, norm = block, s["norms"]["after"]
        if norm:
            mean, rstd = s["stats"]["after"]
            h = (block - mean[:, None] if norm["kind"] == "layer" else block) * rstd[:, None] * norm["gamma"]
            h = h + norm["beta"] if norm["kind"] == "layer" else h
        dh = d
        if s["gate"] is not None:
            out["gate"] = (d * h).view(s["gate"].shape[0], -1, s["cols"]).sum(1)
            dh = d * _each_row(s["gate"].float(), rows)
        if norm:
            dh, out["after_gamma"], out["after_beta"] = _norm_grad(dh, block, norm["kind"], norm["gamma"], *s["stats"]["after"])
        out.update(x=(s["scale"] * d).to(s["dr"].dtype), block=dh.to(dtype))
        return out
    if op == "logprob_forward":
        raw = s["logits"].float()
        x = raw * s["scale"]
        top = x.amax(1)
        x = x - top[:, None]
        e = torch.exp(x)
        total = e.sum(1)
        log = torch.log(total)
        out = dict(entropy=log - torch.where(e > 0, e * x, 0.0).sum(1) / total, lse=top + log)
        tokens = s["tokens"]
        out["logp"] = torch.where(tokens < 0, 0.0, x.gather(1, tokens.clamp(min=0)[:, None])[:, 0] - log)
        if s["top"]:
            # by value, then by place: distinct whole numbers in that order
            bits = (raw + 0.0).view(torch.int32)
            order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + torch.arange(s["vocab"] - 1, -1, -1, device="cuda")
            best = s["vocab"] - 1 - (order.topk(s["top"], 1).values & 0xFFFFFFFF)
            out.update(top_tokens=best, top_logp=x.gather(1, best) - log[:, None])
        return out
    if op == "logprob_backward":
        x = s["logits"].float() * s["scale"] - s["lse"][:, None]
        p = torch.exp(x)
        there = s["tokens"] >= 0
        d = -p * torch.where(there, s["dlogp"], 0.0)[:, None]
        d.scatter_add_(1, s["tokens"].clamp(min=0)[:, None], torch.where(there, s["dlogp"], 0.0)[:, None])
        if s["entropy"]:
            d = d - s["dentropy"][:, None] * torch.where(p > 0, p * (x + s["entropy_of"][:, None]), 0.0)
        return (d * s["scale"]).to(s["logits"].dtype)
    s["step"] += 1
    [_adamw_tensor(s, i) for i in s["ids"]]
    return _adamw_outputs(s)


def _values(s):
    """float32 values of the block's output that is held in 8 bits"""
    codes, scales = s["kept"]
    v = codes.view(torch.float8_e4m3fn).float() if s["held"] == "e4m3" else codes.view(torch.int8).float()
    return v * _power(scales.int() - 127).repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def _run_own(s):
    from paper_2304_14463_amd import training as tr
    op = s["op"]
    if op.startswith("residual"):
        after, before = (n and tr.Norm(n["kind"], n["gamma"], n["beta"], EPS) for n in (s["norms"]["after"], s["norms"]["before"]))
    if op == "residual_forward":
        got = tr.moc_residual_forward(s["x"], s["block"], gate=s["gate"], scale=s["scale"], after=after, before=before, keep=None if s["keep"] == "none" else s["keep"])
        out = dict(r=got.r, n=got.n, before_mean=got.before[0], before_rstd=got.before[1])
        if after:
            out.update(after_mean=got.after[0], after_rstd=got.after[1])
        if got.kept is not None:
            out["kept"] = tr.moc_checkpoint_read(got.kept, got.n.dtype)
        return out
    if op == "residual_backward":
        block = s["block"] if s["kept"] is None else tr.Checkpoint(*s["kept"], s["held"])
        got = tr.moc_residual_backward(s["dr"], s["dn"], s["r"], block, gate=s["gate"], scale=s["scale"], after=after, after_stats=s["stats"]["after"], before=before,
                                       before_stats=s["stats"]["before"], dtype=TYPES[s["dtype"]])
        out = dict(x=got.dx, block=got.dblock, before_gamma=got.before_gamma, before_beta=got.before_beta)
        if s["gate"] is not None:
            out["gate"] = got.gate
        if after:
            out.update(after_gamma=got.after_gamma, after_beta=got.after_beta)
        return out
    if op == "logprob_forward":
        got = tr.moc_logprob_forward(s["logits"], s["tokens"], scale=s["scale"], top=s["top"])
        out = dict(logp=got.logp, lse=got.lse, entropy=got.entropy)
        if s["top"]:
            out.update(top_tokens=got.top_tokens, top_logp=got.top_logp)
        return out
    if op == "logprob_backward":
        return tr.moc_logprob_backward(s["logits"], s["lse"], s["tokens"], s["dlogp"], entropy=s["entropy_of"], dentropy=s["dentropy"], scale=s["scale"])
    s["step"] += 1
    moments = [tr.Moments(m, v) for m, v in zip(s["ms"], s["vs"])] if s["bits"] == 32 else [tr.Moments(*x) for x in zip(s["ms"], s["vs"], s["msc"], s["vsc"])]
    tr.moc_adamw_step(s["params"], s["grads"], moments, LR, s["step"], betas=BETAS, eps=ADAM_EPS, weight_decay=s["decay"], copies=s["copied"], grad_scale=s["clip"], seed=s["seed"])
    if s["bits"] == 8:
        tr.moc_moments_read(moments, out=list(zip(s["mv"], s["vv"])))
    return _adamw_outputs(s)


def work(case):
    op = case["op"]
    size = {"fp32": 4, "bf16": 2, "fp16": 2}
    if op.startswith("residual"):
        rows, cols = case["rows"], case["cols"]
        n, d, t = rows * cols, size[case["dtype"]], size[case["stream"]]
        gates = rows if case["gates"] < 0 else case["gates"]
        gate = gates * cols * (4 if gates == 1 else d)
        norms = sum({"none": 0, "rms": 1, "layer": 2}[case[k]] for k in ("after", "before"))
        if op == "residual_forward":
            kept = 0 if case["keep"] == "none" else 2 * rows * (cols + -(-cols // BLOCK)) + n * d
            return dict(bytes=2 * n * (d + t) + kept + gate + norms * 4 * (rows + cols), flops=16 * n)
        reads = 0 if case["gates"] == 0 and case["after"] == "none" else rows * (cols + -(-cols // BLOCK)) if case["held"] != "tensor" else n * d
        return dict(bytes=n * (2 * d + 3 * t) + reads + gate + 4 * gates * cols + norms * 4 * (rows + 2 * cols), flops=30 * n)
    if op.startswith("logprob"):
        n, d, rows = case["rows"] * case["vocab"], size[case["dtype"]], case["rows"]
        if op == "logprob_forward":
            return dict(bytes=n * d + rows * (20 + 12 * case["top"]), flops=6 * n)
        return dict(bytes=2 * n * d + 24 * rows, flops=(8 if case["entropy"] else 4) * n)
    n = sum(math.prod(shape) for shape in _shapes(case))
    matrices = sum(math.prod(shape) for shape in _shapes(case) if len(shape) == 2)
    vectors = n - matrices
    moments = 16 * n if case["bits"] == 32 else 4 * (n + n // BLOCK) + 2 * (n + n // BLOCK) + 4 * n
    return dict(bytes=matrices * (2 * size[case["param"]] + size[case["grad"]] + (2 if case["copies"] else 0)) + 12 * vectors + moments, flops=20 * n)


# ---- from the definitions, in 64 bits ---------------------------------------------------------------------------------


def _grid(fmt):
    """the magnitudes of a format's codes in rising order: place = code"""
    if fmt == "int8":
        return torch.arange(128, dtype=torch.float64, device="cuda")
    first, last = {"e4m3": (-6, 8), "second": (-22, 8)}[fmt]
    t = [m / 8 * 2.0 ** first for m in range(8)]
    for e in range(first, last + 1):
        t += [(1 + m / 8) * 2.0 ** e for m in range(8)]
    return torch.tensor(t[:-1], dtype=torch.float64, device="cuda")


def _block_scales(mag, top):
    """2^k of each block of 32 in the last dimension"""
    wide = torch.zeros(*mag.shape[:-1], -(-mag.shape[-1] // BLOCK) * BLOCK, dtype=torch.float64, device="cuda")
    wide[..., :mag.shape[-1]] = mag
    peak = wide.unflatten(-1, (-1, BLOCK)).amax(-1)
    k = torch.ceil(torch.log2(torch.where(peak > 0, peak / top, 2.0 ** MIN_EXP))).clamp(min=MIN_EXP)
    k = torch.where(peak > top * torch.exp2(k), k + 1, k)   # the logarithm is only a guess next to a whole number
    k = torch.where((k > MIN_EXP) & (peak <= top * torch.exp2(k - 1)), k - 1, k)
    return torch.exp2(k).repeat_interleave(BLOCK, -1)[..., :mag.shape[-1]]


def _kept_exactly(x, fmt):
    """what a checkpoint of finite values stands for: the nearest of the format's"""
    grid, out = _grid(fmt), torch.empty_like(x)
    between = (grid[1:] + grid[:-1]) / 2
    for r in range(0, x.shape[0], max(1, (1 << 24) // x.shape[1])):
        part = x[r:r + max(1, (1 << 24) // x.shape[1])]
        scale = _block_scales(part.abs(), 448.0 if fmt == "e4m3" else 127.0)
        v = part.abs() / scale
        place = torch.bucketize(v, between)
        on = (place < len(between)) & (v == between[place.clamp(max=len(between) - 1)])   # a border goes to the even code
        place = place + (on & (place % 2 == 1)).long()
        out[r:r + part.shape[0]] = torch.copysign(grid[place] * scale, part)
    return out


def _moment_exactly(x, r, second):
    """what finite values, rounded up where their share of the way reaches what the random 16 bits leave, stand for"""
    grid = _grid("second" if second else "e4m3")
    scale = _block_scales(x.abs(), 448.0)
    q = x.abs() / scale
    low = (torch.bucketize(q, grid, right=True) - 1).clamp(max=len(grid) - 2)
    share = (q - grid[low]) / (grid[low + 1] - grid[low])
    up = torch.floor(share * 2.0 ** 20) + r.double() * 16 + 8 >= 2.0 ** 20
    place = low + up.long()
    place = torch.where((x > 0) & (place < 1), 1, place) if second else place
    return torch.copysign(grid[place] * scale, x)


def _held_exactly(s):
    codes, scales = s["kept"]
    grid = torch.cat([_grid("e4m3"), _grid("e4m3")[:1]]) if s["held"] == "e4m3" else _grid("int8")
    c = codes.long()
    v = torch.where(c >= 128, -grid[c & 127], grid[c & 127]) if s["held"] == "e4m3" else torch.where(c > 127, c - 256, c).double()
    return v * torch.exp2(scales.double() - 127)[:, torch.arange(codes.shape[1], device="cuda") // BLOCK]


def _exact_norm(x, norm):
    layer = norm["kind"] == "layer"
    mean = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    rstd = ((x - mean).square().mean(1, keepdim=True) + EPS).pow(-0.5)
    y = (x - mean) * rstd * norm["gamma"].double()
    return y + norm["beta"].double() if layer else y, mean[:, 0] if layer else None, rstd[:, 0]


def _exact_norm_grad(dy, x, norm, stats):
    layer = norm["kind"] == "layer"
    h = (x - stats[0].double()[:, None] if layer else x) * stats[1].double()[:, None]
    p = dy * norm["gamma"].double()
    dx = p - h * (p * h).mean(1, keepdim=True)
    if layer:
        dx -= p.mean(1, keepdim=True)
    return dx * stats[1].double()[:, None], torch.einsum("ij,ij->j", dy, h), dy.sum(0) if layer else None


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("residual"):
        after, before, rows = s["norms"]["after"], s["norms"]["before"], case["rows"]
        gate = 1.0 if s["gate"] is None else s["gate"].double()[torch.arange(rows, device="cuda") // (rows // s["gate"].shape[0])]
    if op == "residual_forward":
        out, h = {}, s["block"].double()
        if after:
            h, out["after_mean"], out["after_rstd"] = _exact_norm(h, after)
        out["r"] = case["scale"] * s["x"].double() + gate * h
        out["n"], out["before_mean"], out["before_rstd"] = _exact_norm(out["r"], before)
        if case["keep"] != "none":
            out["kept"] = _kept_exactly(out["n"], case["keep"])
        return out
    if op == "residual_backward":
        out, block = {}, s["block"].double() if s["kept"] is None else _held_exactly(s)
        d, out["before_gamma"], out["before_beta"] = _exact_norm_grad(s["dn"].double(), s["r"].double(), before, s["stats"]["before"])
        d += s["dr"].double()
        h = block
        if after:
            mean, rstd = s["stats"]["after"]
            h = (block - (0.0 if mean is None else mean.double()[:, None])) * rstd.double()[:, None] * after["gamma"].double() + (0.0 if after["beta"] is None else after["beta"].double())
        out.update(x=case["scale"] * d, block=d * gate)
        if s["gate"] is not None:
            out["gate"] = torch.stack([part.sum(0) for part in (d * h).chunk(s["gate"].shape[0])]) if s["gate"].shape[0] < rows else d * h
        if after:
            out["block"], out["after_gamma"], out["after_beta"] = _exact_norm_grad(out["block"], block, after, s["stats"]["after"])
        return out
    if op == "logprob_forward":
        parts, step = [], max(1, (1 << 27) // case["vocab"])
        for a in range(0, case["rows"], step):
            x = s["logits"][a:a + step].double() * case["scale"]
            lse = torch.logsumexp(x, 1)
            logp = torch.log_softmax(x, 1)
            tokens = s["tokens"][a:a + step]
            part = dict(lse=lse, entropy=torch.special.entr(logp.exp()).sum(1), logp=torch.where(tokens < 0, 0.0, logp[torch.arange(len(tokens), device="cuda"), tokens.clamp(min=0)]))
            if case["top"]:
                best = torch.sort(s["logits"][a:a + step].float(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
                part.update(top_tokens=best, top_logp=logp.gather(1, best))
            parts.append(part)
        return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if op == "logprob_backward":
        out, step = torch.empty(case["rows"], case["vocab"], dtype=torch.float64, device="cuda"), max(1, (1 << 27) // case["vocab"])
        for a in range(0, case["rows"], step):
            x = s["logits"][a:a + step].double() * case["scale"] - s["lse"][a:a + step].double()[:, None]
            p, tokens = x.exp(), s["tokens"][a:a + step]
            dlogp = torch.where(tokens < 0, 0.0, s["dlogp"][a:a + step].double())
            one = torch.nn.functional.one_hot(tokens.clamp(min=0), case["vocab"]).double()
            d = dlogp[:, None] * (one - p)
            if case["entropy"]:
                d -= s["dentropy"][a:a + step].double()[:, None] * torch.nan_to_num(p * (x + s["entropy_of"][a:a + step].double()[:, None]), nan=0.0)
            out[a:a + step] = case["scale"] * d
        return out
    out = {k: torch.zeros(v.shape, dtype=torch.float64, device="cuda") for k, v in _adamw_outputs(s).items()}
    t, at = s["step"] + 1, {True: 0, False: 0}
    for i, shape in enumerate(s["shapes"]):
        n, two = math.prod(shape), len(shape) == 2
        here = slice(at[two], at[two] + n)
        at[two] += -(-n // BLOCK) * BLOCK
        g = s["grads"][i].double().view(-1) * s["clip"].double()
        if s["bits"] == 32:
            m, v = s["ms"][i].double().view(-1), s["vs"][i].double().view(-1)
        else:
            scales = [torch.exp2(x.double() - 127)[torch.arange(n, device="cuda") // BLOCK] for x in (s["msc"][i], s["vsc"][i])]
            c, grid = s["ms"][i].view(-1).long(), _grid("e4m3")
            m = torch.where(c >= 128, -grid[c & 127], grid[c & 127]) * scales[0]
            v = _grid("second")[s["vs"][i].view(-1).long()] * scales[1]
        m = torch.lerp(g, m, BETAS[0])
        v = torch.lerp(g.square(), v, BETAS[1])
        p = s["params"][i].double().view(-1)
        p = p * (1 - LR * s["decay"][i]) - LR * (m / (1 - BETAS[0] ** t)) / ((v / (1 - BETAS[1] ** t)).sqrt() + ADAM_EPS)
        out["matrices" if two else "vectors"][here] = p
        if two and case["copies"]:
            out["copies"][here] = p
        if s["bits"] == 8:
            r = _random(s["seed"], t, i, n)
            m, v = _moment_exactly(m, r & 0xFFFF, False), _moment_exactly(v, r >> 16, True)
        out["m" if two else "m_vectors"][here] = m
        out["v" if two else "v_vectors"][here] = v
    return out
