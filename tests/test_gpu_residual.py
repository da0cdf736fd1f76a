"""The residual connection and its gradients against their definition in 64 bits.

Tolerances come from running_error: every operation's half step of float32, carried through the formula.  A row's sum is at most 16
values of a lane, six steps over a wave and four over waves, one after the other: 32 additions; 64 are allowed.  A column's is a
workgroup's rows and the workgroups: at most the rows and 64."""
import math
import zlib

import pytest
import torch

import training_reference as ref
from paper_2304_14463_amd.moccasin import MoccasinError
from running_error import Near, check
from training_reference import Framed, TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2304_14463_amd import training
    training.lib()
    return training


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def normal(g, *shape, by=1.0):
    return torch.randn(*shape, generator=g, dtype=torch.float64) * by


def norm(x, kind, gamma, beta, eps):
    """(norm, mean, rstd, normalised) of a Near; mean None without one"""
    n = x.v.shape[1]
    mean = x.sum(1, 64).over(n) if kind == "layer" else None
    d = x - mean.col() if mean else x
    rstd = ((d * d).sum(1, 64).over(n) + Near(eps)).inverse_root()
    h = d * rstd.col()
    y = h * gamma if gamma else h
    return y + beta if beta else y, mean, rstd


def norm_grad(dy, x, kind, gamma, mean, rstd):
    """(dx, dgamma, dbeta)"""
    n, rows = x.v.shape[1], x.v.shape[0]
    h = (x - mean.col() if mean else x) * rstd.col()
    p = dy * gamma if gamma else dy
    out = p - h * (p * h).sum(1, 64).over(n).col()
    if kind == "layer":
        out = out - p.sum(1, 64).over(n).col()
    return out * rstd.col(), (dy * h).sum(0, rows + 64), dy.sum(0, rows + 64)


def each_row(gate, rows):
    at = torch.arange(rows) // (rows // gate.v.shape[0])
    return Near(gate.v[at], gate.e[at])


class Case:
    """Operands of one call and what the definition says of them."""

    def __init__(self, tr, rows, cols, block, stream, held="tensor", gates=0, after=None, before="layer", x=True, scale=0.75, ptype=torch.float32, lead=0, pad=0):
        self.tr, self.rows, self.cols, self.after, self.before, self.gates, self.lead, self.pad = tr, rows, cols, after, before, gates, lead, pad
        self.block_type, self.stream_type, self.held, self.scale = TYPES[block], TYPES[stream], held, scale
        g = self.g = gen(rows, cols, block, stream, held, gates, after, before, lead)
        self.eps = {"after": 1e-5, "before": 1e-3}
        b = (normal(g, rows, cols) * torch.exp(0.5 * normal(g, cols)) + normal(g, rows, 1)).to(self.block_type)
        if held == "tensor":
            self.block = self.framed(b)
            self.b = Near(b)
        else:
            codes, scales = ref.keep(b.double(), held, self.block_type)
            self.block = tr.Checkpoint(self.framed(codes), self.framed(scales), held)
            self.b = Near(ref.values(codes, scales, held))
        xs = normal(g, rows, cols, by=2.0).to(self.stream_type)
        self.x, self.x_near = (self.framed(xs), Near(xs)) if x else (None, None)
        gate = (0.5 + normal(g, max(gates, 1), cols)).to(ptype)
        self.gate, self.gate_near = (self.framed(gate), Near(gate)) if gates else (None, None)
        self.params, self.near = {}, {}
        for k, kind in (("after", after), ("before", before)):
            gamma, beta = (1 + 0.1 * normal(g, cols)).to(ptype), (0.1 * normal(g, cols)).to(ptype)
            beta = beta if kind == "layer" else None
            self.params[k] = tr.Norm(kind, gamma.cuda(), None if beta is None else beta.cuda(), self.eps[k]) if kind else None
            self.near[k] = (Near(gamma), None if beta is None else Near(beta))

    def framed(self, x):
        f = Framed(*x.shape, x.dtype, self.lead, self.pad)
        return f.of(x)

    def definition(self):
        h, out = self.b, {}
        if self.after:
            h, *out["after"] = norm(h, self.after, *self.near["after"], self.eps["after"])
        if self.gates:
            h = each_row(self.gate_near, self.rows) * h
        r = Near(float(torch.tensor(self.scale))) * self.x_near + h if self.x is not None else h
        out["r"] = r
        if self.before:
            out["n"], *out["before"] = norm(r, self.before, *self.near["before"], self.eps["before"])
        return out

    def forward(self, **more):
        return self.tr.moc_residual_forward(self.x, self.block, gate=self.gate, scale=self.scale, after=self.params["after"], before=self.params["before"], **more)

    def gradients(self, r, stats, dr, dn):
        """of the stream r as it is held and the statistics as they are"""
        out, rows = {}, self.rows
        near_stats = {k: [Near(s.cpu()) if s is not None else None for s in stats[k]] if stats[k] else None for k in stats}
        d = None
        if self.before:
            d, out["before_gamma"], out["before_beta"] = norm_grad(dn, r, self.before, self.near["before"][0], *near_stats["before"])
        d = dr if d is None else d + dr if dr else d
        out["dx"] = Near(float(torch.tensor(self.scale))) * d
        y, dh = self.b, d
        if self.after:
            mean, rstd = near_stats["after"]
            y = (self.b - mean.col() if mean else self.b) * rstd.col() * self.near["after"][0]
            y = y + self.near["after"][1] if self.after == "layer" else y
        if self.gates:
            own = d * y
            each = rows // self.gates
            parts = Near(own.v.view(self.gates, each, -1), own.e.view(self.gates, each, -1))
            out["gate"] = parts.sum(1, each + 64)
            dh = d * each_row(self.gate_near, rows)
        if self.after:
            dh, out["after_gamma"], out["after_beta"] = norm_grad(dh, self.b, self.after, self.near["after"][0], *near_stats["after"])
        out["dblock"] = dh
        for k in ("after", "before"):
            if getattr(self, k) != "layer":
                out.pop(k + "_beta", None)
        return out


COLS = [1, 2, 31, 64, 512, 513, 1000, 1247, 2050, 4096, 5000, 8200, 16384]
KINDS = [dict(block="bf16", stream="bf16", after="rms", before="layer", gates=1),
         dict(block="fp16", stream="fp16", after=None, before="rms", gates=0, lead=1, pad=3),
         dict(block="bf16", stream="fp32", after="layer", before="rms", gates=3, ptype=torch.bfloat16, lead=1, pad=5),
         dict(block="fp16", stream="fp16", held="int8", after="layer", before="layer", gates=6),
         dict(block="bf16", stream="bf16", held="e4m3", after=None, before="layer", gates=2, lead=3, pad=1),
         dict(block="fp32", stream="fp32", after="rms", before="rms", gates=6, x=False),
         dict(block="fp32", stream="bf16", after="layer", before=None, gates=1),
         dict(block="bf16", stream="fp32", after=None, before="rms", gates=6),
         dict(block="bf16", stream="fp32", held="int8", after="rms", before="layer", gates=6, lead=1, pad=7),
         dict(block="bf16", stream="bf16", after=None, before="layer", gates=0),
         dict(block="bf16", stream="bf16", after=None, before=None, gates=2, scale=1.0, ptype=torch.float16, lead=1, pad=1)]
IDS = ["-".join(str(v) for v in k.values() if not isinstance(v, torch.dtype)) for k in KINDS]


def check_forward(case, got, want, fmt=None):
    if got.r is not None:
        check(got.r, want["r"])
    for k in ("after", "before"):
        stats = getattr(got, k)
        assert (stats is None) == (k not in want)
        if stats:
            assert (stats[0] is None) == (want[k][0] is None)
            if stats[0] is not None:
                check(stats[0], want[k][0])
            check(stats[1], want[k][1])
    if "n" in want:
        check(got.n, want["n"])
    if fmt:   # of n before its rounding: half a step of the code, and what is next to a border
        n = want["n"]
        kv = ref.values(got.kept.codes, got.kept.scales, fmt)
        wide = torch.exp2(got.kept.scales.cpu().double() - 127).repeat_interleave(32, 1)[:, :case.cols]
        step = torch.maximum(n.v.abs() * 2.0 ** -4, wide * 2.0 ** -10) if fmt == "e4m3" else wide / 2
        assert bool(((kv - n.v).abs() <= step * (1 + 2.0 ** -10) + n.e).all())


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_forward(tr, cols, kind):
    case = Case(tr, 6, cols, **kind)
    want = case.definition()
    out = Framed(6, cols, case.stream_type if case.x is not None else case.block_type, case.lead, case.pad)
    more, fmt = {}, None
    if case.before:
        fmt = "e4m3" if cols % 2 else "int8"
        on = Framed(6, cols, case.block_type, case.lead, case.pad)
        fc, fs = Framed(6, cols, torch.uint8, case.lead, case.pad), Framed(6, -(-cols // 32), torch.uint8, case.lead, case.pad)
        more = dict(out_norm=on.inner, keep=tr.Checkpoint(fc.inner, fs.inner, fmt))
    got = case.forward(out=out.inner, **more)
    assert got.r is out.inner and out.intact()
    if case.before:
        assert got.n is on.inner and on.intact() and fc.intact() and fs.intact()
    check_forward(case, got, want, fmt)
    again = case.forward(dtype=case.block_type)   # a Checkpoint's own default is x's type
    assert torch.equal(again.r, got.r) and again.kept is None and (not case.before or torch.equal(again.n, got.n))
    if case.before:
        alone = case.forward(want_stream=False, dtype=torch.float32)
        assert alone.r is None and alone.n.dtype == torch.float32
        check(alone.n, want["n"])
        assert torch.equal(alone.before[1], got.before[1])


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_backward(tr, cols, kind):
    check_backward(tr, 6, cols, kind)


@pytest.mark.parametrize("rows,cols", [(1, 1000), (3000, 64), (4998, 33), (2002, 1247), (600, 4096)])
@pytest.mark.parametrize("gates", [0, 1, 2, 7, -2, -1])
def test_backward_over_many_rows(tr, rows, cols, gates):
    """Workgroups of many rows, gates of many workgroups and workgroups of many gates (-2: a gate for two rows, -1: for one)."""
    gates = gates if gates >= 0 else rows // -gates
    if gates < 1 or rows % gates:
        gates = min(gates, 1)
    check_backward(tr, rows, cols, dict(block="bf16", stream="bf16", after="layer", before="layer", gates=gates))


def check_backward(tr, rows, cols, kind):
    kind = dict(kind)
    if kind.get("gates", 0) > rows:
        kind["gates"] = 1
    case = Case(tr, rows, cols, **kind)
    f = case.forward(dtype=case.block_type)
    g = case.g
    stats = dict(after=f.after, before=f.before)
    for held, whole in (("tensor", True), ("tensor", False), ("e4m3", False)):
        r = f.r if held == "tensor" else tr.moc_checkpoint_write(f.r, held)
        r_near = Near(f.r.cpu()) if held == "tensor" else Near(ref.values(r.codes, r.scales, held))
        stream_type = f.r.dtype
        dr = normal(g, rows, cols, by=0.1).to(stream_type) if whole or not case.before else None
        dn = normal(g, rows, cols, by=0.3).to(case.block_type) if case.before else None
        want = case.gradients(r_near, stats, Near(dr) if dr is not None else None, Near(dn) if dn is not None else None)
        ox, ob = Framed(rows, cols, stream_type, case.lead, case.pad), Framed(rows, cols, case.block_type, case.lead, case.pad)
        dr, dn = (None if t is None else case.framed(t) for t in (dr, dn))
        args = dict(gate=case.gate, scale=case.scale, after=case.params["after"], after_stats=f.after, before=case.params["before"], before_stats=f.before, dtype=case.block_type)
        got = tr.moc_residual_backward(dr, dn, r, case.block, out_x=ox.inner, out_block=ob.inner, **args)
        assert got.dx is ox.inner and got.dblock is ob.inner and ox.intact() and ob.intact()
        for name, value in got._asdict().items():
            assert (value is None) == (name not in want), name
            if value is not None:
                check(value, want[name])
        again = tr.moc_residual_backward(dr, dn, r, case.block, want_x=False, want_params=False, **args)
        assert torch.equal(again.dblock, got.dblock) and all(v is None for k, v in again._asdict().items() if k != "dblock")
        if whole and case.held == "tensor":
            # over the operands, where types allow it
            a, b = case.framed(dr), case.framed(case.block)
            over = tr.moc_residual_backward(a, dn, r, b, out_x=a, out_block=b, **args)
            assert over.dx is a and over.dblock is b
            assert all(torch.equal(v, w) for v, w in zip(over, got) if v is not None)
            if case.before:
                a, b = case.framed(f.r), case.framed(dn)
                over = tr.moc_residual_backward(dr, b, a, case.block, out_x=a, out_block=b, **args)
                assert all(torch.equal(v, w) for v, w in zip(over, got) if v is not None)


@pytest.mark.parametrize("cols", [33, 1001, 1247, 2049, 4097, 4096])
def test_forward_over_its_operands(tr, cols):
    """A ragged row's last run is loaded whole from within the row where nothing is written over it, and in parts where it is."""
    for kind in (dict(block="bf16", stream="bf16", after=None, before=None, gates=1), dict(block="fp16", stream="fp16", after="rms", before="layer", gates=0)):
        case = Case(tr, 300, cols, **kind)
        want = case.forward()
        for over in ("x", "block"):
            x, b = case.x.clone(), case.block.clone()
            other = {} if not case.before else dict(out_norm=b if over == "x" else x)
            got = tr.moc_residual_forward(x, b, gate=case.gate, scale=case.scale, after=case.params["after"], before=case.params["before"], out=x if over == "x" else b, **other)
            assert torch.equal(got.r, want.r) and (not case.before or torch.equal(got.n, want.n))


def test_norm_alone_and_streams_alone(tr):
    """Without x and gate it is a norm by the root of the squares of what is there; with one norm before a block only, a layer norm
    gives what moc_norm_forward gives of the float32 sum."""
    g = gen("alone")
    e = normal(g, 50, 1000).float().cuda()
    gamma = (1 + 0.1 * normal(g, 1000)).float().cuda()
    got = tr.moc_residual_forward(None, e, before=tr.Norm("rms", gamma), want_stream=False)
    want, _, rstd = norm(Near(e.cpu()), "rms", Near(gamma.cpu()), None, 1e-5)
    check(got.n, want)
    check(got.before[1], rstd)
    assert got.r is None and got.before[0] is None and got.after is None
    d = tr.moc_residual_backward(None, e, e, before=tr.Norm("rms", gamma), before_stats=got.before, want_x=False)
    dx, dgamma, _ = norm_grad(Near(e.cpu()), Near(e.cpu()), "rms", Near(gamma.cpu()), None, Near(got.before[1].cpu()))
    check(d.dblock, dx)
    check(d.before_gamma, dgamma)
    x = normal(g, 50, 1000).float().cuda()
    n = tr.moc_residual_forward(x, e, before=tr.Norm("layer"))
    y, mean, rstd, _ = tr.moc_norm_forward(n.r)
    assert torch.equal(n.r, x + e) and float((n.n - y).abs().max()) < 1e-5 and float((n.before[0] - mean).abs().max()) < 1e-6
    one = tr.moc_residual_forward(x, e, gate=gamma)   # a vector is the gate of all rows
    assert torch.equal(one.r, tr.moc_residual_forward(x, e, gate=gamma[None]).r) and one.n is None


def test_gradients_against_differences(tr):
    """Central differences of the definition in 64 bits, steps of 1e-6: off by some 1e-9 here; the kernels' by below 1e-5 of the
    largest."""
    g = gen("differences")
    rows, cols = 4, 24
    t = {k: normal(g, *s).float().double() for k, s in dict(x=(rows, cols), block=(rows, cols), gate=(2, cols), ga=(cols,), be=(cols,), gb=(cols,)).items()}
    wr, wn = normal(g, rows, cols).float().double(), normal(g, rows, cols).float().double()

    def value(t):
        b = t["block"]
        d = b - b.mean(1, keepdim=True)
        h = d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * t["ga"] + t["be"]
        r = 0.75 * t["x"] + t["gate"].repeat_interleave(2, 0) * h
        return ((r * wr) + r / (r.square().mean(1, keepdim=True) + 1e-5).sqrt() * t["gb"] * wn).sum()

    c = {k: v.float().cuda() for k, v in t.items()}
    after, before = tr.Norm("layer", c["ga"], c["be"]), tr.Norm("rms", c["gb"])
    f = tr.moc_residual_forward(c["x"], c["block"], c["gate"], 0.75, after, before)
    got = tr.moc_residual_backward(wr.float().cuda(), wn.float().cuda(), f.r, c["block"], c["gate"], 0.75, after, f.after, before, f.before)
    got = dict(x=got.dx, block=got.dblock, gate=got.gate, ga=got.after_gamma, be=got.after_beta, gb=got.before_gamma)
    for name, grad in got.items():
        slopes = torch.zeros_like(t[name])
        for i in range(slopes.numel()):
            step = torch.zeros(slopes.numel(), dtype=torch.float64)
            step[i] = 1e-6
            up, down = (value({**t, name: t[name] + s * step.view(slopes.shape)}) for s in (1, -1))
            slopes.view(-1)[i] = (up - down) / 2e-6
        assert float((slopes - grad.cpu().double()).abs().max()) < 1e-5 * max(1.0, float(slopes.abs().max())), name


def test_rows_that_are_not_finite_keep_to_themselves(tr):
    for cols in (100, 1000, 3000):
        x, b, gate = torch.randn(9, cols, device="cuda"), torch.randn(9, cols, device="cuda"), torch.randn(3, cols, device="cuda")
        x[2, 7], b[5, -1] = math.nan, math.inf
        gamma = torch.ones(cols, device="cuda")
        f = tr.moc_residual_forward(x, b, gate, after=tr.Norm("rms", gamma), before=tr.Norm("layer", gamma, gamma), keep="int8")
        bad = torch.zeros(9, dtype=torch.bool, device="cuda")
        bad[2] = bad[5] = True
        assert bool(f.n[bad].isnan().all()) and bool(f.n[~bad].isfinite().all()) and bool(f.r[2].isnan().sum() == 1)
        back = tr.moc_checkpoint_read(f.kept, torch.float32)
        assert torch.equal(back.isnan(), f.n.isnan())
        d = tr.moc_residual_backward(x, b, f.r, b, gate, after=tr.Norm("rms", gamma), after_stats=f.after, before=tr.Norm("layer", gamma, gamma), before_stats=f.before)
        assert bool(d.dx[~bad].isfinite().all()) and bool(d.dx[2].isnan().all()) and bool(d.dblock[~bad].isfinite().all())
    same = torch.full((2, 100), 3.0, device="cuda")   # no variance
    n = tr.moc_residual_forward(None, same, before=tr.Norm("layer"))
    assert not n.n.any() and bool((n.before[0] == 3).all())


def test_no_rows(tr):
    e = lambda *s: torch.empty(*s, device="cuda")   # noqa: E731
    after, before = tr.Norm("layer", e(33), e(33)), tr.Norm("rms", e(33))
    f = tr.moc_residual_forward(e(0, 33), e(0, 33), e(33), 1.0, after, before, keep="int8")
    assert f.r.shape == f.n.shape == (0, 33) and f.after[0].shape == (0,) and f.kept.shape == (0, 33)
    d = tr.moc_residual_backward(e(0, 33), e(0, 33), f.r, e(0, 33), e(33), 1.0, after, f.after, before, f.before)
    assert d.dx.shape == (0, 33) and d.gate.shape == (1, 33) and not any(v.any() for v in d[2:] if v is not None)


def test_captured_and_on_another_stream(tr):
    g = gen("captured")
    rows, cols = 700, 1000
    t = {k: normal(g, rows, cols).bfloat16().cuda() for k in ("x", "b", "dr", "dn")}
    gate, gamma = normal(g, 7, cols).float().cuda(), normal(g, cols).float().cuda()
    after, before = tr.Norm("rms", gamma), tr.Norm("layer", gamma, gamma)

    def step(stream=None):
        f = tr.moc_residual_forward(t["x"], t["b"], gate, 0.5, after, before, keep="e4m3", stream=stream)
        d = tr.moc_residual_backward(t["dr"], t["dn"], f.r, t["b"], gate, 0.5, after, f.after, before, f.before, stream=stream)
        return [f.r, f.n, f.kept.codes, f.kept.scales, *f.before, f.after[1], *[v for v in d if v is not None]]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, step()))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, step()))
    for turn in range(3):
        for v in t.values():
            v.copy_(normal(g, rows, cols))
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        for _, got in graphs:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals(tr):
    x = lambda *s, **k: torch.ones(*s, device="cuda", **k)   # noqa: E731
    a, b, v, n = x(8, 64), x(8, 64), x(64), tr.Norm("rms")
    whole = x(1000)
    f = tr.moc_residual_forward(a, b, before=n)
    forward, backward = tr.moc_residual_forward, tr.moc_residual_backward
    stats = dict(before=n, before_stats=f.before)
    for bad in (lambda: forward(a, b[:4]), lambda: forward(a[:, :8], b), lambda: forward(a.cpu(), b), lambda: forward(a.double(), b), lambda: forward(a.t(), b.t()), lambda: forward(tr.moc_checkpoint_write(a), b),
                lambda: forward(a, b, x(3, 64)), lambda: forward(a, b, x(16, 64)), lambda: forward(a, b, x(63)), lambda: forward(a, b, x(0, 64)), lambda: forward(a, b, scale=math.nan),
                lambda: forward(a, b, scale=math.inf), lambda: forward(a, b, before=tr.Norm("batch")), lambda: forward(a, b, before=tr.Norm("rms", v, v)), lambda: forward(a, b, before=tr.Norm("layer", v[:3])),
                lambda: forward(a, b, before=tr.Norm("layer", v, v.half())), lambda: forward(a, b, before=tr.Norm("rms", eps=-1.0)), lambda: forward(a, b, before=tr.Norm("rms", eps=math.nan)),
                lambda: forward(a, b, keep="int8"), lambda: forward(a, b, out_norm=x(8, 64)), lambda: forward(a, b, want_stream=False), lambda: forward(x(1, 16385), x(1, 16385)),
                lambda: forward(x(3, 0), x(3, 0)), lambda: forward(a, b, before=n, keep="int4"),
                # memory that is shared otherwise than one over the other
                lambda: forward(whole[:512].view(8, 64), b, out=whole[64:576].view(8, 64)), lambda: forward(a, b, v, out=x(8, 64).copy_(a), before=tr.Norm("rms", whole[:64]), out_norm=whole[:512].view(8, 64)),
                lambda: forward(a, b, before=n, out=a, out_norm=a), lambda: forward(a, b, whole[:64], out=whole[:512].view(8, 64)), lambda: forward(a.bfloat16(), b, out=a.bfloat16()[:4]),
                lambda: backward(None, None), lambda: backward(a, None, **stats), lambda: backward(a, b), lambda: backward(a, b, **stats), lambda: backward(None, b, f.r, before=n),
                lambda: backward(a, b, f.r, before=n, before_stats=(None, v[:3])), lambda: backward(a, b, f.r, gate=v, **stats), lambda: backward(a, None, after=n, after_stats=f.before),
                lambda: backward(a, b, f.r, out_x=b, **stats), lambda: backward(a, b, f.r, out_block=f.r, **stats), lambda: backward(a, b, f.r, out_x=a, out_block=a, **stats),
                lambda: backward(a, b, f.r, work=x(4), gate=x(8, 64), block=b, before=tr.Norm("rms", v), before_stats=f.before), lambda: backward(a, b, f.r[:4], **stats), lambda: backward(tr.moc_checkpoint_write(a), b, f.r, **stats),
                lambda: backward(a, b, f.r, dtype=torch.int8, **stats)):
        with pytest.raises((ValueError, TypeError, MoccasinError)):
            bad()
    for bad in (lambda: forward(a, b, before=("rms",)), lambda: forward(a, b, before="rms"), lambda: forward(a, 3), lambda: forward("x", b)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    torch.cuda.synchronize()
    assert bool((a == 1).all()) and bool((b == 1).all()) and bool((whole == 1).all())


def test_every_call_asks_for_the_device_of_its_tensors(tr, monkeypatch):
    a = torch.ones(8, 64, device="cuda")
    f = tr.moc_residual_forward(a, a.clone(), before=tr.Norm("rms"))
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for call in (lambda: tr.moc_residual_forward(a, a.clone()), lambda: tr.moc_residual_backward(a, a.clone(), f.r, before=tr.Norm("rms"), before_stats=f.before)):
            with pytest.raises(ValueError, match="cuda:0.*cuda:1"):
                call()


def test_a_checkpoint_to_write_to_is_apart_from_the_norms(tr):
    room = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    keep = tr.Checkpoint(room[:512].view(8, 64), torch.empty((8, 2), dtype=torch.uint8, device="cuda"), "int8")
    scales = tr.Checkpoint(torch.empty((8, 64), dtype=torch.uint8, device="cuda"), room[:16].view(8, 2), "int8")
    gamma, b = room[256:512].view(torch.float32), torch.ones(8, 64, device="cuda")
    for after, before, kept in ((tr.Norm("rms", gamma), tr.Norm("rms"), keep), (None, tr.Norm("layer", None, gamma), keep), (None, tr.Norm("rms", room[:256].view(torch.float32)), scales)):
        with pytest.raises(ValueError):
            tr.moc_residual_forward(None, b, after=after, before=before, keep=kept)
    assert not room.any()


PARTS = [dict(block="bf16", stream="bf16", after="rms", before=None, gates=1),
         dict(block="fp16", stream="fp32", held="int8", after="layer", before=None, gates=2, ptype=torch.float16),
         dict(block="fp16", stream="fp16", after="layer", before=None, gates=0, lead=1, pad=3),
         dict(block="bf16", stream="fp32", held="e4m3", after=None, before=None, gates=3),
         dict(block="fp32", stream="fp32", after="layer", before="layer", gates=3, lead=1, pad=2),
         dict(block="fp32", stream="fp32", held="e4m3", after=None, before="rms", gates=6),
         dict(block="fp32", stream="fp32", held="int8", after="rms", before="rms", gates=6),
         dict(block="fp32", stream="fp32", after="rms", before=None, gates=0),
         dict(block="fp32", stream="fp32", after=None, before=None, gates=1),
         dict(block="fp32", stream="fp32", after=None, before="layer", gates=0),
         dict(block="fp32", stream="fp32", after=None, before=None, gates=0)]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("kind", PARTS, ids=["-".join(str(v) for v in k.values() if not isinstance(v, torch.dtype)) for k in PARTS])
def test_backward_of_parts_and_of_float32(tr, cols, kind):
    """A norm behind the block or a gate alone, with no norm before the next block; without the stream's gradient."""
    check_backward(tr, 6, cols, kind)


@pytest.mark.parametrize("rows,cols", [(3000, 64), (2002, 1247), (600, 4096), (601, 8192)])
@pytest.mark.parametrize("gates", [0, 1, 2, -2, -1])
@pytest.mark.parametrize("kind", [0, 2, 4, 5, 8])
def test_backward_of_parts_over_many_rows(tr, rows, cols, gates, kind):
    gates = gates if gates >= 0 else rows // -gates
    if gates < 1 or rows % gates:
        gates = min(gates, 1)
    check_backward(tr, rows, cols, dict(PARTS[kind], gates=gates))
