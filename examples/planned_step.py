"""A training step run as a rematerialisation plan says.

A stack of residual blocks (layer norm, a wide linear layer through gelu, a linear layer back and the
residual) becomes a compute graph: node i is block i's forward pass, whose output is its result and what it
keeps for the backward pass in 8 bits; node 2L - 1 - i is its backward pass.  The search brings the plain
schedule below a memory budget by computing blocks again, the decoder turns what it found into a sequence,
and the sequence is run with the operators of `paper_2304_14463_amd.training`.  They give the same bits for the
same inputs (torch's allocator gives every tensor one alignment), so every gradient is that of the plain schedule.

The graph's sizes are those of the blocks' outputs and gradients.  What a block needs while it runs and the parameters' gradients
are not in it, so the allocator's peak is above the plan's.

    python examples/planned_step.py [blocks] [rows] [width] [budget as a share of the plain schedule's peak]
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2304_14463_amd import moccasin as moc  # noqa: E402
from paper_2304_14463_amd import training as tr  # noqa: E402

KIB = 1024


def make_parameters(blocks, width, inner, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, by):
        return torch.randn(*shape, generator=g, device="cuda") * by

    return [dict(gamma=1 + normal(width, by=0.1), beta=normal(width, by=0.1),
                 w1=normal(inner, width, by=width ** -0.5).to(dtype), b1=normal(inner, by=0.1),
                 w2=normal(width, inner, by=0.5 * inner ** -0.5).to(dtype), b2=normal(width, by=0.1)) for _ in range(blocks)]


def block_forward(x, p):
    """What a block leaves: its result and, for the backward pass, 8 bits a value."""
    n, mean, rstd, kept_n = tr.moc_norm_forward(x, p["gamma"], p["beta"], keep="int8")
    h, kept_u = tr.moc_linear_forward(n, p["w1"], p["b1"], act="gelu", keep="e4m3")
    y, _ = tr.moc_linear_forward(h, p["w2"], p["b2"], residual=x)
    return dict(y=y, mean=mean, rstd=rstd, n=kept_n, u=kept_u)


def block_backward(dy, x, kept, p):
    """(gradient of the block's input, gradients of its parameters)"""
    h = tr.moc_checkpoint_read(kept["u"], dy.dtype, act="gelu")
    dw2, db2 = tr.moc_linear_backward_weight(dy, h)
    du = tr.moc_linear_backward_input(dy, p["w2"], act="gelu", pre=kept["u"])
    dw1, db1 = tr.moc_linear_backward_weight(du, kept["n"])
    dn = tr.moc_linear_backward_input(du, p["w1"])
    dx, dgamma, dbeta = tr.moc_norm_backward(dn, x, p["gamma"], kept["mean"], kept["rstd"], residual=dy)
    return dx, dict(gamma=dgamma, beta=dbeta, w1=dw1, b1=db1, w2=dw2, b2=db2)


class Step:
    """The graph of a step of `blocks` blocks and the plans of it."""

    def __init__(self, blocks, rows, width, inner):
        self.blocks, n = blocks, 2 * blocks
        self.inputs = [[i - 1] if i else [] for i in range(blocks)]
        for i in reversed(range(blocks)):   # the backward pass reads the block's input, what it kept, and the gradient
            self.inputs.append([v for v in ((i - 1) if i else None, i, n - 2 - i if i < blocks - 1 else None) if v is not None])
        kept = rows * (2 * width + 8) + rows * (width + inner) * 33 // 32
        self.sizes = [max(1, kept // KIB)] * blocks + [max(1, rows * width * 2 // KIB)] * blocks
        self.durations = [1] * blocks + [2] * blocks
        ptr = np.cumsum([0] + [len(u) for u in self.inputs]).astype(np.int32)
        self.graph = (n, ptr, np.array([u for us in self.inputs for u in us], dtype=np.int32), np.array(self.sizes, dtype=np.int32), np.array(self.durations, dtype=np.int32))
        self.last_use = [max([v for v in range(n) if u in self.inputs[v]], default=u) for u in range(n)]

    def plan(self, share, copies=2):
        """(sequence of nodes, its peak, the plain schedule's peak): the peak in KiB, below `share` of the plain one's if the
        search gets there"""
        n = self.graph[0]
        starts, ends, active = (torch.zeros(1, n * copies, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.uint8))
        starts[0, ::copies] = torch.arange(n, dtype=torch.int32, device="cuda") * copies
        ends[0, ::copies] = torch.tensor(self.last_use, dtype=torch.int32, device="cuda") * copies
        active[0, ::copies] = 1
        plain_graph = moc.moc_graph_upload(*self.graph, 0, copies)
        plain = int(moc.results_to_numpy(moc.moc_eval_batch(plain_graph, starts, ends, active))["peak"][0])
        plain_graph.free()
        g = moc.moc_graph_upload(*self.graph, int(share * plain), copies)
        moc.moc_search_two_phase(g, starts, ends, active, 4 * n, n, K=64)
        out, seq = moc.moc_decode_batch(g, starts, active)
        out, seq = moc.results_to_numpy(out, moc.DECODE_RESULT_DTYPE)[0], seq[0].cpu().numpy()
        g.free()
        if int(out["status"]) != 1:
            raise RuntimeError("the search's result is not a valid sequence")
        return [int(v) for v in seq[:int(out["length"])]], int(out["peak"]), plain

    def plain(self):
        return list(range(2 * self.blocks))

    def run(self, sequence, x, dy, parameters):
        """(result, gradient of x, gradients of the parameters by block) of the sequence; an output is dropped after its last use
        before its node is computed again."""
        last, drop = {}, {}
        for at in reversed(range(len(sequence))):
            v = sequence[at]
            if v in last:
                drop.setdefault(last.pop(v), []).append(v)
            for u in self.inputs[v]:
                last.setdefault(u, at)
        held, grads, result = {}, [None] * self.blocks, None
        n = 2 * self.blocks
        for at, v in enumerate(sequence):
            i = v if v < self.blocks else n - 1 - v
            before = held[i - 1]["y"] if i else x
            if v < self.blocks:
                held[v] = block_forward(before, parameters[i])
                result = held[v]["y"] if i == self.blocks - 1 else result
            else:
                held[v], grads[i] = block_backward(held[v - 1] if i < self.blocks - 1 else dy, before, held[i], parameters[i])
            for u in drop.get(at, ()):
                del held[u]
        return result, held[n - 1], grads


def main(blocks=16, rows=8192, width=1024, share=0.6):
    inner = 4 * width
    step, parameters = Step(blocks, rows, width, inner), make_parameters(blocks, width, inner)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(rows, width, generator=g, device="cuda").bfloat16() for _ in range(2))
    sequence, peak, plain = step.plan(share)
    print(f"{blocks} blocks of {rows} x {width}: plain schedule {plain / KIB:.0f} MiB, budget {share * plain / KIB:.0f}, plan {peak / KIB:.0f} MiB, "
          f"{len(sequence) - 2 * blocks} blocks computed again")
    first = None
    for name, nodes in (("plain", step.plain()), ("planned", sequence)):
        step.run(nodes, x, dy, parameters)
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        torch.cuda.reset_peak_memory_stats()
        base = torch.cuda.memory_allocated()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        result = step.run(nodes, x, dy, parameters)
        end.record()
        torch.cuda.synchronize()
        same = "" if first is None else ", gradients the same bit for bit" if all(torch.equal(a[k], b[k]) for a, b in zip(first[2], result[2]) for k in a) else ", GRADIENTS DIFFER"
        first = first or result
        print(f"{name:8s} {start.elapsed_time(end):8.2f} ms, {(torch.cuda.max_memory_allocated() - base) / KIB ** 2:8.0f} MiB above the parameters{same}", flush=True)


if __name__ == "__main__":
    main(*[kind(v) for kind, v in zip((int, int, int, float), sys.argv[1:])])
