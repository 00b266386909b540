"""Predict what fusing an iteration's element-wise kernels gains, and measure it.

The paper checks each of its models this way (Sec. 6): an iteration is traced
as it is, the trace is transformed and simulated, and the prediction is held
against the optimization itself.  The iteration here is a stack of residual
blocks in bf16 (norm, two products with a GELU between them) with Adam on f32
masters and clipped gradients.  `--plain` runs norms and updates as single
torch operations, tensor by tensor; `--fused` runs them with this library.

    python -m paper_2006_03318_amd.fused_iteration --plain
    python -m paper_2006_03318_amd.fused_iteration --fused
    rocprofv3 --kernel-trace --hip-runtime-trace --memory-copy-trace --marker-trace \\
        --output-format csv -d OUT -o run -- \\
        python3 -m paper_2006_03318_amd.fused_iteration --plain
    python -m paper_2006_03318_amd.fused_iteration --predict OUT

On one MI355X, 8 blocks of hidden size 2,048 over 65,536 rows (`--rows 65536`):
134.4 ms an iteration plain (134.9 while traced, 135.1 simulated from the trace),
99.8 predicted with the norms fused and the update in one pass (104.4 with the
paper's rule, which keeps the summed time of the update), 98.2 measured fused.
Tracing lengthens every host call, so an iteration whose host is the slower side
has to be longer on the GPU for the trace to show it as it is: 16,384 rows take
37.2 ms plain, 46.4 while traced, and 25.9 fused where 29.4 are predicted.
"""
from __future__ import annotations

import argparse
import dataclasses
import time
from typing import Sequence

import numpy as np

from . import recipes as R
from . import trace as TR
from . import workloads as W

EPS = 1e-6
ADAM = dict(lr=1e-4, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, max_norm=1.0)


# ---------------------------------------------------------------------------
# the iteration
def make_stack(hidden: int, layers: int, fused: bool, seed: int = 0, device="cuda"):
    """The blocks as a module: forward(x) of [rows, hidden] in bf16."""
    import torch
    from torch import nn
    from . import training

    class Norm(nn.Module):
        def __init__(self):
            super().__init__()
            self.weight = nn.Parameter(torch.ones(hidden, dtype=torch.bfloat16, device=device))

        def forward(self, x, residual):
            if fused:
                return training.add_rms_norm(x, residual, self.weight, EPS)
            h = (x.float() + residual.float())
            y = h * torch.rsqrt(h.pow(2).mean(-1, keepdim=True) + EPS) * self.weight.float()
            return y.to(x.dtype), h.to(x.dtype)

    class Mlp(nn.Module):
        def __init__(self, gen):
            super().__init__()

            def w(a, b):
                x = torch.randn(a, b, generator=gen, device=device) / a ** 0.5
                return nn.Parameter(x.to(torch.bfloat16))
            self.up, self.down = w(hidden, 4 * hidden), w(4 * hidden, hidden)

        def forward(self, x):
            return torch.nn.functional.gelu(x @ self.up) @ self.down

    class Stack(nn.Module):
        def __init__(self):
            super().__init__()
            gen = torch.Generator(device=device).manual_seed(seed)
            self.norms = nn.ModuleList(Norm() for _ in range(layers))
            self.mlps = nn.ModuleList(Mlp(gen) for _ in range(layers))

        def forward(self, x):
            residual = torch.zeros_like(x)
            for norm, mlp in zip(self.norms, self.mlps):
                y, residual = norm(x, residual)
                x = mlp(y)
            return x + residual

    return Stack()


class PlainAdam:
    """The same update as `training.Adam`, operation by operation and tensor by
    tensor."""

    def __init__(self, params, lr, betas, eps, weight_decay, max_norm):
        import torch
        self.params = list(params)
        self.opt = (lr, betas, eps, weight_decay, max_norm)
        self.masters = [p.detach().float() for p in self.params]
        self.m = [torch.zeros_like(w) for w in self.masters]
        self.v = [torch.zeros_like(w) for w in self.masters]
        self.t = 0

    def zero_grad(self):
        for p in self.params:
            p.grad = None

    def step(self):
        import torch
        lr, (b1, b2), eps, wd, max_norm = self.opt
        self.t += 1
        norm = torch.stack([p.grad.float().square().sum() for p in self.params]).sum().sqrt()
        factor = torch.clamp(max_norm / norm, max=1.0)
        for p, w, m, v in zip(self.params, self.masters, self.m, self.v):
            g = p.grad.float() * factor
            m.mul_(b1).add_(g, alpha=1 - b1)
            v.mul_(b2).addcmul_(g, g, value=1 - b2)
            if p.dim() >= 2:
                w.mul_(1 - lr * wd)
            w.addcdiv_(m, (v.sqrt() / (1 - b2 ** self.t) ** 0.5).add_(eps), value=-lr / (1 - b1 ** self.t))
            p.detach().copy_(w)


def mark(stack):
    """Marker ranges around every layer's forward and backward pass, which the
    trace's tasks take as their layers."""
    import torch

    def begin(name):
        def hook(*_):               # (a hook's value would replace what passes through)
            torch.cuda.nvtx.range_push(name)
        return hook

    def end(*_):
        torch.cuda.nvtx.range_pop()

    for i, pair in enumerate(zip(stack.norms, stack.mlps)):
        for mod, name in zip(pair, ("norm %d" % i, "mlp %d" % i)):
            mod.register_forward_pre_hook(begin("fwd " + name))
            mod.register_forward_hook(end)
            mod.register_full_backward_pre_hook(begin("bwd " + name))
            mod.register_full_backward_hook(end)


def train(hidden: int, layers: int, rows: int, steps: int, fused: bool, marked: bool = False):
    """Milliseconds of an iteration after three to warm up, and the losses."""
    import torch
    from . import training
    stack = make_stack(hidden, layers, fused)
    if marked:
        mark(stack)
    opt = (training.Adam if fused else PlainAdam)(stack.parameters(), **ADAM)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, hidden, generator=gen, device="cuda").to(torch.bfloat16).requires_grad_()
    y = torch.randn(rows, hidden, generator=gen, device="cuda").to(torch.bfloat16)
    losses, t0 = [], 0.0
    for it in range(steps + 3):
        if it == 3:
            torch.cuda.synchronize()
            t0 = time.perf_counter()
        torch.cuda.nvtx.range_push("iteration %d" % it)
        opt.zero_grad()
        loss = (stack(x) - y).float().square().mean()
        loss.backward()
        torch.cuda.nvtx.range_push("weight update")
        opt.step()
        torch.cuda.nvtx.range_pop()
        torch.cuda.nvtx.range_pop()
        losses.append(loss.detach())
    torch.cuda.synchronize()
    return (time.perf_counter() - t0) / steps * 1e3, [float(v) for v in losses]


# ---------------------------------------------------------------------------
# the prediction
@dataclasses.dataclass
class FuseLayers(R.Recipe):
    """The element-wise kernels of each of these layers become one: of a layer's
    GPU kernels in an iteration the longest remains, and the others go with
    their launch calls (one pass over the same data, where there were many)."""
    layers: Sequence[int]

    def apply(self, g, plan):
        k = R.is_kernel(g) & ~plan.removed
        iters = g.iteration if g.iteration is not None else np.zeros(g.n, np.int32)
        gone = np.zeros(g.n, bool)
        for la in self.layers:
            for it in np.unique(iters[k & (g.layer == la)]):
                ids = np.nonzero(k & (g.layer == la) & (iters == it))[0]
                gone[ids] = True
                gone[ids[np.argmax(g.dur[ids])]] = False
        R.remove_tasks(plan, g, gone)


def what_if(tg: TR.TraceGraph):
    """(graph, variants, their names): the iteration as traced, with its weight
    update fused, with its norms fused, with both, and both with the update at
    a quarter of the summed time (a fused update moves 28 bytes an element,
    single operations about four times that)."""
    g = tg.graph
    update = [i for i, n in enumerate(tg.layer_names) if n == "weight update"]
    norms = [i for i, n in enumerate(tg.layer_names) if "norm " in n]
    g.kind[R.is_kernel(g) & R.in_layers(g, update)] = W.K_OPT
    fuse = FuseLayers(norms)
    names = ["as traced", "fused update", "fused norms", "both", "both, update in one pass"]
    g2, vs = R.compile_sweep(g, [[], [R.FusedAdam()], [fuse], [R.FusedAdam(), fuse],
                                 [R.ScaleLayers(update, 1, 4), R.FusedAdam(), fuse]])
    return g2, vs, names


def predict(directory: str, iterations: Sequence[int]):
    """Milliseconds of each variant, simulated on the GPU; and as measured."""
    from . import batch
    tg = TR.build_graph(TR.read_rocprof_csv(directory), iterations=iterations)
    g, vs, names = what_if(tg)
    ms = np.concatenate([m.cpu().numpy() for _, _, _, _, m in batch.simulate(batch.to_device(g, vs))])
    return [(n, t / 1e6 / len(iterations)) for n, t in zip(names, ms)], tg.measured_span / 1e6 / len(iterations)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    how = ap.add_mutually_exclusive_group(required=True)
    how.add_argument("--plain", action="store_true")
    how.add_argument("--fused", action="store_true")
    how.add_argument("--predict", metavar="DIR", help="the trace that rocprofv3 wrote of a --plain run")
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--rows", type=int, default=16384)
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args()
    if a.predict:
        rows, measured = predict(a.predict, [6, 7])
        print("traced iteration: %.3f ms" % measured)
        for name, ms in rows:
            print("%-28s %8.3f ms" % (name, ms))
        return
    ms, losses = train(a.hidden, a.layers, a.rows, a.steps, a.fused, marked=True)
    print("%s: %.3f ms an iteration, loss %.5f -> %.5f" % ("fused" if a.fused else "plain", ms, losses[0], losses[-1]))


if __name__ == "__main__":
    main()
