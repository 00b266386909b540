"""The weight update and the normalization for programs that train with torch.

`add_rms_norm` is a differentiable function and `Adam` an optimizer, both on
the calls of `binding` and on torch's current stream.  They are the fused
forms that the recipes predict: one kernel for the element-wise work around a
norm (forward and backward), two or three launches for the update of all
weights (the paper's fused Adam, Sec. 5.1, with the f32 masters of mixed
precision).
"""
from __future__ import annotations

import contextlib
from typing import Iterable, Optional

import torch

from . import binding as B


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _on(first, *others):
    """The device of all these tensors as the current one, where the library works."""
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError("tensors on %s and %s: one device is needed" % (first.device, t.device))
    return torch.cuda.device(first.device) if first.is_cuda else contextlib.nullcontext()


def _rows(t):
    return t if t.dim() == 2 and t.stride(1) == 1 else t.contiguous()


class _AddRmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        ctx.set_materialize_grads(False)
        x = _rows(x)
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        if residual is None:
            h = x
        else:
            residual = _rows(residual)
            h = torch.empty_like(out)
        with _on(x, residual, weight):
            B.dd_rms_norm(x, residual, weight, eps, out, h=None if residual is None else h, rstd=rstd, stream=_stream())
        ctx.save_for_backward(h, weight, rstd)
        return out if residual is None else (out, h)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh=None):
        h, weight, rstd = ctx.saved_tensors
        if dy is None:
            return dh, dh if ctx.needs_input_grad[1] else None, None, None
        dy = _rows(dy)
        dx = torch.empty_like(dy, memory_format=torch.contiguous_format)
        dw = work = None
        if weight is not None and ctx.needs_input_grad[2]:
            dw = torch.empty_like(weight)
            # (torch's memory: in a captured graph it stays the graph's)
            work = torch.empty(B.dd_rms_norm_grad_work(rstd.numel(), h.shape[-1]), dtype=torch.uint8, device=h.device)
        dh = None if dh is None else _rows(dh)
        with _on(h, dy, dh, weight):
            B.dd_rms_norm_grad(dy, h, weight, rstd, dx, dw, dh=dh, work=work, stream=_stream())
        return dx, dx if ctx.needs_input_grad[1] else None, dw, None


def add_rms_norm(x, residual=None, weight=None, eps: float = 1e-6):
    """rms_norm(x + residual) * weight over the last dimension: the output, and
    the sum where there is a residual (to be the next one's residual)."""
    if residual is not None and residual.shape != x.shape:
        residual = residual.expand_as(x)
    return _AddRmsNorm.apply(x, residual, weight, eps)


class Adam:
    """Adam over all parameters at once, gradients clipped to max_norm on the way
    (0: not clipped), and skipped where one is not finite: two launches a step,
    three for large lists.

    Gradients live in one buffer per type that stays where it is; parameters of
    16 bits get f32 masters.  Weight decay spares parameters of fewer than two
    dimensions.  What else writes a parameter in place (a checkpoint that is
    loaded, a broadcast) is seen at the next step and goes on from there; after
    writes that torch does not count (through `.data`, by other libraries), and
    between replays, call `read_weights()`.  A step is captured into a graph on
    the stream that was current when the optimizer was made, and replayed with
    the settings of the capture.  `stats` holds the last step's gradient norm,
    factor and whether it was skipped, `steps` the steps taken, both on the GPU."""

    def __init__(self, params: Iterable[torch.nn.Parameter], lr=1e-3, betas=(0.9, 0.999), eps=1e-8,
                 weight_decay=0.0, decoupled=True, max_norm=0.0):
        self.params = [p for p in params if p.requires_grad]
        if not self.params:
            raise ValueError("no parameters to train")
        if len({id(p) for p in self.params}) != len(self.params):
            raise ValueError("a parameter is given twice")
        self.lr, self.betas, self.eps = lr, betas, eps
        self.weight_decay, self.decoupled, self.max_norm = weight_decay, decoupled, max_norm
        on = _on(*self.params)
        dev = self.params[0].device
        self.buffers = {}
        for dt in {p.dtype for p in self.params}:
            total = sum(-(-p.numel() // 64) * 64 for p in self.params if p.dtype == dt)
            self.buffers[dt] = torch.zeros(total, dtype=dt, device=dev)
        used = dict.fromkeys(self.buffers, 0)
        tensors, self.masters, self.m, self.v = [], [], [], []
        for p in self.params:
            o = used[p.dtype]
            used[p.dtype] += -(-p.numel() // 64) * 64
            grad = self.buffers[p.dtype][o:o + p.numel()].view_as(p)
            if p.grad is not None:
                grad.copy_(p.grad)
            p.grad = grad
            low = p.dtype != torch.float32
            self.masters.append(p.detach().float() if low else p.detach())
            self.m.append(torch.zeros_like(self.masters[-1]))
            self.v.append(torch.zeros_like(self.masters[-1]))
            t = dict(grad=p.grad, param=p.detach(), m=self.m[-1], v=self.v[-1], decay=p.dim() >= 2)
            if low:
                t["master"] = self.masters[-1]
            tensors.append(t)
        # the handle works on these addresses: they are kept, and looked at in every step
        self._tensors = tensors
        self._places = [(p, p.grad, p.data_ptr()) for p in self.params]
        self._versions = [p._version for p in self.params]
        self.steps = torch.zeros(1, dtype=torch.int64, device=dev)
        self.stats = torch.zeros(3, device=dev)
        self._free = B.dd_tensors_free      # (at the program's end the module may be gone first)
        with on:
            self._handle = B.dd_tensors_load(tensors, _stream())

    def zero_grad(self):
        for b in self.buffers.values():
            b.zero_()

    @torch.no_grad()
    def read_weights(self, which: Optional[Iterable[int]] = None):
        """Takes the parameters as they are (all, or those of these numbers): a
        master whose rounding is no longer its weight becomes the weight."""
        for i in range(len(self.params)) if which is None else which:
            p, w = self.params[i], self.masters[i]
            if p.dtype != w.dtype:
                w.copy_(torch.where(w.to(p.dtype) == p, w, p.to(w.dtype)))
            self._versions[i] = p._version

    def step(self, inv_scale: Optional[torch.Tensor] = None):
        """inv_scale: float32 [1] on the GPU, 1 / the scale of the loss."""
        for p, g, at in self._places:
            if p.grad is not g or p.data_ptr() != at:
                raise RuntimeError("a parameter or its gradient was replaced: both stay where they were when this "
                                   "optimizer was made (its zero_grad() keeps gradients in place)")
        written = [i for i, (p, seen) in enumerate(zip(self.params, self._versions)) if p._version != seen]
        if written:
            self.read_weights(written)
        with _on(self.params[0], inv_scale):
            s = _stream()
            B.dd_grad_norm(self._handle, self.stats, max_norm=self.max_norm, d_inv_scale=inv_scale, stream=s)
            B.dd_adam_step(self._handle, self.steps, self.stats, lr=self.lr, beta1=self.betas[0], beta2=self.betas[1],
                           eps=self.eps, weight_decay=self.weight_decay, decoupled=self.decoupled, stream=s)
        torch.autograd.graph.increment_version(self.params)     # (graphs that kept the old weights are refused)
        self._versions = [p._version for p in self.params]

    def close(self):
        h, self._handle = self._handle, None
        self._free(h)

    def __del__(self):
        if getattr(self, "_handle", None):
            self.close()
