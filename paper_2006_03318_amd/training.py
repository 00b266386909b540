"""The weight update, the normalization and a block's other kernels for programs that
train with torch.

`add_rms_norm`, `linear`, `mlp`, `Dropout` and `embed` are differentiable
functions and `Adam` an optimizer, all on the calls of `binding` and on torch's current
stream.  They are the fused forms that the recipes predict: one kernel for the
element-wise work around a norm (forward and backward), the activation,
bias and residual in the products they belong to, two or three launches for the
update of all weights (the paper's fused Adam, Sec. 5.1, with the f32 masters
of mixed precision).
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


def _matrix(w):
    if w.dim() != 2 or 0 in w.shape:
        raise ValueError("a weight or table must have two dimensions and not be empty, got %s" % (tuple(w.shape),))
    return w if w.stride(1) == 1 or w.stride(0) == 1 else w.contiguous()


def _workspace(size, like):
    # (torch's memory: in a captured graph it stays the graph's)
    return torch.empty(size, dtype=torch.uint8, device=like.device) if size else None


def _same(t, what, dtype):
    if t is not None and t.dtype != dtype:
        raise TypeError("%s is %s, the rows are %s" % (what, t.dtype, dtype))


def _linear(x, weight, bias, residual, act, want_z):
    """(y, z): z where it is wanted."""
    k, n = weight.shape
    shape = x.shape[:-1] + (n,)
    y = torch.empty(shape, dtype=x.dtype, device=x.device)
    z = torch.empty_like(y) if want_z else None
    with _on(x, weight, bias, residual):
        B.dd_linear(x, weight, y, bias=bias, residual=residual, act=act, z=z, work=lambda size: _workspace(size, x), stream=_stream())
    return y, z


def _linear_grad(dy, x, weight, bias, wanted, in_act="none", in_z=None):
    """dx, dw and db, those of the three that are wanted."""
    k, n = weight.shape
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if wanted[0] else None
    dw = torch.empty_like(weight) if wanted[1] else None
    db = torch.empty_like(bias) if wanted[2] and bias is not None else None
    if dx is not None or dw is not None or db is not None:
        with _on(dy, x, weight, bias):
            B.dd_linear_grad(dy, x, weight, dx=dx, dw=dw, db=db, in_act=in_act, in_z=in_z, work=lambda size: _workspace(size, dy),
                             stream=_stream())
    return dx, dw, db


# (What an activation takes is kept for the gradient alone.  Inside forward gradients are always off, and
# needs_input_grad tells of the inputs, so whether they are on is an argument.)
class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act, grad):
        x = _rows(x)
        ctx.act = act
        y, z = _linear(x, weight, bias, None if residual is None else _rows(residual), act,
                       grad and act != "none" and any(ctx.needs_input_grad[:3]))
        ctx.save_for_backward(x, weight, bias, z)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, z = ctx.saved_tensors
        dz = dy = _rows(dy)
        if z is not None:
            dz = torch.empty_like(z)
            with _on(dy, z):
                B.dd_act_grad(dy, z, dz, ctx.act, stream=_stream())
        return (*_linear_grad(dz, x, weight, bias, ctx.needs_input_grad[:3]), dy if ctx.needs_input_grad[3] else None, None, None)


def linear(x, weight, bias=None, act="none", residual=None):
    """act(x weight + bias) + residual, for x [..., k] and weight [k, n] in bfloat16 or float16 (the
    transpose of an [n, k] weight as it is); bias in that type or float32.  act: none,
    relu, gelu, gelu_tanh or silu."""
    for t, what in ((weight, "weight"), (residual, "residual")):
        _same(t, what, x.dtype)
    weight = _matrix(weight)
    if residual is not None:
        residual = residual.expand(x.shape[:-1] + weight.shape[1:])
    return _Linear.apply(x, weight, bias, residual, act, torch.is_grad_enabled())


class _Mlp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, up, down, bias_up, bias_down, residual, act, grad):
        x = _rows(x)
        ctx.act = act
        need = ctx.needs_input_grad
        a, z = _linear(x, up, bias_up, None, act, grad and act != "none" and (need[0] or need[1] or need[3]))
        y, _ = _linear(a, down, bias_down, None if residual is None else _rows(residual), "none", False)
        ctx.save_for_backward(x, up, down, bias_up, bias_down, z, a)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, up, down, bias_up, bias_down, z, a = ctx.saved_tensors
        need = ctx.needs_input_grad
        dy = _rows(dy)
        first = need[0] or need[1] or need[3]
        dz, ddown, dbias_down = _linear_grad(dy, a, down, bias_down, (first, need[2], need[4]), ctx.act, z)
        dx = dup = dbias_up = None
        if first:
            dx, dup, dbias_up = _linear_grad(dz, x, up, bias_up, (need[0], need[1], need[3]))
        return dx, dup, ddown, dbias_up, dbias_down, dy if need[5] else None, None, None


def mlp(x, up, down, bias_up=None, bias_down=None, act="gelu", residual=None):
    """linear(linear(x, up, bias_up, act), down, bias_down, residual=residual), whose gradient
    multiplies with the activation's derivative in the product that comes to it."""
    for t, what in ((up, "up"), (down, "down"), (residual, "residual")):
        _same(t, what, x.dtype)
    up, down = _matrix(up), _matrix(down)
    if residual is not None:
        residual = residual.expand(x.shape[:-1] + down.shape[1:])
    return _Mlp.apply(x, up, down, bias_up, bias_down, residual, act, torch.is_grad_enabled())


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, state, call):
        x = _rows(x)
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        used = torch.empty_like(state)
        with _on(x, residual, state):
            B.dd_dropout(x, None if residual is None else _rows(residual), p, state, out, call=call, used=used, stream=_stream())
        ctx.p = p
        ctx.save_for_backward(used)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        used, = ctx.saved_tensors
        dx = None
        if ctx.needs_input_grad[0]:
            rows = _rows(dy)
            dx = torch.empty_like(rows, memory_format=torch.contiguous_format)
            with _on(rows, used):
                B.dd_dropout(rows, None, ctx.p, used, dx, stream=_stream())
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None


class Dropout:
    """The dropouts of a model: drop(x, p, residual) is residual + x / (1 - p) where
    the generator keeps x.  Every call has a mask of its own, which the gradient makes
    again; p counts in 65,536ths.  The generator's key and counter are on the GPU
    (`state`): `step()`, once an iteration, moves the counter behind the calls made
    so far, and is captured with them where an iteration is captured, so that every replay has
    other masks.  A forward pass that is run again for its gradient (checkpointed) gets
    other masks than the first time: keep dropouts out of it."""

    def __init__(self, seed: int = 0, device="cuda"):
        key = seed & (1 << 64) - 1
        self.state = torch.tensor([key - (1 << 64) if key >> 63 else key, 0], dtype=torch.int64, device=device)
        self.calls = 0

    def __call__(self, x, p: float, residual=None):
        _same(residual, "residual", x.dtype)
        if residual is not None:
            residual = residual.expand_as(x)
        call, self.calls = self.calls, self.calls + 1
        return _Dropout.apply(x, residual, p, self.state, call)

    def step(self):
        self.state[1:].add_(self.calls)
        self.calls = 0


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, table, scale, pad):
        ids, table = ids.contiguous(), _rows(table)
        out = torch.empty(ids.shape + table.shape[1:], dtype=table.dtype, device=table.device)
        with _on(table, ids):
            B.dd_embed(ids, table, out, scale=scale, stream=_stream())
        ctx.save_for_backward(ids)
        ctx.table = table.shape, scale, pad
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        ids, = ctx.saved_tensors
        shape, scale, pad = ctx.table
        dy = _rows(dy)
        dtable = torch.empty(shape, dtype=dy.dtype, device=dy.device)
        with _on(dy, ids):
            work = _workspace(B.dd_embed_grad_work(ids.numel(), *shape), dy)
            B.dd_embed_grad(ids, dy, dtable, scale=scale, pad=pad, work=work, stream=_stream())
        return None, dtable, None, None


def embed(ids, table, scale: float = 1.0, pad: int = -1):
    """scale * table[ids], for int64 or int32 ids of any shape.  The row `pad` (-1: none) gets no
    gradient.  An id that the table does not have gives a row of NaNs, and no gradient."""
    _matrix(table)
    if not -1 <= pad < table.shape[0]:
        raise ValueError("pad must be -1 or a row of the table, got %d" % pad)
    return _Embed.apply(ids, table, float(scale), int(pad))


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
