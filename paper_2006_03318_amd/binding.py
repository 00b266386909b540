"""Thin ctypes binding over libdd.so with the C-ABI's names (include/dd.h).

Arguments are numpy arrays or torch tensors (host or GPU); this module only
checks dtypes/shapes and passes raw pointers.  All computation happens in the
HIP library.  Importing works without a GPU; calling into the library needs
the built libdd.so and fails loudly if it is missing.
"""
from __future__ import annotations

import ctypes
import os
import re
import struct
from typing import Optional, Tuple

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libdd.so")
HEADER = os.path.join(os.path.dirname(PKG), "include", "dd.h")

DD_OK, DD_EINVAL, DD_ECYCLE, DD_ECHAIN, DD_ERANGE, DD_ENOMEM, DD_EHIP, DD_EMISMATCH, \
    DD_ELIMIT = range(9)
DD_LEVELS, DD_PHASES = 0, 1
DD_LOAD_SHARED_THREADS = 1
DD_POLICY_EARLIEST, DD_POLICY_PRIORITY = 0, 1
DD_F32, DD_BF16, DD_F16, DD_E4M3, DD_I8 = range(5)
STATUS_NAMES = ["DD_OK", "DD_EINVAL", "DD_ECYCLE", "DD_ECHAIN", "DD_ERANGE", "DD_ENOMEM",
                "DD_EHIP", "DD_EMISMATCH", "DD_ELIMIT"]


class DDError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("%s: %s" % (STATUS_NAMES[code] if 0 <= code < len(STATUS_NAMES)
                                     else code, msg))
        self.code = code
        self.msg = msg


_lib = None
_vp = ctypes.c_void_p
_i32, _i64, _u64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64


def declared_symbols():
    """Function names declared in include/dd.h."""
    txt = open(HEADER).read()
    return sorted(set(re.findall(r"\b(dd_[a-z_]+)\s*\(", txt)))


def lib():
    """Load libdd.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libdd.so not built: run __graft_entry__.build() "
                          "(hipcc --offload-arch=gfx950)")
    try:        # let torch bring up its HIP runtime first so both share one
        import torch  # noqa: F401
    except ImportError:
        pass
    L = ctypes.CDLL(LIB_PATH)
    sig = {
        "dd_graph_load": (_i32, [_i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                 ctypes.POINTER(_vp)]),
        "dd_graph_load_ex": (_i32, [_i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                    ctypes.c_uint32, _vp, ctypes.POINTER(_vp)]),
        "dd_levelize": (_i32, [_vp, _u64, _i32, _vp, ctypes.POINTER(_vp), ctypes.POINTER(_i64)]),
        "dd_simulate_policy": (_i32, [_vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
        "dd_apply_transforms": (_i32, [_vp, _i32, _i32, _vp, _vp, _vp, _vp, ctypes.POINTER(_vp)]),
        "dd_simulate_batch": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _vp]),
        "dd_simulate_batch_vs": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp]),
        "dd_set_lookback_polls": (None, [_i32]),
        "dd_simulate_plan": (_i32, [_vp, _vp, ctypes.POINTER(_i32)]),
        "dd_release_cache": (_i32, []),
        "dd_simulate_batch_noalloc": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _vp]),
        "dd_runtime_breakdown": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _vp]),
        "dd_sched_task_steps": (_i32, [_vp, _vp, _vp]),
        "dd_sched_info": (_i32, [_vp, ctypes.POINTER(_i64), ctypes.POINTER(_i64),
                                 ctypes.POINTER(_i64), ctypes.POINTER(_i64)]),
        "dd_tensors_load": (_i32, [_i32, _vp, _vp, ctypes.POINTER(_vp)]),
        "dd_tensors_free": (None, [_vp]),
        "dd_grad_norm": (_i32, [_vp, ctypes.c_float, _vp, _vp, _vp]),
        "dd_grad_clip": (_i32, [_vp, _vp, _vp, _vp]),
        "dd_adam_step": (_i32, [_vp, _vp, _vp] + [ctypes.c_double] * 5 + [_i32, _vp]),
        "dd_rms_norm": (_i32, [ctypes.c_char_p, _vp]),
        "dd_rms_norm_grad": (_i32, [ctypes.c_char_p, _vp]),
        "dd_rms_norm_grad_work": (ctypes.c_size_t, [_i64, _i64]),
        "dd_graph_free": (None, [_vp]),
        "dd_sched_free": (None, [_vp]),
        "dd_variants_free": (None, [_vp]),
        "dd_status_str": (ctypes.c_char_p, [_i32]),
        "dd_last_error": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


# ---------------------------------------------------------------------------
def _ptr(x, dtype_name: Optional[str] = None, count: Optional[int] = None):
    """Raw pointer of a numpy array / torch tensor (contiguous) or None."""
    if x is None:
        return None
    if hasattr(x, "data_ptr"):           # torch tensor
        if not x.is_contiguous():
            raise ValueError("tensor must be contiguous")
        if dtype_name is not None:
            tn = str(x.dtype).replace("torch.", "")
            if tn != dtype_name:
                raise TypeError("expected %s, got %s" % (dtype_name, tn))
        if count is not None and x.numel() < count:
            raise ValueError("expected at least %d elements, got %d" % (count, x.numel()))
        return x.data_ptr() if x.numel() else None
    import numpy as np
    if not x.flags["C_CONTIGUOUS"]:
        raise ValueError("array must be C-contiguous")
    if dtype_name is not None and x.dtype != np.dtype(dtype_name):
        raise TypeError("expected %s, got %s" % (dtype_name, x.dtype))
    if count is not None and x.size < count:
        raise ValueError("expected at least %d elements, got %d" % (count, x.size))
    return x.ctypes.data if x.size else None


def _stream(stream):
    if stream is None:
        return None
    if hasattr(stream, "cuda_stream"):
        return stream.cuda_stream
    return int(stream)


def _check(rc: int):
    if rc != DD_OK:
        raise DDError(rc, lib().dd_last_error().decode())


def dd_status_str(code: int) -> str:
    return lib().dd_status_str(code).decode()


def dd_last_error() -> str:
    return lib().dd_last_error().decode()


def dd_graph_load(n, n_threads, in_ptr, in_src, edge_cls, thread_prev, thread_id, dur_ns, gap_ns,
                  node_cls, stream=None):
    out = _vp()
    rc = lib().dd_graph_load(int(n), int(n_threads), _ptr(in_ptr, "int64", n + 1),
                             _ptr(in_src, "int32"), _ptr(edge_cls, "uint8"),
                             _ptr(thread_prev, "int32", n), _ptr(thread_id, "int32", n),
                             _ptr(dur_ns, "int64", n), _ptr(gap_ns, "int64", n),
                             _ptr(node_cls, "uint16", n), _stream(stream), ctypes.byref(out))
    _check(rc)
    return out


def dd_graph_load_ex(n, n_threads, in_ptr, in_src, edge_cls, thread_prev, thread_id, dur_ns,
                     gap_ns, node_cls, flags, stream=None):
    out = _vp()
    rc = lib().dd_graph_load_ex(int(n), int(n_threads), _ptr(in_ptr, "int64", n + 1),
                                _ptr(in_src, "int32"), _ptr(edge_cls, "uint8"),
                                _ptr(thread_prev, "int32", n), _ptr(thread_id, "int32", n),
                                _ptr(dur_ns, "int64", n), _ptr(gap_ns, "int64", n),
                                _ptr(node_cls, "uint16", n), ctypes.c_uint32(int(flags)),
                                _stream(stream), ctypes.byref(out))
    _check(rc)
    return out


def dd_simulate_policy(g, var, policy, pp, prio, d_finish, d_start, d_makespan, stream=None):
    rc = lib().dd_simulate_policy(g, var, int(policy), _ptr(pp, "uint8"), _ptr(prio, "int32"),
                                  _ptr(d_finish, "int64"), _ptr(d_start, "int64"),
                                  _ptr(d_makespan, "int64"), _stream(stream))
    _check(rc)


def dd_levelize(g, active_edge_classes: int, mode: int, stream=None) -> Tuple[object, int]:
    out = _vp()
    steps = _i64(0)
    rc = lib().dd_levelize(g, ctypes.c_uint64(active_edge_classes & (2 ** 64 - 1)), int(mode),
                           _stream(stream), ctypes.byref(out), ctypes.byref(steps))
    _check(rc)
    return out, int(steps.value)


def dd_apply_transforms(g, n_variants, n_cls, scale, remove_bits, edge_on, stream=None):
    out = _vp()
    rc = lib().dd_apply_transforms(g, int(n_variants), int(n_cls), _ptr(scale, "int32"),
                                   _ptr(remove_bits, "uint32"), _ptr(edge_on, "uint64"),
                                   _stream(stream), ctypes.byref(out))
    _check(rc)
    return out


def dd_simulate_batch(g, sched, var, d_finish, d_start, d_makespan, stream=None):
    rc = lib().dd_simulate_batch(g, sched, var, _ptr(d_finish, "int64"), _ptr(d_start, "int64"),
                                 _ptr(d_makespan, "int64"), _stream(stream))
    _check(rc)


def dd_simulate_batch_vs(g, sched, var, d_finish, d_start, d_makespan, variants_per_wg,
                         stream=None):
    rc = lib().dd_simulate_batch_vs(g, sched, var, _ptr(d_finish, "int64"),
                                    _ptr(d_start, "int64"), _ptr(d_makespan, "int64"),
                                    int(variants_per_wg), _stream(stream))
    _check(rc)


def dd_simulate_plan(sched, var) -> int:
    """Launch shape dd_simulate_batch takes: > 0 variants per workgroup of the
    strip kernel, < 0 the few-variant path (one launch per step)."""
    w = _i32()
    _check(lib().dd_simulate_plan(sched, var, ctypes.byref(w)))
    return int(w.value)


def dd_set_lookback_polls(polls: int):
    lib().dd_set_lookback_polls(int(polls))


def dd_runtime_breakdown(g, var, role, d_finish, d_makespan, d_out, stream=None):
    rc = lib().dd_runtime_breakdown(g, var, _ptr(role, "uint8"), _ptr(d_finish, "int64"),
                                    _ptr(d_makespan, "int64"), _ptr(d_out, "int64"),
                                    _stream(stream))
    _check(rc)


def dd_simulate_batch_noalloc(g, sched, var, d_finish, d_start, d_makespan, stream=None):
    rc = lib().dd_simulate_batch_noalloc(g, sched, var, _ptr(d_finish, "int64"),
                                         _ptr(d_start, "int64"), _ptr(d_makespan, "int64"),
                                         _stream(stream))
    _check(rc)


def dd_release_cache():
    _check(lib().dd_release_cache())


def dd_sched_task_steps(sched, out, stream=None):
    _check(lib().dd_sched_task_steps(sched, _ptr(out, "int32"), _stream(stream)))


def dd_sched_info(sched):
    a, b, c, d = _i64(), _i64(), _i64(), _i64()
    _check(lib().dd_sched_info(sched, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c),
                               ctypes.byref(d)))
    return dict(n_steps=a.value, n_segments=b.value, max_step_width=c.value, n_gathers=d.value)


def dd_graph_free(g):
    if g:
        lib().dd_graph_free(g)


def dd_sched_free(s):
    if s:
        lib().dd_sched_free(s)


def dd_variants_free(v):
    if v:
        lib().dd_variants_free(v)


# ---------------------------------------------------------------------------
# The weight update and the root-mean-square norm.  All arguments are torch
# tensors on the GPU; the checks are kept short, as these calls take a few
# microseconds themselves.
_DT = {}
_NAMED = {}


def _types():
    if not _DT:
        import torch
        _NAMED.update(float32=torch.float32, int64=torch.int64)
        _DT.update({torch.float32: DD_F32, torch.bfloat16: DD_BF16, torch.float16: DD_F16,
                    torch.float8_e4m3fn: DD_E4M3, torch.int8: DD_I8})
    return _DT


def _gpu(name, t, count, *types):
    """Address of a contiguous tensor on the GPU (None stays None)."""
    if t is None:
        return 0
    if (t.is_cuda and (_DT or _types()).get(t.dtype, -1) in types and t.numel() == count
            and t.is_contiguous()):
        return t.data_ptr()
    if not isinstance(name, str):
        name = "tensor %d: %s" % name
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.numel() != count:
        raise ValueError("%s: expected %d elements, got %d" % (name, count, t.numel()))
    raise TypeError("%s: unexpected type %s" % (name, t.dtype))


def _small(name, t, count, dtype):
    """Address of a few numbers of one type on the GPU."""
    if (not t.is_cuda or t.dtype is not (_NAMED or _types() and _NAMED)[dtype]
            or t.numel() < count or not t.is_contiguous()):
        raise ValueError("%s must be %s [%d] on the GPU" % (name, dtype, count))
    return t.data_ptr()


_TENSOR = struct.Struct("@5Pq4i")


def dd_tensors_load(tensors, stream=None):
    """A handle for a list of tensors: each a dict with `grad` and, for
    dd_adam_step, `param`, `m`, `v`, `master` (16-bit params) and `decay`
    (default True).  They must live, where they are, as long as the handle."""
    known = {"grad", "param", "master", "m", "v", "decay"}
    rows = []
    for i, t in enumerate(tensors):
        if not known.issuperset(t):
            raise ValueError("tensor %d: unknown %s" % (i, ", ".join(sorted(set(t) - known))))
        g, p = t["grad"], t.get("param")
        n = g.numel()
        rows.append(_TENSOR.pack(_gpu((i, "grad"), g, n, DD_F32, DD_BF16, DD_F16),
                                 _gpu((i, "param"), p, n, DD_F32, DD_BF16, DD_F16),
                                 _gpu((i, "master"), t.get("master"), n, DD_F32),
                                 _gpu((i, "m"), t.get("m"), n, DD_F32),
                                 _gpu((i, "v"), t.get("v"), n, DD_F32), n, _DT[g.dtype],
                                 DD_F32 if p is None else _DT[p.dtype],
                                 0 if t.get("decay", True) else 1, 0))
    out = _vp()
    buf = ctypes.create_string_buffer(b"".join(rows), len(rows) * _TENSOR.size + 1)
    _check(lib().dd_tensors_load(len(rows), buf, _stream(stream), ctypes.byref(out)))
    return out


def dd_tensors_free(t):
    if t and _lib is not None:      # (None: the interpreter is shutting down)
        _lib.dd_tensors_free(t)


def dd_grad_norm(t, d_stats, max_norm=0.0, d_inv_scale=None, stream=None):
    """d_stats (float32 [3] on the GPU) receives the norm of all gradients, the
    factor that unscales and clips them, and 1 if one is not finite."""
    u = None if d_inv_scale is None else _small("d_inv_scale", d_inv_scale, 1, "float32")
    rc = (_lib or lib()).dd_grad_norm(t, max_norm, u, _small("d_stats", d_stats, 3, "float32"),
                                      None if stream is None else _stream(stream))
    if rc:
        _check(rc)


def dd_grad_clip(src, dst, d_stats, stream=None):
    rc = (_lib or lib()).dd_grad_clip(src, dst, _small("d_stats", d_stats, 3, "float32"),
                                      None if stream is None else _stream(stream))
    if rc:
        _check(rc)


def dd_adam_step(t, d_step, d_stats=None, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                 weight_decay=0.0, decoupled=True, stream=None):
    """One step of Adam; d_step: int64 [1] on the GPU, the steps taken."""
    st = None if d_stats is None else _small("d_stats", d_stats, 3, "float32")
    rc = (_lib or lib()).dd_adam_step(t, _small("d_step", d_step, 1, "int64"), st, lr, beta1,
                                      beta2, eps, weight_decay, 1 if decoupled else 0,
                                      None if stream is None else _stream(stream))
    if rc:
        _check(rc)


def _rows(name, t, shape, cols, dtype):
    """(address, row stride) of rows of cols elements: the last dimension is
    one row."""
    if t is None:
        return 0, 0
    if t.dtype is dtype and t.is_cuda and t.shape == shape:
        if t.is_contiguous():
            return t.data_ptr(), cols
        if t.dim() == 2 and (cols == 1 or t.stride(1) == 1):
            return t.data_ptr(), t.stride(0)
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU" % name)
    if t.dtype is not dtype:
        raise TypeError("%s: expected %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s: expected shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    raise ValueError("%s: elements of a row must be consecutive, and more than two dimensions "
                     "contiguous" % name)


_RMS = struct.Struct("@6q7P4if i")
_RMS_GRAD = struct.Struct("@6q8P2i")


def _row_types(x, weight):
    """Types of the rows and the weight, and the rows' shape and length."""
    types = _DT or _types()
    kind = types.get(x.dtype, -1)
    if not 0 <= kind <= DD_F16:
        raise TypeError("rows must be float32, bfloat16 or float16")
    shape = x.shape
    if not shape or shape[-1] < 1:
        raise ValueError("rows must have a dimension and not be empty")
    wk = DD_F32 if weight is None else types.get(weight.dtype, -1)
    if wk != DD_F32 and wk != kind:
        raise TypeError("weight must be float32 or the rows' type")
    return kind, wk, shape, shape[-1]


def dd_rms_norm(x, residual, weight, eps, out, h=None, rstd=None, scales=None, group=0, stream=None):
    """out = (x + residual) normalized over its last dimension, times weight:
    in x's type, or in 8 bits (out float8_e4m3fn or int8, with scales float32
    [rows, groups]).  residual, weight, h (receives x + residual) and rstd may
    be None."""
    kind, wk, shape, cols = _row_types(x, weight)
    rows, dt, odt = x.numel() // cols, x.dtype, out.dtype
    px, sx = _rows("x", x, shape, cols, dt)
    pr, sr = _rows("residual", residual, shape, cols, dt)
    ph, sh = _rows("h", h, shape, cols, dt)
    po, so = _rows("out", out, shape, cols, odt)
    args = _RMS.pack(rows, cols, sx, sr, sh, so, px, pr, _gpu("weight", weight, cols, wk), ph, po,
                     _gpu("scales", scales, rows * (-(-cols // group) if group > 0 else 1), DD_F32),
                     _gpu("rstd", rstd, rows, DD_F32), kind, wk, _DT.get(odt, -1), group, eps, 0)
    rc = (_lib or lib()).dd_rms_norm(args, None if stream is None else _stream(stream))
    if rc:
        _check(rc)


def dd_rms_norm_grad(dy, h, weight, rstd, dx, dw=None, dh=None, work=None, stream=None):
    """dx and dw from the gradient dy of the norm's output; dh: what reaches h
    on its other ways.  work: uint8 of dd_rms_norm_grad_work(rows, cols), or
    None (from the library's cache; not under graph capture)."""
    kind, wk, shape, cols = _row_types(h, weight if weight is not None else dw)
    rows, dt = h.numel() // cols, h.dtype
    pd, sd = _rows("dy", dy, shape, cols, dt)
    ph, sh = _rows("h", h, shape, cols, dt)
    pe, se = _rows("dh", dh, shape, cols, dt)
    px, sx = _rows("dx", dx, shape, cols, dt)
    if work is not None and (not work.is_cuda or not work.is_contiguous()
                             or work.numel() * work.element_size() < dd_rms_norm_grad_work(rows, cols)):
        raise ValueError("work must hold dd_rms_norm_grad_work(rows, cols) bytes on the GPU")
    args = _RMS_GRAD.pack(rows, cols, sd, sh, se, sx, pd, ph, pe, _gpu("weight", weight, cols, wk),
                          _gpu("rstd", rstd, rows, DD_F32), px, _gpu("dw", dw, cols, wk),
                          0 if work is None else work.data_ptr(), kind, wk)
    rc = (_lib or lib()).dd_rms_norm_grad(args, None if stream is None else _stream(stream))
    if rc:
        _check(rc)


def dd_rms_norm_grad_work(rows: int, cols: int) -> int:
    return lib().dd_rms_norm_grad_work(int(rows), int(cols))
