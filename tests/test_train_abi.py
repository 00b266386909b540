"""Argument checks of the weight update's and the norm's entry points, without
a GPU: every refusal comes before the first device call."""
import ctypes
import math
import os
import struct

import pytest

from paper_2006_03318_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2006_03318_amd import build
        build.build()
    return B.lib()


def _load(lib, *tensors, count=None):
    out = ctypes.c_void_p(1)
    buf = ctypes.create_string_buffer(b"".join(B._TENSOR.pack(*t) for t in tensors) or b"\0")
    rc = lib.dd_tensors_load(len(tensors) if count is None else count, buf, None, ctypes.byref(out))
    return rc, out.value


P = 1 << 20      # an address that is never read
#        grad param master m v n grad_type param_type no_decay reserved
GOOD = (P, P, 0, P, P, 5, B.DD_F32, B.DD_F32, 0, 0)


def _with(t, **kw):
    names = ("grad", "param", "master", "m", "v", "n", "grad_type", "param_type", "no_decay", "reserved")
    return tuple(kw.get(k, x) for k, x in zip(names, t))


@pytest.mark.parametrize("change,word", [
    (dict(n=-1), "n < 0"),
    (dict(grad=0), "grad is NULL"),
    (dict(grad_type=3), "grad_type"),
    (dict(grad_type=-1), "grad_type"),
    (dict(param_type=4), "param_type"),
    (dict(grad=P + 2), "aligned"),
    (dict(grad=P + 1, grad_type=B.DD_BF16), "aligned"),
    (dict(m=P + 2), "aligned"),
    (dict(v=0), "m and v"),
    (dict(m=0), "m and v"),
    (dict(master=P), "master"),
    (dict(param_type=B.DD_BF16), "master"),
    (dict(param=0, m=0), "param"),
    (dict(no_decay=2), "no_decay"),
    (dict(reserved=1), "reserved"),
    (dict(n=1 << 62), "2^62"),
    (dict(n=1 << 50), "too many"),
])
def test_tensor_refusals(lib, change, word):
    rc, out = _load(lib, GOOD, _with(GOOD, **change))
    assert rc == B.DD_EINVAL and out is None
    assert word in B.dd_last_error(), B.dd_last_error()


def test_list_refusals(lib):
    assert lib.dd_tensors_load(0, None, None, None) == B.DD_EINVAL
    assert _load(lib, count=-1)[0] == B.DD_EINVAL
    out = ctypes.c_void_p(1)
    assert lib.dd_tensors_load(1, None, None, ctypes.byref(out)) == B.DD_EINVAL and out.value is None
    rc, out = _load(lib, GOOD, _with(GOOD, param=0, m=0, v=0))
    assert rc == B.DD_EINVAL and "some tensors have params" in B.dd_last_error()
    lib.dd_tensors_free(None)


def test_null_handles(lib):
    f = ctypes.c_void_p(P)
    assert lib.dd_grad_norm(None, 1.0, None, f, None) == B.DD_EINVAL
    assert "NULL handle" in B.dd_last_error()
    assert lib.dd_grad_clip(None, None, f, None) == B.DD_EINVAL
    assert lib.dd_adam_step(None, f, None, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, None) == B.DD_EINVAL


# rows cols x r h out strides; x residual weight h out scales rstd; types; group eps reserved
NORM = dict(rows=3, cols=8, sx=8, sr=8, sh=8, so=8, x=P, r=P, w=P, h=P, out=P, scales=0, rstd=0, type=B.DD_BF16,
            wt=B.DD_F32, ot=B.DD_BF16, group=0, eps=1e-6, res=0)


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(cols=1 << 31), "2^31"), (dict(rows=1 << 31), "2^31"),
    (dict(type=3), "type"), (dict(wt=B.DD_F16), "weight_type"), (dict(ot=B.DD_F32), "out_type"), (dict(ot=9), "out_type"),
    (dict(group=128), "8 bits"), (dict(scales=P), "8 bits"), (dict(ot=B.DD_E4M3), "scales"),
    (dict(ot=B.DD_E4M3, scales=P, group=100), "group"), (dict(ot=B.DD_I8, scales=P + 2), "scales"),
    (dict(x=0), "x is NULL"), (dict(out=0), "out is NULL"), (dict(x=P + 1), "x is not aligned"),
    (dict(r=P + 1), "residual"), (dict(h=P + 1), "h is not"), (dict(w=P + 2), "weight"), (dict(rstd=P + 2), "rstd"),
    (dict(sx=-8), "stride"), (dict(so=7), "out: stride"), (dict(sh=0), "h: stride"), (dict(sx=1 << 60), "too large"),
    (dict(eps=-1.0), "eps"), (dict(eps=math.inf), "eps"), (dict(eps=math.nan), "eps"), (dict(res=1), "reserved"),
])
def test_norm_refusals(lib, change, word):
    a = B._RMS.pack(*{**NORM, **change}.values())
    assert lib.dd_rms_norm(a, None) == B.DD_EINVAL
    assert word in B.dd_last_error(), B.dd_last_error()


GRAD = dict(rows=3, cols=8, sd=8, sh=8, se=8, sx=8, dy=P, h=P, dh=P, w=P, rstd=P, dx=P, dw=P, work=0, type=B.DD_F32,
            wt=B.DD_F32)


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(type=B.DD_E4M3), "type"), (dict(wt=B.DD_BF16), "weight_type"),
    (dict(dy=0), "dy is NULL"), (dict(h=0), "h is NULL"), (dict(dx=0), "dx is NULL"), (dict(rstd=0), "rstd"),
    (dict(dy=P + 2), "dy"), (dict(dh=P + 2), "dh"), (dict(dw=P + 2), "dw"), (dict(work=P + 8), "work"),
    (dict(sd=-1), "dy: stride"), (dict(sx=0), "dx: stride"),
])
def test_norm_gradient_refusals(lib, change, word):
    a = B._RMS_GRAD.pack(*{**GRAD, **change}.values())
    assert lib.dd_rms_norm_grad(a, None) == B.DD_EINVAL
    assert word in B.dd_last_error(), B.dd_last_error()


def test_no_work_needs_no_device(lib):
    assert lib.dd_rms_norm(None, None) == B.DD_EINVAL and lib.dd_rms_norm_grad(None, None) == B.DD_EINVAL
    assert lib.dd_rms_norm(B._RMS.pack(*{**NORM, "rows": 0, "x": 0, "out": 0}.values()), None) == B.DD_OK
    assert lib.dd_rms_norm_grad(B._RMS_GRAD.pack(*{**GRAD, "rows": 0, "dw": 0}.values()), None) == B.DD_OK
    assert B.dd_rms_norm_grad_work(-1, 4) == 0 and B.dd_rms_norm_grad_work(4, 0) == 0
    assert B.dd_rms_norm_grad_work(1, 1000) >= 4000
    assert B.dd_rms_norm_grad_work(0, 1000) >= 4000     # dw of no rows is written too


def test_structs_match_the_header(tmp_path):
    """The packed arguments of the binding have the header's layout."""
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#include "dd.h"\n#include <stdio.h>\nint main(void) {\n'
                   'printf("%zu %zu %zu ", sizeof(dd_tensor), sizeof(dd_rms_norm_args), sizeof(dd_rms_norm_grad_args));\n'
                   'printf("%zu %zu %zu %zu\\n", offsetof(dd_tensor, grad_type), offsetof(dd_rms_norm_args, type),\n'
                   'offsetof(dd_rms_norm_args, eps), offsetof(dd_rms_norm_grad_args, type)); return 0; }\n')
    exe = str(tmp_path / "t")
    subprocess.check_call(["gcc", "-I", os.path.dirname(B.HEADER), str(src), "-o", exe])
    got = [int(x) for x in subprocess.check_output([exe]).split()]
    fields = (struct.calcsize("@5Pq"), struct.calcsize("@6q7P"), struct.calcsize("@6q7P4i"), struct.calcsize("@6q8P"))
    assert got == [B._TENSOR.size, B._RMS.size, B._RMS_GRAD.size, *fields]


def test_binding_refuses_host_tensors(lib):
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        B.dd_rms_norm(x, None, None, 1e-6, torch.empty(4, 8))
    with pytest.raises(ValueError, match="GPU"):
        B.dd_tensors_load([dict(grad=x)])
    with pytest.raises(ValueError, match="unknown"):
        B.dd_tensors_load([dict(grad=x, weight=x)])
    with pytest.raises(ValueError, match="GPU"):
        B.dd_grad_norm(None, torch.zeros(3))
    with pytest.raises(TypeError):
        B.dd_rms_norm(x.double(), None, None, 1e-6, x)
    with pytest.raises(TypeError):
        B.dd_rms_norm_grad(x, x, torch.zeros(8, dtype=torch.float16), x, x)
