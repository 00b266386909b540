"""Argument checks of the product, dropout and embedding entry points, without a GPU:
every refusal comes before the first device call."""
import math
import os
import struct

import pytest

from paper_2006_03318_amd import binding as B
from tests.test_train_abi import P, lib  # noqa: F401

LINEAR = dict(rows=3, k=8, n=16, sx=8, sw=16, sr=16, sy=16, sz=16, x=P, w=P, b=P, r=P, y=P, z=P, work=0,
              type=B.DD_BF16, bt=B.DD_F32, act=0, turned=0)


def refused(lib, name, record, base, change, word):  # noqa: F811
    assert getattr(lib, name)(record.pack(*{**base, **change}.values()), None) == B.DD_EINVAL
    assert word in B.dd_last_error(), B.dd_last_error()


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(k=0), "k and n"), (dict(n=0), "k and n"), (dict(rows=1 << 31), "2^31"), (dict(k=1 << 31), "2^31"),
    (dict(n=1 << 31), "2^31"), (dict(type=B.DD_F32), "type must be"), (dict(type=B.DD_E4M3), "type must be"), (dict(bt=B.DD_F16), "bias_type"),
    (dict(act=5), "act"), (dict(act=-1), "act"), (dict(turned=2), "turned"),
    (dict(x=0), "x is NULL"), (dict(w=0), "w is NULL"), (dict(y=0), "y is NULL"), (dict(x=P + 1), "x is not aligned"), (dict(w=P + 1), "w is not"),
    (dict(b=P + 2), "bias"), (dict(r=P + 1), "residual"), (dict(y=P + 1), "y is not"), (dict(z=P + 1), "z is not"), (dict(work=P + 8), "work"),
    (dict(sx=-1), "x: stride"), (dict(sw=-1), "w: stride"), (dict(sr=-1), "residual: stride"), (dict(sy=15), "y: stride"), (dict(sz=0), "z: stride"),
    (dict(sx=1 << 60), "too large"), (dict(rows=(1 << 31) - 1, n=1 << 21, sy=1 << 21, sw=1 << 21, sz=1 << 21), "one launch"),
])
def test_linear_refusals(lib, change, word):  # noqa: F811
    refused(lib, "dd_linear", B._LINEAR, LINEAR, change, word)


GRAD = dict(rows=3, k=8, n=16, sd=16, sx=8, sw=16, si=8, sdx=8, sdw=16, dy=P, x=P, w=P, iz=P, dx=P, dw=P, db=P, work=0,
            type=B.DD_F16, bt=B.DD_F16, act=0, turned=0)


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(type=B.DD_F32), "type must be"), (dict(bt=B.DD_BF16), "bias_type"), (dict(act=9), "in_act"),
    (dict(act=2, iz=0), "in_z"), (dict(turned=-1), "turned"), (dict(dy=0), "dy is NULL"), (dict(x=0), "x is NULL"), (dict(w=0), "w is NULL"),
    (dict(dy=P + 1), "dy is not"), (dict(dx=P + 1), "dx is not"), (dict(dw=P + 1), "dw is not"), (dict(db=P + 1), "db"), (dict(iz=P + 1), "in_z is not"),
    (dict(sd=-1), "dy: stride"), (dict(sdx=7), "dx: stride"), (dict(sdw=15), "dw: stride"), (dict(turned=1, sdw=7), "dw: stride"),
    (dict(rows=0, dw=P + 1), "dw is not"), (dict(work=P + 4), "work"),
])
def test_linear_gradient_refusals(lib, change, word):  # noqa: F811
    refused(lib, "dd_linear_grad", B._LINEAR_GRAD, GRAD, change, word)


ACT = dict(rows=3, cols=8, sd=8, sz=8, so=8, dy=P, z=P, dz=P, type=B.DD_F32, act=1)


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(cols=1 << 31), "2^31"), (dict(type=4), "type"), (dict(act=7), "act"),
    (dict(dy=0), "dy is NULL"), (dict(z=P + 2), "z is not"), (dict(dz=0), "dz is NULL"), (dict(so=7), "dz: stride"),
])
def test_activation_gradient_refusals(lib, change, word):  # noqa: F811
    refused(lib, "dd_act_grad", B._ACT_GRAD, ACT, change, word)


DROP = dict(rows=3, cols=8, sx=8, sr=8, so=8, x=P, r=P, out=P, state=P, used=P + 16, call=0, p=0.5, type=B.DD_F32, res=0)


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(rows=1 << 31), "2^31"), (dict(type=3), "type"), (dict(p=-0.1), "p must"),
    (dict(p=1.1), "p must"), (dict(p=math.nan), "p must"), (dict(state=0), "d_state"), (dict(state=P + 4), "d_state"), (dict(used=P + 4), "d_used"),
    (dict(used=P), "d_used is d_state"), (dict(used=P + 8), "overlaps"), (dict(res=1), "reserved"), (dict(x=0), "x is NULL"), (dict(out=P + 2), "out is not"),
    (dict(r=P + 1), "residual"), (dict(sx=-1), "x: stride"), (dict(so=7), "out: stride"),
])
def test_dropout_refusals(lib, change, word):  # noqa: F811
    refused(lib, "dd_dropout", B._DROPOUT, DROP, change, word)


EMBED = dict(tokens=3, vocab=5, cols=8, st=8, so=8, ids=P, table=P, out=P, scale=1.0, type=B.DD_F32, bytes=8, res=0)


@pytest.mark.parametrize("change,word", [
    (dict(tokens=-1), "tokens"), (dict(vocab=0), "vocab"), (dict(cols=0), "cols"), (dict(tokens=1 << 28), "2^28"), (dict(vocab=1 << 31), "2^31"),
    (dict(type=3), "type"), (dict(bytes=2), "id_bytes"), (dict(ids=0), "ids"), (dict(ids=P + 4), "ids"), (dict(scale=math.nan), "scale"),
    (dict(res=1), "reserved"), (dict(table=0), "table is NULL"), (dict(out=P + 1), "out is not"), (dict(st=-1), "table: stride"), (dict(so=7), "out: stride"),
])
def test_embedding_refusals(lib, change, word):  # noqa: F811
    refused(lib, "dd_embed", B._EMBED, EMBED, change, word)


EGRAD = dict(tokens=3, vocab=5, cols=8, sd=8, st=8, ids=P, dy=P, dtable=P, work=0, pad=-1, scale=1.0, type=B.DD_F32, bytes=4, res=0)


@pytest.mark.parametrize("change,word", [
    (dict(tokens=-1), "tokens"), (dict(bytes=0), "id_bytes"), (dict(ids=P + 2), "ids"), (dict(pad=-2), "pad"), (dict(pad=5), "pad"),
    (dict(vocab=1 << 29), "2^29"), (dict(dy=0), "dy is NULL"), (dict(dtable=0), "dtable is NULL"), (dict(st=7), "dtable: stride"), (dict(work=P + 1), "work"), (dict(res=2), "reserved"),
])
def test_embedding_gradient_refusals(lib, change, word):  # noqa: F811
    refused(lib, "dd_embed_grad", B._EMBED_GRAD, EGRAD, change, word)


def test_no_work_needs_no_device(lib):  # noqa: F811
    for name in ("dd_linear", "dd_linear_grad", "dd_act_grad", "dd_dropout", "dd_embed", "dd_embed_grad"):
        assert getattr(lib, name)(None, None) == B.DD_EINVAL
    assert lib.dd_linear(B._LINEAR.pack(*{**LINEAR, "rows": 0, "x": 0, "y": 0}.values()), None) == B.DD_OK
    assert lib.dd_linear_grad(B._LINEAR_GRAD.pack(*{**GRAD, "rows": 0, "dw": 0, "db": 0}.values()), None) == B.DD_OK
    assert lib.dd_linear_grad(B._LINEAR_GRAD.pack(*{**GRAD, "dx": 0, "dw": 0, "db": 0, "dy": 0}.values()), None) == B.DD_OK
    assert lib.dd_act_grad(B._ACT_GRAD.pack(*{**ACT, "rows": 0}.values()), None) == B.DD_OK
    assert lib.dd_embed(B._EMBED.pack(*{**EMBED, "tokens": 0, "ids": 0}.values()), None) == B.DD_OK


def test_working_memory(lib):  # noqa: F811
    """What bad sizes need is 0; sums that are cut need room for all their parts."""
    for f in (B.dd_linear_work, B.dd_linear_grad_work, B.dd_embed_grad_work):
        assert f(-1, 8, 8) == f(8, 0, 8) == f(8, 8, 0) == f(8, 1 << 31, 8) == 0
    assert B.dd_linear_work(0, 8, 8) == 0
    assert B.dd_linear_work(1, 1 << 16, 128) >= 2 * 128 * 4
    assert B.dd_linear_grad_work(1 << 16, 64, 64) >= 2 * 64 * 64 * 4
    assert B.dd_embed_grad_work(0, 10, 10) == 0 and B.dd_embed_grad_work(1000, 10, 64) >= 1000 * 16


def test_structs_match_the_header(tmp_path):
    """The packed arguments of the binding have the header's layout."""
    import subprocess
    fields = [("dd_linear_args", "type", B._LINEAR, "@8q7P"), ("dd_linear_grad_args", "type", B._LINEAR_GRAD, "@9q8P"),
              ("dd_act_grad_args", "type", B._ACT_GRAD, "@5q3P"), ("dd_dropout_args", "p", B._DROPOUT, "@5q5PQ"),
              ("dd_embed_args", "type", B._EMBED, "@5q3Pf"), ("dd_embed_grad_args", "scale", B._EMBED_GRAD, "@5q4Pq")]
    src = tmp_path / "t.c"
    src.write_text('#include "dd.h"\n#include <stdio.h>\nint main(void) {\n' + "".join(
        'printf("%%zu %%zu ", sizeof(%s), offsetof(%s, %s));\n' % (s, s, f) for s, f, _, _ in fields) + "return 0; }\n")
    exe = str(tmp_path / "t")
    subprocess.check_call(["gcc", "-I", os.path.dirname(B.HEADER), str(src), "-o", exe])
    got = [int(x) for x in subprocess.check_output([exe]).split()]
    assert got == [v for _, _, r, f in fields for v in (r.size, struct.calcsize(f))]


def test_binding_refusals(lib):  # noqa: F811
    import torch
    h, f = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int64)
    state = torch.zeros(2, dtype=torch.int64)
    for call in (lambda: B.dd_linear(h, h.t(), h[:, :4]), lambda: B.dd_linear_grad(h, h, h.t(), dx=h), lambda: B.dd_linear_grad(h, db=f[0]),
                 lambda: B.dd_act_grad(f, f, f, "relu"), lambda: B.dd_dropout(f, None, 0.1, state, f), lambda: B.dd_embed(ids, f, f),
                 lambda: B.dd_embed_grad(ids, f, f)):
        with pytest.raises(ValueError, match="GPU|expected shape"):
            call()
    with pytest.raises(TypeError, match="bfloat16"):
        B.dd_linear(f, f, f)
    with pytest.raises(ValueError, match="expected shape"):
        B.dd_linear(h, h, h)
    with pytest.raises(ValueError, match="needs"):
        B.dd_linear_grad(h, dx=h)
    with pytest.raises(ValueError, match="act must be"):
        B._act("tanh")
    with pytest.raises(TypeError, match="int64"):
        B.dd_embed(f, f, f)
    with pytest.raises(TypeError):
        B.dd_dropout(f.double(), None, 0.1, state, f)
