"""The weight update and the norm where a launch's workgroups each do several
pieces of work: long lists, and more rows than workgroups.  Tolerances are
those of the tests of small sizes."""
import numpy as np
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu
from tests.test_gpu_rms_norm import EPS, _check_norm, _grad64, _inside, _rand, _t, _weight
from tests.test_gpu_update import _adam64, _adam_list, _f64, _stats64, _tensors

pytestmark = pytest.mark.gpu

# past 320 shares in two launches, at 4, 2 and 1 workgroups a chunk; up to 320 in one, at 2 and 1
LISTS = {
    "four to a chunk": [700_003, 300_001, 5, 0, 8192],
    "two to a chunk": [3001 + 37 * (i % 20) for i in range(200)],
    "one to a chunk": [1 + 97 * (i % 30) for i in range(700)],
    "two to a chunk, one launch": [2049 + 61 * (i % 20) for i in range(120)],
    "one to a chunk, one launch": [1 + 53 * (i % 40) for i in range(250)],
}


@pytest.mark.parametrize("name", sorted(LISTS))
@pytest.mark.parametrize("gkind,pkind", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float16"),
                                         ("float32", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("decoupled", [True, False])
def test_adam(name, gkind, pkind, decoupled):
    import torch
    require_gpu()
    rng = np.random.default_rng(15)
    grads = _tensors(LISTS[name], (gkind,), rng, 1.0, offset=1)
    decay = [i % 3 != 1 for i in range(len(grads))]
    e = _adam_list(grads, rng, pkind, decay, offset=3)
    opt = dict(lr=0.01, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.1)
    want = [(_f64(w), _f64(m), _f64(v)) for w, m, v in zip(e["w"], e["m"], e["v"])]
    step = torch.tensor([2], device="cuda")
    stats = torch.empty(3, device="cuda")
    B.dd_grad_norm(e["list"].h, stats, max_norm=1.5)
    B.dd_adam_step(e["list"].h, step, stats, decoupled=decoupled, **opt)
    assert int(step) == 3
    f = _stats64(grads, 1.5)[1]
    for i, (w, m, v) in enumerate(want):
        w1, m1, v1, ew, em, ev = _adam64(_f64(grads[i]), w, m, v, 3, f, decay[i], opt["lr"], opt["beta1"], opt["beta2"],
                                         opt["eps"], opt["weight_decay"], decoupled)
        assert np.all(np.abs(_f64(e["m"][i]) - m1) <= em)
        assert np.all(np.abs(_f64(e["v"][i]) - v1) <= ev)
        assert np.all(np.abs(_f64(e["w"][i]) - w1) <= ew)
        if pkind != "float32":
            assert torch.equal(e["param"][i], e["w"][i].to(_t(pkind)))


@pytest.mark.parametrize("rows,cols", [(40_000, 64), (33_000, 100), (20_000, 200), (5000, 520), (9000, 1000), (1100, 2000),
                                       (1300, 4000), (700, 6000), (600, 12_000), (530, 16_384)])
@pytest.mark.parametrize("kind,wkind", [("bfloat16", "bfloat16"), ("float16", "float32"), ("float32", "float32")])
def test_gradient(rows, cols, kind, wkind):
    import torch
    require_gpu()
    rng = np.random.default_rng(rows + cols)
    w = _weight(rng, cols, wkind)
    h, dy, dh = _rand(rng, rows, cols, kind, 2.0, 3, 1), _rand(rng, rows, cols, kind), _rand(rng, rows, cols, kind)
    rstd, out = torch.empty(rows, device="cuda"), torch.empty(rows, cols, dtype=_t(kind), device="cuda")
    B.dd_rms_norm(h, None, w, EPS, out, rstd=rstd)
    _check_norm(h, None, w, out, None, rstd, kind)
    dx, dw = torch.empty_like(dy), torch.empty_like(w)
    B.dd_rms_norm_grad(dy, h, w, rstd, dx, dw, dh=dh)
    x1, w1, ex, ew = _grad64(dy, h, w, rstd, dh)
    assert _inside(dx, x1, ex * 1.01 + 2.0 ** -149, kind)
    assert _inside(dw, w1, ew * 1.01 + 2.0 ** -149, wkind)


@pytest.mark.parametrize("out_kind", ["bfloat16", "float8_e4m3fn"])
@pytest.mark.parametrize("cols,extra", [(1030, 1000), (20, 33_554_432 - (1 << 20) + 77)])
def test_more_workgroups_than_a_launch_takes(cols, extra, out_kind):
    """Rows past 2^20 workgroups go round: the same bits as from two calls."""
    import torch
    require_gpu()
    rows = (1 << 20) + extra
    gen = torch.Generator("cuda").manual_seed(cols)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    for part in x.split(1 << 20):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))

    def run(x):
        out = torch.empty(x.shape, dtype=_t(out_kind), device="cuda")
        rstd = torch.empty(x.shape[0], device="cuda")
        scales = torch.empty(x.shape[0], 1, device="cuda") if out_kind != "bfloat16" else None
        B.dd_rms_norm(x, None, None, EPS, out, rstd=rstd, scales=scales)
        return [out.view(torch.uint8 if out_kind != "bfloat16" else torch.int16), rstd] + ([scales] if scales is not None else [])

    whole = run(x)
    cut = rows // 2
    for z in (slice(0, cut), slice(cut, rows)):
        assert all(torch.equal(a[z], b) for a, b in zip(whole, run(x[z])))
