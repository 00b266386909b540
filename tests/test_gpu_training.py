"""The differentiable norm, the optimizer, and an iteration that runs them
together."""
import math

import numpy as np
import pytest

from tests.gpu_common import require_gpu, say
from tests.test_gpu_rms_norm import EPS, _check_norm, _f64, _grad64, _inside, _rand, _weight
from tests.test_gpu_update import U, _adam64, _stats64

pytestmark = pytest.mark.gpu


def _leaf(t):
    return None if t is None else t.clone().requires_grad_()


@pytest.mark.parametrize("kind,wkind", [("float32", "float32"), ("bfloat16", "float32"), ("float16", "float16"),
                                        ("bfloat16", None)])
@pytest.mark.parametrize("with_residual", [True, False])
def test_add_rms_norm(kind, wkind, with_residual):
    import torch
    from paper_2006_03318_amd.training import add_rms_norm
    require_gpu()
    rng = np.random.default_rng(1)
    rows, cols = 37, 200
    x, w = _leaf(_rand(rng, rows, cols, kind)), _leaf(_weight(rng, cols, wkind))
    r = _leaf(_rand(rng, rows, cols, kind)) if with_residual else None
    dy, dh = _rand(rng, rows, cols, kind), _rand(rng, rows, cols, kind)
    if with_residual:
        y, h = add_rms_norm(x, r, w, EPS)
        torch.autograd.backward((y, h), (dy, dh))
    else:
        y, h = add_rms_norm(x, None, w, EPS), x
        y.backward(dy)
    _check_norm(x, r, w, y, h if with_residual else None, None, kind)
    rstd = torch.from_numpy(1 / np.sqrt((_f64(x) + (_f64(r) if with_residual else 0.0)) ** 2 @ np.ones((cols, 1)) / cols + EPS))[:, 0]
    x1, w1, ex, ew = _grad64(dy, h, w, rstd, dh if with_residual else None)
    # rstd itself is off by the forward pass's bound, and scales every term of both
    er = (cols / 16 + 40) * U
    terms = np.abs(x1 - (_f64(dh) if with_residual else 0.0))
    slack = er * (terms + 3 * np.abs(_f64(dy)) * (1.0 if w is None else np.abs(_f64(w))) * rstd.numpy()[:, None] + 3 * terms.max())
    assert _inside(x.grad, x1, ex * 1.01 + slack, kind)
    if with_residual:
        assert torch.equal(x.grad, r.grad)
    if w is not None:
        assert _inside(w.grad, w1, ew * 1.01 + er * np.sum(np.abs(_f64(dy) * _f64(h) * rstd.numpy()[:, None]), axis=0), wkind)


def test_add_rms_norm_shapes_and_unused_outputs():
    import torch
    from paper_2006_03318_amd.training import add_rms_norm
    require_gpu()
    rng = np.random.default_rng(2)
    x = _leaf(_rand(rng, 24, 64, "float32"))
    r = _leaf(_rand(rng, 1, 64, "float32"))
    y, h = add_rms_norm(x.view(2, 12, 64), r, None, EPS)            # one residual for all rows
    assert y.shape == h.shape == (2, 12, 64)
    h.backward(torch.ones_like(h))                                   # the norm's output is not used
    assert torch.equal(x.grad, torch.ones_like(x)) and torch.equal(r.grad, torch.full_like(r, 24.0))
    x.grad = r.grad = None
    wide = _rand(rng, 24, 64, "float32", pad=9)
    y, h = add_rms_norm(wide, r, None, EPS)
    y.sum().backward()                                               # the sum is not used
    _check_norm(wide, r.expand(24, 64), None, y, h, None, "float32")
    y2 = add_rms_norm(x.t().contiguous().t(), None, None, EPS)       # columns consecutive, not rows
    _check_norm(x, None, None, y2, None, None, "float32")


def test_second_derivatives_are_refused():
    import torch
    from paper_2006_03318_amd.training import add_rms_norm
    require_gpu()
    x = torch.randn(4, 32, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(add_rms_norm(x).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_adam(kind):
    import torch
    from paper_2006_03318_amd.training import Adam
    require_gpu()
    rng = np.random.default_rng(3)
    t = getattr(torch, kind)
    params = [torch.nn.Parameter(torch.from_numpy(rng.standard_normal(s)).to(t).cuda()) for s in ((33, 7), (129,), (64, 64))]
    opt = Adam(params, lr=0.02, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1, max_norm=1.0)
    for step in range(1, 4):
        opt.zero_grad()
        loss = sum(((p.float() - 0.5) ** 2).sum() for p in params)
        loss.backward()
        old = [(_f64(w), _f64(m), _f64(v)) for w, m, v in zip(opt.masters, opt.m, opt.v)]
        opt.step()
        grads = [p.grad for p in params]
        norm, f = _stats64(grads, 1.0)
        assert int(opt.steps) == step and abs(float(opt.stats[0]) - norm) <= 2 * U * norm and float(opt.stats[2]) == 0.0
        for p, g, w1, m1, v1, (w, m, v) in zip(params, grads, opt.masters, opt.m, opt.v, old):
            a, b, c, ew, em, ev = _adam64(_f64(g), w, m, v, step, f, p.dim() >= 2, 0.02, 0.8, 0.95, 1e-6, 0.1, True)
            assert np.all(np.abs(_f64(w1) - a) <= ew) and np.all(np.abs(_f64(m1) - b) <= em) and np.all(np.abs(_f64(v1) - c) <= ev)
            assert torch.equal(p.detach(), w1.to(t))
    kept = params[0].grad
    params[0].grad = torch.zeros_like(params[0])
    with pytest.raises(RuntimeError, match="replaced"):
        opt.step()
    params[0].grad = kept
    params[1].data = params[1].data.clone()
    with pytest.raises(RuntimeError, match="replaced"):
        opt.step()
    opt.close()


def test_adam_skips_an_overflow_of_the_scaled_loss():
    import torch
    from paper_2006_03318_amd.training import Adam
    require_gpu()
    p = torch.nn.Parameter(torch.ones(100, dtype=torch.float16, device="cuda"))
    opt = Adam([p], lr=0.1)
    scale = torch.tensor([2.0 ** 14], device="cuda")
    for factor, skipped in ((8.0, 1.0), (1.0, 0.0)):
        opt.zero_grad()
        ((p.float() * factor).sum() * scale[0]).backward()           # 2^17 overflows float16, 2^14 does not
        opt.step(inv_scale=1.0 / scale)
        assert float(opt.stats[2]) == skipped and int(opt.steps) == int(1 - skipped)
        assert bool((p == 1.0).all()) == bool(skipped)
    assert abs(float(opt.stats[0]) - math.sqrt(100)) <= 2 * U * 10


def test_iteration_fused_against_plain():
    """The same training run with single operations and with the fused ones.
    Both round to bf16 at the same places from values that differ in the last
    bits of 32, so single elements differ by one step of bf16, 2^-8 of them:
    no mean of squares differs by more than twice that, of which each step's
    update adds as much again."""
    from paper_2006_03318_amd import fused_iteration as F
    require_gpu()
    _, plain = F.train(hidden=256, layers=3, rows=500, steps=5, fused=False)
    _, fused = F.train(hidden=256, layers=3, rows=500, steps=5, fused=True, marked=True)
    say(plain, fused)
    for k, (a, b) in enumerate(zip(plain, fused)):
        assert abs(a - b) <= 2 * 2.0 ** -8 * (k + 1) * a
    assert fused[-1] < fused[0]


def test_predictions_match_the_oracle():
    import os
    from oracle import oracle as O
    from paper_2006_03318_amd import batch, fused_iteration as F, trace as TR
    require_gpu()
    gold = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "rocprof_cnn")
    rows, measured = F.predict(gold, [2, 3])
    g, vs, names = F.what_if(TR.build_graph(TR.read_rocprof_csv(gold), iterations=[2, 3]))
    _, _, ms, _ = O.run(g, vs)
    assert [n for n, _ in rows] == names and [t for _, t in rows] == [int(m) / 1e6 / 2 for m in ms]
    assert abs(rows[0][1] - measured) <= 0.01 * measured
