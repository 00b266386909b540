"""Adam where numbers are small beside others: what has to survive the rounding
of a step."""
import numpy as np
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu
from tests.test_gpu_update import List, _adam64, _f64, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1 << 18, 1 << 21])       # one launch, and two
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("decay", [1e-6, 1e-7, 1e-8])
def test_small_weight_decay(n, kind, decay):
    """lr * weight_decay below the grid of 32 bits at 1.  Weights in [1, 2) change
    by about 1e-3 either way, so the rounding of a step is as good as random: up
    to half of 2^-23, 2^-23 / sqrt(12) in the mean square, and the mean over n
    weights is within six times that / sqrt(n) (and 2^-22 of the decay, for its
    own roundings) of the mean in 64 bits."""
    import torch
    require_gpu()
    rng = np.random.default_rng(n + len(kind))
    w = torch.from_numpy(1 + rng.random(n)).float().clamp(max=1.999).cuda()
    g, m = (torch.from_numpy(rng.standard_normal(n)).float().cuda() for _ in range(2))
    v = torch.from_numpy(0.5 + rng.random(n)).float().cuda()
    t = dict(grad=g, param=w, m=m, v=v)
    if kind != "float32":
        t.update(param=w.to(_t(kind)), master=w)
    li = List([t])
    step = torch.full((1,), 1000, dtype=torch.int64, device="cuda")
    lr, drift, want = 1e-3, 0.0, 0.0
    for k in range(4):
        old = _f64(w), _f64(m), _f64(v)
        B.dd_adam_step(li.h, step, lr=lr, weight_decay=decay / lr)
        w1 = _adam64(_f64(g), *old, 1001 + k, 1.0, True, lr, 0.9, 0.999, 1e-8, decay / lr, True)[0]
        drift += float(np.mean(_f64(w) - w1))
        want += decay * float(np.mean(old[0]))
    assert abs(drift) <= 4 * 6 * 2.0 ** -23 / np.sqrt(12 * n) + 2.0 ** -22 * want


@pytest.mark.parametrize("n", [1000, 1 << 20])
@pytest.mark.parametrize("value,beta2", [(1e20, 0.999), (-5e20, 0.999), (1e20, 0.99), (3e18, 0.5)])
def test_second_moment_of_large_gradients(n, value, beta2):
    """(1 - beta2) g^2 within the range of 32 bits, though g^2 is not."""
    import torch
    require_gpu()
    g = torch.full((n,), value, device="cuda")
    w, m, v = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    li = List([dict(grad=g, param=w, m=m, v=v)])
    B.dd_adam_step(li.h, torch.zeros(1, dtype=torch.int64, device="cuda"), lr=0.25, beta2=beta2)
    one = np.ones(1)
    w1, m1, v1, ew, em, ev = _adam64(_f64(g)[:1], one, 0 * one, 0 * one, 1, 1.0, True, 0.25, 0.9, beta2, 1e-8, 0.0, True)
    assert np.all(np.abs(_f64(v) - v1) <= ev) and np.all(np.abs(_f64(m) - m1) <= em)
    assert np.all(np.abs(_f64(w) - w1) <= ew)


@pytest.mark.parametrize("n", [1000, 1 << 20])
@pytest.mark.parametrize("eps", [1e-42, 1e-60, 1e-300])
def test_eps_below_the_range_of_32_bits(n, eps):
    """Weights without a gradient stay where they are for any eps above 0."""
    import torch
    require_gpu()
    w = torch.linspace(-2, 2, n, device="cuda")
    g, m, v, before = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), w.clone()
    li = List([dict(grad=g, param=w, m=m, v=v)])
    B.dd_adam_step(li.h, torch.zeros(1, dtype=torch.int64, device="cuda"), lr=0.1, eps=eps)
    assert torch.equal(w, before)
