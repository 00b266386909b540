"""Weights that others than the optimizer write, or read later."""
import numpy as np
import pytest

from tests.gpu_common import require_gpu
from tests.test_gpu_rms_norm import _f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_a_loaded_checkpoint_stays(kind):
    import torch
    from paper_2006_03318_amd.training import Adam
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(3)
    model = torch.nn.Linear(70, 30).to(getattr(torch, kind)).cuda()
    saved = {k: v.clone() for k, v in model.state_dict().items()}
    opt = Adam(model.parameters(), lr=0.05)
    for load in (False, True, False):
        if load:
            model.load_state_dict(saved)
        before = [_f64(p) for p in model.parameters()]
        opt.zero_grad()
        model(torch.randn(8, 70, generator=gen, device="cuda").to(getattr(torch, kind))).float().square().sum().backward()
        opt.step()
        # m_hat and sqrt(v_hat) are means of three gradients or fewer, whose weights a and b have sum(a^2 / b) < 1.01:
        # a step is at most 1.005 lr, and a 16-bit weight's roundings 2^-7 of it
        for p, b in zip(model.parameters(), before):
            assert np.all(np.abs(_f64(p) - b) <= 0.051 + 2.0 ** -7 * np.abs(b))
        if load:
            for p, b, k in zip(model.parameters(), before, saved):
                assert np.array_equal(b, _f64(saved[k]))
    with torch.no_grad():
        for p in model.parameters():
            p.fill_(100.0)
    opt.lr = 0.0
    opt.step()
    assert all(bool((p == 100.0).all()) for p in model.parameters())
    opt.close()


def test_a_graph_from_before_the_step_is_refused():
    import torch
    from paper_2006_03318_amd.training import Adam, add_rms_norm
    require_gpu()
    w = torch.nn.Parameter(torch.ones(64, dtype=torch.bfloat16, device="cuda"))
    x = torch.randn(10, 64, device="cuda").to(torch.bfloat16).requires_grad_()
    opt = Adam([w], lr=0.1)
    loss = add_rms_norm(x, None, w).float().square().sum()
    loss.backward(retain_graph=True)
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    opt.close()
