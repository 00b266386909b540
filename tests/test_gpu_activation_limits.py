"""Activations and their derivatives at infinities: the limits, through every call that has them."""
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def limits(act):
    """The derivative at minus and plus infinity."""
    return (1.0, 1.0) if act == "none" else (0.0, 1.0)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_activation_gradient(kind, act):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    inf, nan = float("inf"), float("nan")
    most = torch.finfo(t).max
    z = torch.tensor([-inf, inf, -most, most, -inf, inf, nan], device="cuda").to(t)
    dy = torch.tensor([1.0, 1.0, 3.0, 3.0, -2.0, -2.0, 1.0], device="cuda").to(t)
    dz = torch.empty_like(dy)
    B.dd_act_grad(dy, z, dz, act)
    torch.cuda.synchronize()
    low, high = limits(act)
    assert dz[:6].tolist() == [low, high, 3 * low, 3 * high, -2 * low, -2 * high]
    if act not in ("none", "relu"):        # (relu's is 1 above 0 and 0 elsewhere)
        assert bool(dz[6].isnan())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,k,n", [(5, 40, 24), (70, 64, 128), (131, 77, 33), (2304, 2048, 512)])
def test_product_gradient(rows, k, n, kind, act):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(k)
    dy, w = (torch.randint(-2, 3, s, generator=gen, device="cuda").to(t) for s in ((rows, n), (k, n)))
    up = torch.rand(rows, k, generator=gen, device="cuda") < 0.5
    z = torch.where(up, float("inf"), float("-inf")).to(t)
    dx = torch.empty(rows, k, device="cuda", dtype=t)
    B.dd_linear_grad(dy, w=w, dx=dx, in_act=act, in_z=z)
    torch.cuda.synchronize()
    low, high = limits(act)
    want = dy.double() @ w.double().t() * torch.where(up, high, low).double()
    assert torch.equal(dx, want.to(t))


@pytest.mark.parametrize("act", ACTS[1:])
def test_sums_that_float16_does_not_hold(act):
    """A sum of -80,000 is an output of 0, and the z that is kept of it -inf: its gradient is 0 as well."""
    import torch
    from paper_2006_03318_amd.training import linear, mlp
    require_gpu()
    x = torch.tensor([[200.0, -200.0]], device="cuda").half().requires_grad_()
    w = torch.tensor([[-200.0, 1.0], [200.0, 1.0]], device="cuda").half().requires_grad_()
    y = linear(x, w, act=act)
    assert y.tolist() == [[0.0, 0.0]]
    dx, dw = torch.autograd.grad(y, (x, w), torch.tensor([[1.0, 0.0]], device="cuda").half())
    assert not dx.any() and not dw.any()
    down = torch.tensor([[1.0], [0.0]], device="cuda").half().requires_grad_()
    grads = torch.autograd.grad(mlp(x, w, down, act=act), (x, w, down), torch.ones(1, 1, device="cuda").half())
    assert all(not g.any() for g in grads)


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
def test_infinite_sums(kind):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    x = torch.tensor([[float("-inf")], [float("inf")]], device="cuda").to(t)
    one, y = torch.ones(1, 1, device="cuda", dtype=t), torch.empty(2, 1, device="cuda", dtype=t)
    for act in ACTS:
        B.dd_linear(x, one, y, act=act)
        torch.cuda.synchronize()
        low, high = y.flatten().tolist()
        assert high == float("inf"), act
        assert low == {"none": float("-inf"), "relu": 0.0, "gelu": 0.0}[act] if act in ACTS[:3] else low != low, act
