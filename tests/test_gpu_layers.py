"""The differentiable forms for torch programs: gradients against torch's own in 64 bits and
against differences, captured graphs, streams, and a run of them together."""
import math

import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


def act64(z, act):
    import torch
    return {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu,
            "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh"), "silu": torch.nn.functional.silu}[act](z)


def near(got, want, steps, label=""):
    """Off by that many roundings (half steps of got's type) of the largest value in 2-norm: each
    rounding of a 16-bit value between here and the inputs adds one at most."""
    import torch
    got, want = got.detach(), want.detach()
    off = float((got.double() - want).norm()) / (float(want.norm()) or 1.0)
    assert off <= steps * torch.finfo(got.dtype).eps / 2, "%s: %g" % (label, off)


def leaves(gen, kind, *shapes):
    import torch
    out = []
    for s in shapes:
        std = s[0] ** -0.5 if len(s) == 2 and s[0] > 1 else 1.0
        out.append((torch.randn(*s, generator=gen, device="cuda") * std).to(kind).requires_grad_())
    return out


def in64(ts):
    return [t.detach().double().requires_grad_() for t in ts]


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape,n,turned", [((40, 72), 136, False), ((3, 5, 33), 47, True), ((7,), 9, False), ((300, 256), 512, True)])
def test_linear(shape, n, turned, kind, act):
    import torch
    from paper_2006_03318_amd.training import linear
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(n)
    t = getattr(torch, kind)
    x, w, b, r = leaves(gen, t, shape, (n, shape[-1]) if turned else (shape[-1], n), (n,), shape[:-1] + (n,))
    y = linear(x, w.t() if turned else w, b, act, r)
    dy = torch.randn(y.shape, generator=gen, device="cuda").to(t)
    got = torch.autograd.grad(y, (x, w, b, r), dy)
    x64, w64, b64, r64 = in64((x, w, b, r))
    want = act64(x64 @ (w64.t() if turned else w64) + b64, act) + r64
    near(y, want.detach(), 2, "y")
    # z, dz and the gradient itself are rounded; 8 leaves room for a derivative that bends (z's rounding)
    for name, a, c in zip("xwbr", got, torch.autograd.grad(want, (x64, w64, b64, r64), dy.double())):
        assert a.shape == c.shape and a.dtype == t
        near(a, c, 8, "d" + name)


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,hidden,wide,bias_kind", [(50, 64, 256, "float32"), (5, 33, 70, "same"), (1, 128, 512, None)])
def test_mlp(rows, hidden, wide, bias_kind, kind):
    import torch
    from paper_2006_03318_amd.training import linear, mlp
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(wide)
    t = getattr(torch, kind)
    x, up, down, r = leaves(gen, t, (rows, hidden), (hidden, wide), (wide, hidden), (1, hidden))
    bu, bd = (None, None) if bias_kind is None else leaves(gen, t if bias_kind == "same" else torch.float32, (wide,), (hidden,))
    y = mlp(x, up, down, bu, bd, "gelu", r)
    assert torch.equal(y, linear(linear(x, up, bu, "gelu"), down, bd, residual=r))
    dy = torch.randn(y.shape, generator=gen, device="cuda").to(t)
    ins = [v for v in (x, up, down, bu, bd, r) if v is not None]
    got = torch.autograd.grad(y, ins, dy)
    c = dict(zip(map(id, ins), in64(ins)))
    p = lambda v: 0.0 if v is None else c[id(v)]  # noqa: E731
    want = act64(p(x) @ p(up) + p(bu), "gelu") @ p(down) + p(bd) + p(r)
    near(y, want.detach(), 4, "y")
    for i, (a, b) in enumerate(zip(got, torch.autograd.grad(want, [p(v) for v in ins], dy.double()))):
        assert a.shape == b.shape
        # (those of f32 come from values of 16 bits)
        near(a.to(t) if a.dtype != t else a, b, 10, str(i))


def test_linear_gradient_against_differences():
    """With relu, whose derivative is a step: sums are odd numbers of quarters, so a weight that moves by 2^-6 turns
    no sign and the difference is exact."""
    import torch
    from paper_2006_03318_amd.training import linear
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(8)
    x = torch.randint(-3, 4, (20, 24), generator=gen, device="cuda").to(torch.bfloat16)
    w = (torch.randint(-2, 3, (24, 16), generator=gen, device="cuda") + 0.5).to(torch.bfloat16).requires_grad_()
    b = torch.full((16,), 0.25, device="cuda")
    dw, = torch.autograd.grad(linear(x, w, b, "relu").float().sum(), w)
    for i, j in ((0, 0), (5, 7), (23, 15), (11, 3)):
        h = torch.zeros(24, 16, device="cuda", dtype=torch.float64)
        h[i, j] = 2.0 ** -6
        ahead, back = (torch.relu(x.double() @ (w.detach().double() + s * h) + 0.25).sum() for s in (1, -1))
        assert float(dw[i, j]) == float(((ahead - back) * 32).to(torch.bfloat16))


def test_only_what_is_wanted():
    import torch
    from paper_2006_03318_amd.training import embed, linear, mlp
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(9)
    x, w, b = leaves(gen, torch.bfloat16, (12, 16), (16, 24), (24,))
    for some in ((x,), (w,), (b,), (x, b)):
        for v in (x, w, b):
            v.requires_grad_(any(v is s for s in some))
            v.grad = None
        linear(x, w, b, "silu").sum().backward()
        assert [v.grad is not None for v in (x, w, b)] == [any(v is s for s in some) for v in (x, w, b)]
    with torch.no_grad():
        assert not linear(x, w, b, "gelu").requires_grad
    for v in (x, w, b):
        v.requires_grad_(False)
    down = leaves(gen, torch.bfloat16, (24, 16))[0]
    mlp(x, w, down, b).sum().backward()
    assert down.grad is not None and w.grad is None
    table = torch.ones(5, 8, device="cuda")
    assert not embed(torch.zeros(3, dtype=torch.int32, device="cuda"), table).requires_grad


def test_refusals():
    import torch
    from paper_2006_03318_amd.training import Dropout, embed, linear
    require_gpu()
    x, w = torch.ones(4, 8, device="cuda", dtype=torch.bfloat16), torch.ones(8, 8, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="weight"):
        linear(x, w.half())
    with pytest.raises(TypeError, match="residual"):
        linear(x, w, residual=x.float())
    with pytest.raises(ValueError, match="act"):
        linear(x, w, act="tanh")
    with pytest.raises(ValueError, match="empty"):
        linear(x[:, :0], w[:0])
    with pytest.raises(ValueError, match="device"):
        linear(x, w.cpu())
    with pytest.raises(B.DDError, match="p must"):
        Dropout()(x, 1.5)
    with pytest.raises(TypeError, match="ids"):
        embed(torch.zeros(3, device="cuda"), w)
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError, match="pad"):
        embed(ids, w, pad=8)
    for table in (w[0], w[None], w[:0]):
        with pytest.raises(ValueError, match="two dimensions"):
            embed(ids, table)
    y = linear(x.requires_grad_(), w)
    g, = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(40, 24), (3, 5, 7), (9,)])
def test_dropout(shape, kind):
    import torch
    from paper_2006_03318_amd.training import Dropout
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(2)
    x, r = leaves(gen, t, shape, shape[-1:])
    drop = Dropout(seed=-5)
    y = drop(x, 0.5, r)
    z = drop(x, 0.5)
    dx, dr = torch.autograd.grad(y.float().sum(), (x, r))
    assert set(dx.float().unique().tolist()) <= {0.0, 2.0}
    assert torch.equal(y, torch.where(dx != 0, 2 * x.float(), 0.0).add(r.float()).to(t))
    assert torch.equal(dr.float(), torch.full_like(r, x.numel() / shape[-1]).float())
    dz, = torch.autograd.grad(z.float().sum(), x)
    assert torch.equal(z, torch.where(dz != 0, 2 * x.float(), 0.0).to(t))
    # a step later the same calls have other masks; a new one of the same seed has the first again
    drop.step()
    assert drop.state[1].item() == 2 and drop.calls == 0
    if x.numel() > 100:
        assert not torch.equal(y, drop(x, 0.5, r)) and not torch.equal(dx != 0, dz != 0)
    assert torch.equal(y, Dropout(seed=-5)(x, 0.5, r))


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_embedding(kind):
    import torch
    from paper_2006_03318_amd.training import embed
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(6)
    table = torch.randint(-3, 4, (70, 40), generator=gen, device="cuda").to(t).requires_grad_()
    ids = torch.randint(0, 70, (30, 11), generator=gen, device="cuda")
    ids[:, 3] = 5
    y = embed(ids.t(), table, 4.0, pad=5)
    assert torch.equal(y, (4 * table.detach()[ids.t()]))
    dy = torch.randint(-3, 4, y.shape, generator=gen, device="cuda").to(t)
    got, = torch.autograd.grad(y, table, dy)
    want = torch.zeros(70, 40, dtype=torch.float64, device="cuda").index_add_(0, ids.t().reshape(-1), 4 * dy.reshape(-1, 40).double())
    want[5] = 0
    assert torch.equal(got, want.to(t))


def _model(kind, seed=0):
    """Embedding, two blocks of norm, mlp and dropout into the residual, and a product at the end."""
    import torch
    gen = torch.Generator("cuda").manual_seed(seed)

    def p(*shape):
        std = shape[0] ** -0.5 if len(shape) == 2 else 0.1
        return torch.nn.Parameter((torch.randn(*shape, generator=gen, device="cuda") * std).to(kind))
    return dict(table=p(50, 64), norm=[p(64), p(64)], up=[p(64, 256), p(64, 256)], down=[p(256, 64), p(256, 64)], bu=[p(256), p(256)],
                bd=[p(64), p(64)], head=p(50, 64))


def _forward(m, ids, drop):
    import torch
    from paper_2006_03318_amd.training import add_rms_norm, embed, linear, mlp
    h = embed(ids, m["table"], 8.0)
    x = torch.zeros_like(h)
    for i in range(2):
        y, h = add_rms_norm(x, h, m["norm"][i])
        x = drop(mlp(y, m["up"][i], m["down"][i], m["bu"][i], m["bd"][i], "gelu"), 0.1)
    y, _ = add_rms_norm(x, h, None)
    return linear(y, m["head"].t())


def _params(m):
    return [p for v in m.values() for p in (v if isinstance(v, list) else [v])]


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
def test_together_against_64_bits(kind):
    """The model's output and all its gradients against torch in 64 bits with the same masks (those
    that the dropout calls report)."""
    import torch
    from paper_2006_03318_amd.training import Dropout
    require_gpu()
    t = getattr(torch, kind)
    m = _model(t)
    gen = torch.Generator("cuda").manual_seed(7)
    ids = torch.randint(0, 50, (6, 37), generator=gen, device="cuda")
    out = _forward(m, ids, Dropout(3))
    dy = torch.randn(out.shape, generator=gen, device="cuda").to(t)
    got = torch.autograd.grad(out, _params(m), dy)
    shape = (6, 37, 64)
    again, ones = Dropout(3), torch.ones(shape, device="cuda")
    masks = [again(ones, 0.1).double() for _ in range(2)]
    c = {k: [p.detach().double().requires_grad_() for p in v] if isinstance(v, list) else v.detach().double().requires_grad_() for k, v in m.items()}
    h, x = c["table"][ids] * 8.0, torch.zeros(shape, dtype=torch.float64, device="cuda")

    def norm(v, w):
        return v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
    for i in range(2):
        h = x + h
        x = (torch.nn.functional.gelu(norm(h, c["norm"][i]) @ c["up"][i] + c["bu"][i]) @ c["down"][i] + c["bd"][i]) * masks[i]
    want = norm(x + h, 1.0) @ c["head"].t()
    # about five roundings on each of three stages, each kept or halved by the next
    near(out, want.detach(), 16, "out")
    for i, (a, b) in enumerate(zip(got, torch.autograd.grad(want, _params(c), dy.double()))):
        near(a, b, 32, str(i))


def test_together_captured():
    """A whole step in a graph, replayed with other tokens on the capture's stream, the library's cache emptied and
    eager steps of another model between: every replay gives what the eager step gives."""
    import torch
    from paper_2006_03318_amd.training import Adam, Dropout
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(5)
    ids = torch.randint(0, 50, (300,), generator=gen, device="cuda")
    dy = torch.randn(300, 50, generator=gen, device="cuda").to(torch.bfloat16)

    def make():
        m = _model(torch.bfloat16)
        return m, Adam(_params(m), lr=0.01, max_norm=1.0), Dropout(11)

    def step(m, opt, drop):
        opt.zero_grad()
        _forward(m, ids, drop).backward(dy)
        opt.step()
        drop.step()

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        mine = make()
        step(*mine)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(*mine)
    other = make()
    step(*other)
    for k in range(4):
        ids.copy_(torch.randint(0, 50, (300,), generator=gen, device="cuda"))
        dy.mul_(-1.5)
        step(*other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(_params(mine[0]), _params(other[0]))), k
        assert torch.equal(mine[2].state, other[2].state) and mine[2].state[1].item() == 2 * (k + 2)
        B.dd_release_cache()
    del graph
    mine[1].close()
    other[1].close()


def test_captured_calls_without_working_memory_are_refused():
    import torch
    require_gpu()
    t = torch.bfloat16
    x, w, y = torch.ones(4, 8192, device="cuda", dtype=t), torch.ones(8192, 64, device="cuda", dtype=t), torch.empty(4, 64, device="cuda", dtype=t)
    ids, dt = torch.zeros(40, dtype=torch.int64, device="cuda"), torch.empty(30, 64, device="cuda", dtype=t)
    dy = torch.ones(40, 64, device="cuda", dtype=t)
    room = [torch.empty(B.dd_linear_work(4, 8192, 64), dtype=torch.uint8, device="cuda"),
            torch.empty(B.dd_embed_grad_work(40, 30, 64), dtype=torch.uint8, device="cuda")]
    B.dd_linear(x, w, y)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for call in (lambda: B.dd_linear(x, w, y, stream=side), lambda: B.dd_embed_grad(ids, dy, dt, stream=side)):
            with pytest.raises(B.DDError, match="work"):
                call()
        B.dd_linear(x, w, y, work=room[0], stream=side)
        B.dd_embed_grad(ids, dy, dt, work=room[1], stream=side)
    for k in range(3):
        y.zero_(), dt.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert bool((y == 8192).all()) and bool((dt[0] == 40).all()) and not dt[1:].any()
    with pytest.raises(ValueError, match="work must hold"):
        B.dd_linear(x, w, y, work=room[0][:16])


def test_two_streams_at_once():
    """Calls with sums that are cut, on two streams, with memory of the library's: neither sees the other's."""
    import torch
    require_gpu()
    t = torch.bfloat16
    gen = torch.Generator("cuda").manual_seed(12)
    n = 60000
    xs = [torch.randint(-2, 3, (8, 16384), generator=gen, device="cuda").to(t) for _ in range(2)]
    w = torch.randint(-2, 3, (16384, 256), generator=gen, device="cuda").to(t)
    ids = [torch.randint(0, 100, (n,), generator=gen, device="cuda") for _ in range(2)]
    dy = torch.randint(-2, 3, (n, 72), generator=gen, device="cuda").float()
    ys, ds = [torch.empty(8, 256, device="cuda", dtype=t) for _ in range(2)], [torch.empty(100, 72, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, x, y, i, d in zip(streams, xs, ys, ids, ds):
            B.dd_linear(x, w, y, stream=s)
            B.dd_embed_grad(i, dy, d, stream=s)
    torch.cuda.synchronize()
    for x, y, i, d in zip(xs, ys, ids, ds):
        assert torch.equal(y, (x.double() @ w.double()).to(t))
        assert torch.equal(d.double(), torch.zeros(100, 72, dtype=torch.float64, device="cuda").index_add_(0, i, dy.double()))


def test_no_rows():
    """Batches without rows: outputs without rows, gradients that are zeros."""
    import torch
    from paper_2006_03318_amd.training import Dropout, embed, linear, mlp
    require_gpu()
    t = torch.bfloat16
    w, v, b = (torch.ones(s, device="cuda", dtype=t, requires_grad=True) for s in ((24, 40), (40, 24), (40,)))
    x = torch.ones(3, 0, 24, device="cuda", dtype=t, requires_grad=True)
    ids = torch.zeros(0, 5, dtype=torch.int64, device="cuda")
    for y, leaves_ in ((linear(x, w, b, "gelu"), (x, w, b)), (mlp(x, w, v, b), (x, w, v, b)), (embed(ids, w), (w,)), (Dropout()(x, 0.5), (x,))):
        assert y.numel() == 0
        for p, g in zip(leaves_, torch.autograd.grad(y.sum(), leaves_)):
            assert g.shape == p.shape and not g.any()
