"""Products and their gradients on every path that the plan has for them, in whole numbers, whose sums have
no rounding: the rounded truth, bit for bit."""
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu
from tests.product_cases import CASES
from tests.test_gpu_linear import Rows, act64, check, matrix, rand

pytestmark = pytest.mark.gpu


def name(case):
    return "-".join(map(str, case[:6]))


@pytest.mark.parametrize("case", [c for c in CASES if c[0] == "fwd"], ids=name)
def test_products(case):
    """With a bias, relu, a residual and z, in buffers whose gaps are NaNs, or a number that stays."""
    import torch
    require_gpu()
    _, rows, k, n, pad, turned, _ = case
    t = (torch.bfloat16, torch.float16)[CASES.index(case) % 2]
    gen = torch.Generator("cuda").manual_seed(rows + 3 * k + 7 * n)
    whole = lambda *s: torch.randint(-2, 3, s, generator=gen, device="cuda").to(t)  # noqa: E731
    x, w, bias, residual = whole(rows, k), whole(k, n), whole(n).float(), whole(rows, n)
    y, z = (Rows(torch.zeros(rows, n, device="cuda", dtype=t), pad, 7.0) for _ in range(2))
    B.dd_linear(Rows(x, pad).t, matrix(w, turned, pad), y.t, bias=bias, residual=Rows(residual, pad).t, act="relu", z=z.t)
    torch.cuda.synchronize()
    want = x.double() @ w.double() + bias.double()
    assert torch.equal(z.t, want.to(t))
    assert torch.equal(y.t, (want.clamp(min=0) + residual.double()).to(t))
    assert y.rest_is_kept() and z.rest_is_kept()


@pytest.mark.parametrize("case", [c for c in CASES if c[0] == "grad"], ids=name)
def test_gradients(case):
    """All three, through relu."""
    import torch
    require_gpu()
    _, rows, k, n, pad, turned, _ = case
    t = (torch.bfloat16, torch.float16)[CASES.index(case) % 2]
    gen = torch.Generator("cuda").manual_seed(rows + 3 * k + 7 * n)
    whole = lambda *s: torch.randint(-2, 3, s, generator=gen, device="cuda").to(t)  # noqa: E731
    dy, x, w, z = whole(rows, n), whole(rows, k), whole(k, n), whole(rows, k)
    dx = Rows(torch.zeros(rows, k, device="cuda", dtype=t), pad, 7.0)
    dw = Rows(torch.zeros((n, k) if turned else (k, n), device="cuda", dtype=t), pad, 7.0)
    db = torch.empty(n, device="cuda")
    B.dd_linear_grad(Rows(dy, pad).t, Rows(x, pad).t, matrix(w, turned, pad), dx=dx.t, dw=dw.t.t() if turned else dw.t, db=db, in_act="relu",
                     in_z=Rows(z, pad).t)
    torch.cuda.synchronize()
    assert torch.equal(dx.t, ((dy.double() @ w.double().t()) * (z > 0)).to(t))
    want = x.double().t() @ dy.double()
    assert torch.equal(dw.t, (want.t() if turned else want).to(t))
    assert torch.equal(db.double(), dy.double().sum(0))
    assert dx.rest_is_kept() and dw.rest_is_kept()


# many tiles of 256 x 256 a workgroup, the last ragged
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("kind,act", [("bfloat16", "gelu"), ("float16", "silu"), ("bfloat16", "gelu_tanh")])
def test_epilogues_between_tiles(kind, act, turned):
    """Against the formulas in 64 bits, within the bounds that the tests of the product derive."""
    import torch
    require_gpu()
    t = getattr(torch, kind)
    rows, k, n = 16389, 520, 4104
    gen = torch.Generator("cuda").manual_seed(k)
    x, w, residual = rand(gen, rows, k, t, 2.0), rand(gen, k, n, t, k ** -0.5), rand(gen, rows, n, t, 3.0)
    bias = rand(gen, 1, n, torch.float32)[0]
    y, z = torch.empty(rows, n, device="cuda", dtype=t), torch.empty(rows, n, device="cuda", dtype=t)
    B.dd_linear(x, matrix(w, turned, 0), y, bias=bias, residual=residual, act=act, z=z)
    torch.cuda.synchronize()
    want = x.double() @ w.double() + bias.double()
    slack = (k + 8) * 2.0 ** -23 * (x.double().abs() @ w.double().abs() + bias.double().abs())
    check("z", z, want, slack)
    check("y", y, act64(want, act)[0] + residual.double(), 1.2 * slack + 2.0 ** -20 * (want.abs() + residual.double().abs()))
    # the other way: rows of n back to rows of k, whose z this is
    dy, back, in_z = rand(gen, rows, k, t), rand(gen, n, k, t, k ** -0.5), rand(gen, rows, n, t, 2.0)
    dx = torch.empty(rows, n, device="cuda", dtype=t)
    B.dd_linear_grad(dy, w=matrix(back, turned, 0), dx=dx, in_act=act, in_z=in_z)
    torch.cuda.synchronize()
    first, size = dy.double() @ back.double().t(), dy.double().abs() @ back.double().abs().t()
    check("dx", dx, first * act64(in_z.double(), act)[1], 1.2 * (k + 8) * 2.0 ** -23 * size + 2.0 ** -20 * first.abs() * (1 + in_z.double().abs()))


@pytest.mark.parametrize("rows,k,n", [(256, 256, 256), (40, 72, 88), (2048, 136, 2048), (300, 1024, 520), (4096, 512, 64), (16, 4096, 1024),
                                      (12001, 1544, 4104)])
def test_a_gradient_alone_has_the_bits_that_it_has_beside_the_other(rows, k, n):
    """Where operands load directly."""
    import torch
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(n)
    for turned in (False, True):
        dy, x, w = rand(gen, rows, n, torch.bfloat16), rand(gen, rows, k, torch.bfloat16), matrix(rand(gen, k, n, torch.bfloat16), turned, 0)
        one, both = [torch.empty_like(x), torch.empty_like(w)], [torch.empty_like(x), torch.empty_like(w)]
        B.dd_linear_grad(dy, x, w, dx=both[0], dw=both[1])
        B.dd_linear_grad(dy, w=w, dx=one[0])
        B.dd_linear_grad(dy, x=x, dw=one[1])
        torch.cuda.synchronize()
        assert torch.equal(one[0], both[0]) and torch.equal(one[1], both[1])


def test_rows_longer_than_a_load_reaches():
    """Rows of 17,100,001 elements: 64 of them are more than 2 GiB, which the offset of a load does not reach, so
    no operand is copied to be loaded so."""
    import torch
    require_gpu()
    rows, k, n, step = 129, 66, 17100001, 1 << 20
    gen = torch.Generator("cuda").manual_seed(1)
    whole = lambda *s: torch.randint(-1, 2, s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, w, dy = whole(rows, k), torch.empty(k, n, device="cuda", dtype=torch.bfloat16), torch.empty(rows, n, device="cuda", dtype=torch.bfloat16)
    parts = [slice(c, min(c + step, n)) for c in range(0, n, step)]
    for c in parts:
        w[:, c], dy[:, c] = whole(k, c.stop - c.start), whole(rows, c.stop - c.start)
    y, dx, dw = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w)
    B.dd_linear(x, w, y)
    B.dd_linear_grad(dy, x, w, dx=dx, dw=dw)
    torch.cuda.synchronize()
    want = torch.zeros(rows, k, device="cuda", dtype=torch.float64)
    for c in parts:
        assert torch.equal(y[:, c], (x.float() @ w[:, c].float()).to(torch.bfloat16)), c
        assert torch.equal(dw[:, c], (x.float().t() @ dy[:, c].float()).to(torch.bfloat16)), c
        want += dy[:, c].double() @ w[:, c].double().t()
    assert torch.equal(dx, want.to(torch.bfloat16))


@pytest.mark.parametrize("case", [c for c in CASES if "cut" in c[6] or "c" in c[6].replace("direct", "").replace("rounds", "")][::5], ids=name)
def test_working_memory_of_a_call(case):
    """A function is asked for what the call uses: no less, as nothing behind it is touched, and the same bits."""
    import torch
    require_gpu()
    op, rows, k, n, pad, turned, _ = case
    gen = torch.Generator("cuda").manual_seed(k)
    x, w, dy = (Rows(rand(gen, a, b, torch.bfloat16), pad).t for a, b in ((rows, k), (n, k) if turned else (k, n), (rows, n)))
    asked = []

    def give(size):
        asked.append(torch.full((1024 + size + 4096,), 171, device="cuda", dtype=torch.uint8))
        return asked[-1][1024:1024 + size]
    got = []
    for work in (None, give):
        y, dx, dw, db = (torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in ((rows, n), (rows, k), w.shape, (n,)))
        if op == "fwd":
            B.dd_linear(x, w.t() if turned else w, y, work=work)
        else:
            B.dd_linear_grad(dy, x, w.t() if turned else w, dx=dx, dw=dw.t() if turned else dw, db=db, work=work)
        torch.cuda.synchronize()
        got.append((y, dx, dw, db))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert len(asked) == 1 and bool((asked[0][:1024] == 171).all()) and bool((asked[0][-4096:] == 171).all())


def test_layers_take_no_memory_that_they_do_not_use():
    """Aligned rows: the gradient's peak is its outputs, dz and the sums' parts."""
    import torch
    from paper_2006_03318_amd.training import linear
    require_gpu()
    x, w = (torch.ones(s, device="cuda", dtype=torch.bfloat16, requires_grad=True) for s in ((8192, 1024), (1024, 1024)))
    for _ in range(2):
        x.grad = w.grad = None
        y = linear(x, w, act="relu")
        dy = torch.ones_like(y)
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        y.backward(dy)
        torch.cuda.synchronize()
        over = torch.cuda.max_memory_allocated() - before
    assert over <= 2 * x.numel() * 2 + w.numel() * 2 + (2 << 20)
