"""dd_linear, dd_linear_grad and dd_act_grad against the formulas in 64 bits.

Tolerances: a stored value is off by half a step of its type (eps / 2 relative, and half of the
smallest number); a sum of k products (each exact in 32 bits) by (k + 8) steps of 2^-23 of the sum of
their magnitudes at most; an activation changes its argument's error by a factor of 1.2 at most and
adds 2^-20 of the argument."""
import math

import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def act64(z, act):
    """The activation and its derivative."""
    import torch
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        phi = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        s = torch.sigmoid(2 * c * (z + 0.044715 * z ** 3))
        return z * s, s + z * s * (1 - s) * 2 * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def step(t):
    """Half a step: (relative, absolute)."""
    import torch
    f = torch.finfo(t)
    return f.eps / 2, f.smallest_normal * f.eps / 2


def check(label, got, want, slack):
    """|got - want| <= half a step of got's type + slack, everywhere."""
    rel, least = step(got.dtype)
    off = (got.double() - want).abs() - (rel * want.abs() * (1 + rel) + least + slack * (1 + rel))
    assert bool((off <= 0).all()), "%s: off by %g too much" % (label, float(off.max()))


class Rows:
    """Rows in a wider buffer of NaNs (outputs: of a number that stays), or end to end."""
    def __init__(self, values, pad, fill=float("nan")):
        import torch
        self.wide = torch.full((values.shape[0] + (1 if pad else 0), values.shape[1] + pad), fill, dtype=values.dtype, device="cuda")
        self.t = self.wide[:values.shape[0], :values.shape[1]]
        self.t.copy_(values)
        self.fill = fill

    def rest_is_kept(self):
        import torch
        rest = self.wide.clone()
        rest[:self.t.shape[0], :self.t.shape[1]] = self.fill
        return bool((rest == self.fill).all())


def rand(gen, rows, cols, kind, std=1.0):
    import torch
    return (torch.randn(rows, cols, generator=gen, device="cuda") * std).to(kind)


def matrix(values, turned, pad):
    """[k, n] values by rows or by columns, in a buffer with padding of NaNs."""
    if not turned:
        return Rows(values, pad).t
    return Rows(values.t(), pad).t.t()


# rows, k, n; padding: tiles of 16, 128 and 256 rows, direct loads (aligned) and others, sums cut and not
SHAPES = [
    (1, 1, 1, 0), (1, 8, 8, 0), (3, 64, 128, 8), (16, 200, 136, 0), (17, 72, 40, 8), (15, 333, 7, 3), (4, 2048, 1024, 0), (2, 5000, 9, 1),
    (130, 64, 256, 0), (128, 1, 128, 0), (257, 136, 264, 8), (300, 321, 130, 5), (129, 127, 129, 0), (100, 4104, 104, 16), (33, 1031, 65, 0),
    (2048, 96, 1032, 8), (2049, 511, 999, 1), (4096, 128, 4096, 0), (1, 63, 70000, 0), (70000, 9, 3, 0),
    (4400, 64, 8192, 0), (4400, 136, 8201, 0), (6000, 72, 1032, 1), (40, 512, 264, 1), (64, 4096, 1000, 0), (65, 4096, 1000, 3), (1300, 1024, 1300, 0),
]


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,k,n,pad", SHAPES)
def test_whole_numbers_are_exact(rows, k, n, pad, kind, turned):
    """Sums of small whole numbers have no rounding: forward and all gradients are the rounded
    truth, bit for bit."""
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(rows + 3 * k + 7 * n)

    def whole(a, b):
        return torch.randint(-2, 3, (a, b), generator=gen, device="cuda").to(t)

    x, w, dy = whole(rows, k), whole(k, n), whole(rows, n)
    bias, residual = whole(1, n)[0], whole(rows, n)
    px, pw, pd, pr = Rows(x, pad).t, matrix(w, turned, pad), Rows(dy, pad).t, Rows(residual, pad).t
    y = Rows(torch.zeros(rows, n, device="cuda", dtype=t), pad, 7.0)
    z = Rows(torch.zeros(rows, n, device="cuda", dtype=t), pad, 7.0)
    B.dd_linear(px, pw, y.t, bias=bias, residual=pr, z=z.t)
    torch.cuda.synchronize()
    want = x.double() @ w.double() + bias.double()
    assert torch.equal(z.t, want.to(t))
    assert torch.equal(y.t, (want + residual.double()).to(t))
    assert y.rest_is_kept() and z.rest_is_kept()
    dx = Rows(torch.zeros(rows, k, device="cuda", dtype=t), pad, 7.0)
    dw = Rows(torch.zeros((n, k) if turned else (k, n), device="cuda", dtype=t), pad, 7.0)
    db = torch.empty(n, device="cuda")
    B.dd_linear_grad(pd, px, pw, dx=dx.t, dw=dw.t.t() if turned else dw.t, db=db)
    torch.cuda.synchronize()
    assert torch.equal(dx.t, (dy.double() @ w.double().t()).to(t))
    want = x.double().t() @ dy.double()
    assert torch.equal(dw.t, (want.t() if turned else want).to(t))
    assert torch.equal(db.double(), dy.double().sum(0))
    assert dx.rest_is_kept() and dw.rest_is_kept()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind,bias_kind", [("bfloat16", "float32"), ("float16", "float16"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("rows,k,n,pad", [(1, 300, 77, 0), (16, 512, 640, 8), (200, 264, 520, 0), (257, 131, 515, 3), (2304, 64, 2048, 0)])
def test_epilogue(rows, k, n, pad, kind, bias_kind, act):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(k)
    x, w = rand(gen, rows, k, t, 2.0), rand(gen, k, n, t, k ** -0.5)
    bias, residual = rand(gen, 1, n, getattr(torch, bias_kind))[0], rand(gen, rows, n, t, 3.0)
    y, z = (Rows(torch.zeros(rows, n, device="cuda", dtype=t), pad, 7.0) for _ in range(2))
    B.dd_linear(Rows(x, pad).t, w, y.t, bias=bias, residual=Rows(residual, pad).t, act=act, z=z.t)
    torch.cuda.synchronize()
    want = x.double() @ w.double() + bias.double()
    slack = (k + 8) * 2.0 ** -23 * (x.double().abs() @ w.double().abs() + bias.double().abs())
    check("z", z.t, want, slack)
    value, _ = act64(want, act)
    check("y", y.t, value + residual.double(), 1.2 * slack + 2.0 ** -20 * (want.abs() + residual.double().abs()))
    # without bias, residual and z; and into the residual
    B.dd_linear(Rows(x, pad).t, w, y.t, act=act)
    into = residual.clone()
    B.dd_linear(x, w, into, residual=into, act=act)
    torch.cuda.synchronize()
    want = x.double() @ w.double()
    value, _ = act64(want, act)
    check("y alone", y.t, value, 1.2 * slack + 2.0 ** -20 * want.abs())
    check("y in place", into, value + residual.double(), 1.2 * slack + 2.0 ** -20 * (want.abs() + residual.double().abs()))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,k,n,pad", [(1, 77, 300, 0), (16, 640, 512, 8), (200, 520, 264, 0), (257, 515, 131, 3), (2304, 2048, 64, 0)])
def test_gradient(rows, k, n, pad, kind, act):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(n)
    dy, x, w, z = rand(gen, rows, n, t), rand(gen, rows, k, t), rand(gen, k, n, t, n ** -0.5), rand(gen, rows, k, t, 2.0)
    dx = Rows(torch.zeros(rows, k, device="cuda", dtype=t), pad, 7.0)
    dw, db = torch.empty(k, n, device="cuda", dtype=t), torch.empty(n, device="cuda")
    B.dd_linear_grad(Rows(dy, pad).t, Rows(x, pad).t, w, dx=dx.t, dw=dw, db=db, in_act=act, in_z=Rows(z, pad).t)
    torch.cuda.synchronize()
    slope = act64(z.double(), act)[1]
    first = dy.double() @ w.double().t()
    size = dy.double().abs() @ w.double().abs().t()
    check("dx", dx.t, first * slope, 1.2 * (n + 8) * 2.0 ** -23 * size + 2.0 ** -20 * first.abs() * (1 + z.double().abs()))
    check("dw", dw, x.double().t() @ dy.double(), (rows + 8) * 2.0 ** -23 * (x.double().abs().t() @ dy.double().abs()))
    check("db", db, dy.double().sum(0), (rows + 8) * 2.0 ** -23 * dy.double().abs().sum(0))
    # dx where x or in_z were
    for place in (x.clone(), z.clone()):
        B.dd_linear_grad(dy, None, w, dx=place, in_act=act, in_z=place if torch.equal(place, z) else z)
        torch.cuda.synchronize()
        assert torch.equal(place, dx.t)
    both = x.clone()
    B.dd_linear_grad(dy, both, w, dx=both, dw=dw, in_act=act, in_z=z)
    torch.cuda.synchronize()
    assert torch.equal(both, dx.t)
    check("dw", dw, x.double().t() @ dy.double(), (rows + 8) * 2.0 ** -23 * (x.double().abs().t() @ dy.double().abs()))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 1001, 5), (64, 512, 8)])
def test_activation_gradient(rows, cols, pad, kind, act):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(cols)
    dy, z = rand(gen, rows, cols, t), rand(gen, rows, cols, t, 3.0)
    dz = Rows(torch.zeros(rows, cols, device="cuda", dtype=t), pad, 7.0)
    B.dd_act_grad(Rows(dy, pad).t, Rows(z, pad).t, dz.t, act)
    torch.cuda.synchronize()
    check("dz", dz.t, dy.double() * act64(z.double(), act)[1], 2.0 ** -20 * dy.double().abs() * (1 + z.double().abs()))
    assert dz.rest_is_kept()
    again = dy.clone()
    B.dd_act_grad(again, z, again, act)
    torch.cuda.synchronize()
    assert torch.equal(again, dz.t)


@pytest.mark.parametrize("act", ACTS[1:])
def test_derivative_is_that_of_the_activation(act):
    """Against differences of the forward pass: h = 2^-6 in 64 bits of the kernel's own values would
    lose them, so the two are compared through the formula's differences, off by h^2 / 6 times a
    third derivative of at most 3."""
    import torch
    require_gpu()
    z = torch.linspace(-6, 6, 4001, device="cuda")
    z = z[z.abs() > 0.01]
    dz = torch.empty_like(z)
    B.dd_act_grad(torch.ones_like(z), z, dz, act)
    h = 2.0 ** -10
    diff = (act64(z.double() + h, act)[0] - act64(z.double() - h, act)[0]) / (2 * h)
    assert float((dz.double() - diff).abs().max()) <= h * h / 2 + 2.0 ** -20 * 7


@pytest.mark.parametrize("act", ACTS)
def test_special_values_stay_in_their_row_and_column(act):
    """An infinity or a NaN in a row of x, a column of w or one place of the residual reaches that row,
    column or place alone; far arguments give the activation's limits."""
    import torch
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(1)
    rows, k, n = 150, 200, 264
    x, w, residual = (rand(gen, a, b, torch.bfloat16) for a, b in ((rows, k), (k, n), (rows, n)))
    clean = torch.empty(rows, n, device="cuda", dtype=torch.bfloat16)
    B.dd_linear(x, w, clean, residual=residual, act=act)
    x[17, 3], x[18, 199], w[70, 250], residual[5, 6] = float("nan"), float("inf"), float("nan"), float("nan")
    y = torch.empty_like(clean)
    B.dd_linear(x, w, y, residual=residual, act=act)
    torch.cuda.synchronize()
    hit = torch.zeros(rows, n, dtype=torch.bool, device="cuda")
    hit[17] = hit[18] = True
    hit[:, 250] = True
    hit[5, 6] = True
    assert torch.equal(y[~hit], clean[~hit])
    assert bool(y[17].isnan().all()) and bool(y[:, 250].isnan().all()) and bool(y[5, 6].isnan())
    one = torch.eye(16, device="cuda", dtype=torch.bfloat16)
    far = torch.tensor([-1e30, -300.0, -40.0, 0.0, 40.0, 300.0, 1e30] + [1.0] * 9, device="cuda").repeat(16, 1).to(torch.bfloat16)
    out = torch.empty_like(far)
    B.dd_linear(one, far, out, act=act)
    torch.cuda.synchronize()
    # (silu(-40) = -40 / (1 + e^40) = -1.7e-16, the others' are nearer to the limits)
    want = act64(far.double(), act)[0].to(torch.bfloat16)
    assert bool(((out - want)[:, :7].abs() <= 2.0 ** -52).all())


def test_same_bits_again_and_with_given_memory():
    import torch
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(3)
    for rows, k, n in ((3, 4096, 520), (70, 8192, 136), (8192, 24, 40)):
        x, w, dy = (rand(gen, a, b, torch.float16) for a, b in ((rows, k), (k, n), (rows, n)))
        got = []
        for i in range(3):
            y, dx, dw, db = (torch.full(s, float(i), device="cuda", dtype=torch.float16) for s in ((rows, n), (rows, k), (k, n), (n,)))
            a, b = B.dd_linear_work(rows, k, n), B.dd_linear_grad_work(rows, k, n)
            assert a > 0 or b > 0
            work = torch.full((max(a, b, 16),), 255, device="cuda", dtype=torch.uint8) if i else None
            B.dd_linear(x, w, y, work=work)
            B.dd_linear_grad(dy, x, w, dx=dx, dw=dw, db=db, work=work)
            torch.cuda.synchronize()
            got.append((y, dx, dw, db))
        for other in got[1:]:
            assert all(torch.equal(p, q) for p, q in zip(got[0], other))


def test_no_rows():
    import torch
    require_gpu()
    t = torch.bfloat16
    x, dy = torch.empty(0, 24, device="cuda", dtype=t), torch.empty(0, 40, device="cuda", dtype=t)
    w = torch.ones(24, 40, device="cuda", dtype=t)
    B.dd_linear(x, w, torch.empty(0, 40, device="cuda", dtype=t))
    dw, db = torch.ones_like(w), torch.ones(40, device="cuda")
    B.dd_linear_grad(dy, x, w, dx=torch.empty_like(x), dw=dw, db=db)
    torch.cuda.synchronize()
    assert not dw.any() and not db.any()


def test_each_gradient_alone_and_layouts_that_differ():
    import torch
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(4)
    rows, k, n = 45, 72, 88
    dy, x, w = (torch.randint(-2, 3, s, generator=gen, device="cuda").to(torch.bfloat16) for s in ((rows, n), (rows, k), (k, n)))
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, device="cuda", dtype=torch.bfloat16)
    B.dd_linear_grad(dy, w=w, dx=dx)
    B.dd_linear_grad(dy, x=x, dw=dw)
    B.dd_linear_grad(dy, db=db)
    B.dd_linear_grad(dy)
    torch.cuda.synchronize()
    want = [(dy.double() @ w.double().t()), x.double().t() @ dy.double(), dy.double().sum(0)]
    assert all(torch.equal(a, b.to(torch.bfloat16)) for a, b in zip((dx, dw, db), want))
    turned = torch.empty(n, k, device="cuda", dtype=torch.bfloat16).t()
    both = x.clone()
    B.dd_linear_grad(dy, both, w, dx=both, dw=turned, db=db)
    torch.cuda.synchronize()
    assert torch.equal(turned, dw) and torch.equal(both, dx) and torch.equal(db, want[2].to(torch.bfloat16))


def test_one_row_for_all():
    """Rows of stride 0 (an expanded input)."""
    import torch
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(5)
    for k, n in ((64, 128), (65, 129)):
        row, w, residual = (torch.randint(-2, 3, s, generator=gen, device="cuda").to(torch.bfloat16) for s in ((1, k), (k, n), (1, n)))
        y = torch.empty(300, n, device="cuda", dtype=torch.bfloat16)
        B.dd_linear(row.expand(300, k), w, y, residual=residual.expand(300, n))
        torch.cuda.synchronize()
        assert torch.equal(y, (row.double() @ w.double() + residual.double()).to(torch.bfloat16).expand(300, n))


@pytest.mark.parametrize("odd", [0, 1])
def test_offsets_past_32_bits(odd):
    """Rows of x, and of y, that begin more than 2^32 elements apart from the first."""
    import torch
    require_gpu()
    rows, k, n, stride = 66000, 64 + odd, 72, 65600 + odd
    gen = torch.Generator("cuda").manual_seed(2)
    wide = torch.zeros(rows * stride, device="cuda", dtype=torch.bfloat16)
    x = wide.as_strided((rows, k), (stride, 1))
    y = wide.as_strided((rows, n), (stride, 1), 128)
    x.copy_(torch.randint(-2, 3, (rows, k), generator=gen, device="cuda"))
    w = torch.randint(-2, 3, (k, n), generator=gen, device="cuda").to(torch.bfloat16)
    B.dd_linear(x, w, y)
    dw = torch.empty_like(w)
    B.dd_linear_grad(y, x, w, dw=dw)
    torch.cuda.synchronize()
    want = x.double() @ w.double()
    assert torch.equal(y, want.to(torch.bfloat16))
    want = x.double().t() @ y.double()      # (sums of whole numbers, but too large to be exact in 32 bits)
    check("dw", dw, want, (rows + 8) * 2.0 ** -23 * (x.double().abs().t() @ y.double().abs()))
    assert not wide.as_strided((rows, 20), (stride, 1), 100).any() and not wide.as_strided((rows - 1, 1000), (stride, 1), 200).any()


def test_calls_of_many_sizes_share_given_memory():
    """One piece of working memory for calls of different shapes in a row on a stream."""
    import torch
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(6)
    shapes = [(4, 8192, 136), (300, 321, 131), (8192, 24, 40), (70, 5000, 90), (129, 127, 129)]
    work = torch.empty(max(max(B.dd_linear_work(*s), B.dd_linear_grad_work(*s)) for s in shapes), dtype=torch.uint8, device="cuda")
    kept = []
    for rows, k, n in shapes * 2:
        x, w, dy = (torch.randint(-2, 3, s, generator=gen, device="cuda").to(torch.float16) for s in ((rows, k), (k, n), (rows, n)))
        y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty(n, device="cuda")
        B.dd_linear(x, w, y, work=work)
        B.dd_linear_grad(dy, x, w, dx=dx, dw=dw, db=db, work=work)
        kept.append((x, w, dy, y, dx, dw, db))
    torch.cuda.synchronize()
    for x, w, dy, y, dx, dw, db in kept:
        assert torch.equal(y, (x.double() @ w.double()).half()) and torch.equal(dx, (dy.double() @ w.double().t()).half())
        assert torch.equal(dw, (x.double().t() @ dy.double()).half()) and torch.equal(db.double(), dy.double().sum(0))


def test_sums_of_more_columns_than_a_launch_has_threads_for():
    import torch
    require_gpu()
    n = (1 << 28) + 24
    dy = torch.ones(2, n, device="cuda", dtype=torch.bfloat16)
    dy[1, 5::7] = -3
    db = torch.empty(n, device="cuda", dtype=torch.bfloat16)
    B.dd_linear_grad(dy, w=torch.empty(1, n, device="cuda", dtype=torch.bfloat16), db=db)
    torch.cuda.synchronize()
    assert torch.equal(db, dy[0] + dy[1])


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("rows,k,n", [(4, 8192, 136), (300, 321, 131), (8192, 24, 40), (70, 5000, 90), (129, 127, 129), (1021, 777, 1237),
                                      (256, 1440, 1136), (2048, 136, 2048), (72, 3471, 1219)])
def test_nothing_behind_the_working_memory(rows, k, n, pad):
    """Exactly the bytes that are asked for, at the end of a buffer of which the rest stays as it was."""
    import torch
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(8)
    x, w, dy = (torch.randint(-2, 3, (a, b + pad), generator=gen, device="cuda").to(torch.bfloat16)[:, :b] for a, b in ((rows, k), (k, n), (rows, n)))
    y, dx, dw, db = torch.empty(rows, n, device="cuda", dtype=x.dtype), torch.empty(rows, k, device="cuda", dtype=x.dtype), torch.empty_like(w), torch.empty(n, device="cuda")
    for need, call in ((B.dd_linear_work(rows, k, n), lambda m: B.dd_linear(x, w, y, work=m)),
                       (B.dd_linear_grad_work(rows, k, n), lambda m: B.dd_linear_grad(dy, x, w, dx=dx, dw=dw, db=db, work=m))):
        room = torch.full((1024 + need + 4096,), 171, device="cuda", dtype=torch.uint8)
        call(room[1024:1024 + need])
        torch.cuda.synchronize()
        assert bool((room[:1024] == 171).all()) and bool((room[1024 + need:] == 171).all())
    assert torch.equal(y, (x.double() @ w.double()).to(torch.bfloat16)) and torch.equal(db.double(), dy.double().sum(0))
    assert torch.equal(dx, (dy.double() @ w.double().t()).to(torch.bfloat16)) and torch.equal(dw, (x.double().t() @ dy.double()).to(torch.bfloat16))
