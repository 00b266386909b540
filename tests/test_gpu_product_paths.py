"""Products and their gradients on every path that the plan has for them, in whole numbers, whose sums have
no rounding: the rounded truth, bit for bit."""
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


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
