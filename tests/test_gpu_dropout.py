"""dd_dropout: the generator's numbers, the mask, and what is made of it.

The generator's words are checked against numbers published with it; values are compared with
the formula in 64 bits: x times a factor of 32 bits (half a step of 2^-24), a product and a sum
of 32 bits, and the stored value's half step."""
import numpy as np
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


def words(block, counter, key):
    """Philox 4x32-10, in Python's whole numbers."""
    low = 0xffffffff
    c = [block & low, block >> 32, counter & low, counter >> 32]
    k = [key & low, key >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & low, a >> 32 ^ c[3] ^ k[1], a & low]
        k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
    return c


def kept(n, p, key, counter):
    """Which of n elements stay."""
    gone = round(p * 65536)
    halves = []
    for block in range(-(-n // 8)):
        for w in words(block, counter & (1 << 64) - 1, key & (1 << 64) - 1):
            halves += [w & 0xffff, w >> 16]
    return np.array(halves[:n]) >= gone, gone


def state_of(key, counter):
    import torch
    wrap = lambda v: (v + (1 << 63)) % (1 << 64) - (1 << 63)  # noqa: E731
    return torch.tensor([wrap(key), wrap(counter)], dtype=torch.int64, device="cuda")


def test_published_numbers():
    """The known answers for a counter and a key of zeros, and of ones."""
    assert words(0, 0, 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = (1 << 64) - 1
    assert words(ones, ones, ones) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 7, 0), (1, 8, 0), (5, 3, 0), (5, 3, 2), (33, 64, 0), (33, 64, 8), (21, 37, 0), (21, 37, 1), (700, 1, 3)])
@pytest.mark.parametrize("p,with_residual", [(0.1, True), (0.5, False), (0.0, True), (1.0, True), (1.0, False), (0.99999, False)])
def test_values(rows, cols, pad, kind, p, with_residual):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(rows * cols)
    key, counter, call = 0x123456789abcdef0 + rows, (1 << 64) - 2, cols
    nan = float("nan")

    def wide(fill):
        w = torch.full((rows, cols + pad), fill, device="cuda", dtype=t)
        return w, w[:, :cols]

    (_, x), (_, r), (all_out, out) = wide(nan), wide(nan), wide(7.0)
    x.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
    r.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
    used = torch.zeros(2, dtype=torch.int64, device="cuda")
    B.dd_dropout(x, r if with_residual else None, p, state_of(key, counter), out, call=call, used=used)
    torch.cuda.synchronize()
    stay, gone = kept(rows * cols, p, key, counter + call)
    assert torch.equal(used, state_of(key, counter + call))
    stay = torch.from_numpy(stay).view(rows, cols).cuda()
    factor = 65536 / (65536 - gone) if gone < 65536 else 0.0
    want = torch.where(stay, x.double() * factor, 0.0) + (r.double() if with_residual else 0.0)
    rel, least = torch.finfo(t).eps / 2, torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2
    slack = 3 * 2.0 ** -24 * (x.double().abs() * factor + (r.double().abs() if with_residual else 0.0))
    assert bool(((out.double() - want).abs() <= rel * want.abs() * (1 + rel) + least + slack * (1 + rel)).all())
    if not with_residual:
        assert torch.equal(out != 0, stay & (x != 0))
    if pad:
        assert bool((all_out[:, cols:] == 7.0).all())
    # the gradient's call on what was used: the same mask, strides or not
    dy = torch.ones(rows, cols, device="cuda", dtype=t)
    dx, (_, apart) = torch.empty_like(dy), wide(0.0)
    B.dd_dropout(dy, None, p, used, dx)
    B.dd_dropout(dy, None, p, used, apart)
    torch.cuda.synchronize()
    assert torch.equal(dx != 0, stay) and torch.equal(apart, dx)
    # in place
    B.dd_dropout(x, r if with_residual else None, p, used, x)
    torch.cuda.synchronize()
    assert torch.equal(x, out)


def test_dropped_values_count_for_nothing():
    import torch
    require_gpu()
    for p in (0.25, 1.0):
        stay, _ = kept(512, p, 5, 6)
        x = torch.where(torch.from_numpy(stay).cuda(), 1.0, float("nan"))
        x[::3] = torch.where(torch.from_numpy(stay).cuda(), 1.0, float("inf"))[::3]
        out = torch.empty_like(x)
        B.dd_dropout(x, None, p, state_of(5, 6), out)
        torch.cuda.synchronize()
        assert bool(out.isfinite().all())


def test_rows_beyond_a_launch_and_the_share_that_stays():
    """More elements than one round of workgroups has; of 2^28 the share kept is within six standard
    deviations; a second call's mask is another."""
    import torch
    require_gpu()
    n = (1 << 28) + 5
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    out, other = torch.empty_like(x), torch.empty_like(x)
    state = state_of(99, 0)
    B.dd_dropout(x, None, 0.25, state, out)
    B.dd_dropout(x, None, 0.25, state, other, call=1)
    torch.cuda.synchronize()
    share = float((out != 0).sum()) / n
    assert abs(share - 0.75) < 6 * (0.75 * 0.25 / n) ** 0.5
    both = float(((out != 0) & (other != 0)).sum()) / n
    assert abs(both - 0.5625) < 6 * (0.5625 * 0.4375 / n) ** 0.5
    for block in ((1 << 25), (1 << 25) - 1, (1 << 24) + 3):         # past one round of the grid
        halves = [h for w in words(block, 0, 99) for h in (w & 0xffff, w >> 16)]
        at = out[8 * block:8 * block + 8]
        assert [bool(v) for v in at != 0] == [h >= 16384 for h in halves][:len(at)]


def test_one_row_for_all_as_residual_and_no_rows():
    import torch
    require_gpu()
    x, r = torch.ones(40, 24, device="cuda"), torch.arange(24.0, device="cuda")
    out = torch.empty_like(x)
    used = torch.zeros(2, dtype=torch.int64, device="cuda")
    B.dd_dropout(x, r.expand(40, 24), 1.0, state_of(1, 2), out)
    B.dd_dropout(x[:0], None, 0.5, state_of(1, 2), out[:0], call=3, used=used)
    torch.cuda.synchronize()
    assert torch.equal(out, r.expand(40, 24)) and used.tolist() == [1, 5]
