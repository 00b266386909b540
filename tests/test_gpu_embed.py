"""dd_embed and dd_embed_grad against the formulas in 64 bits.

Tolerances: a row of the table times the scale is one product of 32 bits and the stored value's half
step; a sum of c rows is off by (c + 2) steps of 2^-24 of the sum of their magnitudes at most."""
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu
KINDS = ("float32", "bfloat16", "float16")


def _bound(got, want, slack):
    import torch
    f = torch.finfo(got.dtype)
    rel, least = f.eps / 2, f.smallest_normal * f.eps / 2
    return bool(((got.double() - want).abs() <= rel * want.abs() * (1 + rel) + least + slack * (1 + rel)).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("id_kind", ["int64", "int32"])
@pytest.mark.parametrize("tokens,vocab,cols,pad", [(1, 1, 1, 0), (4, 100, 2048, 0), (77, 5, 7, 3), (300, 1000, 129, 7), (2000, 50, 16, 0), (40001, 50, 250, 0), (5001, 70, 1700, 3)])
def test_lookup(tokens, vocab, cols, pad, kind, id_kind):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(tokens)
    table = torch.full((vocab, cols + pad), float("nan"), device="cuda", dtype=t)[:, :cols]
    table.copy_(torch.randn(vocab, cols, generator=gen, device="cuda"))
    ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda").to(getattr(torch, id_kind))
    wide = torch.full((tokens, cols + pad), 7.0, device="cuda", dtype=t)
    B.dd_embed(ids, table, wide[:, :cols], scale=1.7)
    torch.cuda.synchronize()
    want = table.double()[ids.long()] * 1.7
    assert _bound(wide[:, :cols], want, 2 * 2.0 ** -24 * want.abs())        # (the scale and the product, in 32 bits)
    assert bool((wide[:, cols:] == 7.0).all())


def test_ids_that_the_table_does_not_have():
    import torch
    require_gpu()
    table = torch.ones(10, 24, device="cuda")
    ids = torch.tensor([[0, -1, 9], [10, 1 << 40, -(1 << 40)]], device="cuda")
    out = torch.empty(2, 3, 24, device="cuda")
    B.dd_embed(ids, table, out)
    torch.cuda.synchronize()
    bad = torch.tensor([[False, True, False], [True, True, True]], device="cuda")
    assert bool(out[bad].isnan().all()) and bool((out[~bad] == 1).all())
    dtable = torch.full((10, 24), 7.0, device="cuda")
    B.dd_embed_grad(ids, torch.ones(2, 3, 24, device="cuda"), dtable)
    torch.cuda.synchronize()
    assert dtable[:, 0].tolist() == [1.0] + [0.0] * 8 + [1.0]


def _ids(gen, how, tokens, vocab):
    import torch
    u = torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64)
    if how == "one":
        return torch.full((tokens,), vocab // 2, device="cuda")
    if how == "few":
        return (u * u * u * vocab).long()
    if how == "last":
        return torch.where(u < 0.5, vocab - 1, (u * vocab).long())
    return (u * vocab).long()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("how", ["even", "few", "one", "last"])
@pytest.mark.parametrize("tokens,vocab,cols,pad", [
    (1, 1, 1, 0), (1, 70000, 16, 0), (31, 7, 8, 0), (32, 300, 100, 3), (33, 2, 129, 0), (64, 64, 640, 8), (65, 1000, 128, 0),
    (2047, 256, 24, 0), (2049, 257, 513, 0), (5000, 40, 72, 5), (9000, 66000, 40, 0), (30000, 300, 520, 0), (4097, 1 << 24, 1, 0), (8192, 3000, 24, 0), (8193, 3000, 24, 0), (1100000, 5000, 8, 0), (1048577, 70001, 2, 0),
    (15, 4, 130, 0), (16, 9, 128, 0), (17, 9, 257, 3), (129, 3, 140, 0), (8192, 600, 512, 0), (8192, 600, 513, 0), (4100, 30, 1100, 1), (300, 5, 8200, 0)])
def test_gradient(tokens, vocab, cols, pad, how, kind):
    """Whole numbers: sums without rounding, so every row is the rounded truth bit for bit."""
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(tokens + vocab)
    ids = _ids(gen, how, tokens, vocab)
    dy = torch.full((tokens, cols + pad), float("nan"), device="cuda", dtype=t)[:, :cols]
    dy.copy_(torch.randint(-3, 4, (tokens, cols), generator=gen, device="cuda"))
    wide = torch.full((vocab, cols + pad), 7.0, device="cuda", dtype=t)
    B.dd_embed_grad(ids, dy, wide[:, :cols], scale=2.0)
    torch.cuda.synchronize()
    # (on the host: a million additions to one row take the GPU's 64-bit atomics many seconds)
    want = torch.zeros(vocab, cols, dtype=torch.float64).index_add_(0, ids.cpu(), 2.0 * dy.cpu().double())
    assert torch.equal(wide[:, :cols].cpu(), want.to(t))
    assert bool((wide[:, cols:] == 7.0).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens,vocab,cols", [(500, 20, 200), (20000, 3000, 96), (70000, 11, 40)])
def test_gradient_of_real_numbers(tokens, vocab, cols, kind):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(vocab)
    ids = _ids(gen, "few", tokens, vocab)
    dy = (torch.randn(tokens, cols, generator=gen, device="cuda") * 0.1).to(t)
    got = []
    for i in range(3):
        out = torch.full((vocab, cols), float(i), device="cuda", dtype=t)
        work = torch.full((B.dd_embed_grad_work(tokens, vocab, cols),), 255, dtype=torch.uint8, device="cuda") if i else None
        B.dd_embed_grad(ids.int() if i == 2 else ids, dy, out, scale=1.5, work=work)
        torch.cuda.synchronize()
        got.append(out)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    zero = torch.zeros(vocab, cols, dtype=torch.float64, device="cuda")
    want, size = zero.index_add(0, ids, dy.double()) * 1.5, zero.index_add(0, ids, dy.double().abs()) * 1.5
    count = torch.bincount(ids, minlength=vocab)[:, None]
    assert _bound(got[0], want, (count + 2) * 2.0 ** -24 * size)


def test_pad_and_no_tokens():
    import torch
    require_gpu()
    ids = torch.tensor([3, 0, 3, 5, -1, 99], device="cuda")
    dy = torch.ones(6, 40, device="cuda", dtype=torch.float16)
    dy[4:] = float("nan")
    out = torch.full((6, 40), 7.0, device="cuda", dtype=torch.float16)
    B.dd_embed_grad(ids, dy, out, pad=3)
    torch.cuda.synchronize()
    assert out[:, 0].tolist() == [1, 0, 0, 0, 0, 1]
    all_pad = torch.full((5000,), 2, device="cuda")
    B.dd_embed_grad(all_pad, torch.full((5000, 40), float("nan"), device="cuda", dtype=torch.float16), out, pad=2)
    torch.cuda.synchronize()
    assert not out.any()
    out.fill_(7.0)
    B.dd_embed_grad(ids[:0], dy[:0], out)
    B.dd_embed(ids[:0], out, dy[:0])
    torch.cuda.synchronize()
    assert not out.any()


def test_values_that_are_not_finite_stay_in_their_row():
    import torch
    require_gpu()
    ids = (torch.arange(4000, device="cuda") * 7) % 100
    dy = torch.ones(4000, 72, device="cuda")
    dy[5, 6], dy[2001, 70] = float("nan"), float("inf")
    out = torch.empty(100, 72, device="cuda")
    B.dd_embed_grad(ids, dy, out)
    torch.cuda.synchronize()
    want = torch.full((100, 72), 40.0, device="cuda")
    a, b = int(ids[5]), int(ids[2001])
    assert bool(out[a, 6].isnan()) and bool(out[b, 70].isinf())
    out[a, 6] = out[b, 70] = 40.0
    assert torch.equal(out, want)


def test_offsets_past_32_bits():
    """A table and a gradient of more than 2^32 elements: the last rows."""
    import torch
    require_gpu()
    vocab, cols = (1 << 21) + 3, 2056
    table = torch.zeros(vocab, cols, device="cuda", dtype=torch.bfloat16)
    table[-1], table[-2] = 3.0, 5.0
    ids = torch.tensor([vocab - 1, 0, vocab - 2, vocab - 1], device="cuda")
    out = torch.empty(4, cols, device="cuda", dtype=torch.bfloat16)
    B.dd_embed(ids, table, out)
    torch.cuda.synchronize()
    assert out[:, 17].tolist() == [3, 0, 5, 3]
    table.fill_(7.0)
    B.dd_embed_grad(ids, out, table)
    torch.cuda.synchronize()
    assert bool((table[-1] == 6).all()) and bool((table[-2] == 5).all()) and not table[:-2].any()


@pytest.mark.parametrize("tokens,vocab,cols", [(9, 300, 40), (3000, 40, 136), (8192, 600, 24), (20000, 300, 513), (1100000, 70000, 8)])
def test_nothing_behind_the_working_memory(tokens, vocab, cols):
    """Exactly the bytes that are asked for, at the end of a buffer of which the rest stays as it was."""
    import torch
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(3)
    ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    dy = torch.ones(tokens, cols, device="cuda")
    out = torch.empty(vocab, cols, device="cuda")
    need = B.dd_embed_grad_work(tokens, vocab, cols)
    room = torch.full((1024 + need + 4096,), 171, device="cuda", dtype=torch.uint8)
    B.dd_embed_grad(ids, dy, out, work=room[1024:1024 + need])
    torch.cuda.synchronize()
    assert bool((room[:1024] == 171).all()) and bool((room[1024 + need:] == 171).all())
    assert torch.equal(out, torch.bincount(ids, minlength=vocab).float()[:, None].expand(vocab, cols))


@pytest.mark.parametrize("kind", KINDS)
def test_many_ids_that_the_table_does_not_have(kind):
    import torch
    require_gpu()
    t = getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(9)
    table = torch.randint(-3, 4, (1000, 520), generator=gen, device="cuda").to(t)
    ids = torch.randint(-200, 1200, (20003,), generator=gen, device="cuda")
    out = torch.empty(20003, 520, device="cuda", dtype=t)
    B.dd_embed(ids, table, out, scale=2.0)
    torch.cuda.synchronize()
    bad = (ids < 0) | (ids >= 1000)
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], 2 * table[ids[~bad]])
