"""The functions for torch programs in captured graphs."""
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(700, 264), (3000, 1024), (20, 17_000)])
def test_norm_and_gradient(rows, cols):
    """Replayed with gradients of other rows on the capture's stream and an
    emptied cache between: every replay gives what the eager call gives."""
    import torch
    from paper_2006_03318_amd.training import add_rms_norm
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(rows)

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)

    x, r, w = (rand(rows, cols).requires_grad_(), rand(rows, cols).requires_grad_(), rand(cols).requires_grad_())
    dy, dh = rand(rows, cols), rand(rows, cols)
    other = rand(rows, cols).requires_grad_()

    def both(x):
        y, h = add_rms_norm(x, r, w)
        return (y, h) + torch.autograd.grad((y, h), (x, r, w), (dy, dh))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = both(x)
    for k in range(4):
        with torch.no_grad():
            x.mul_(1.25)
            dy.mul_(0.75)
        want = both(x)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):                  # while the graph runs on the current stream
            both(other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        B.dd_release_cache()


def test_gradient_without_working_memory_is_not_captured():
    import torch
    require_gpu()
    rows, cols = 5000, 64
    dy, h, dx = (torch.ones(rows, cols, device="cuda") for _ in range(3))
    rstd, dw = torch.ones(rows, device="cuda"), torch.empty(cols, device="cuda")
    work = torch.empty(B.dd_rms_norm_grad_work(rows, cols), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    B.dd_rms_norm_grad(dy, h, None, rstd, dx, dw, stream=side)       # the cache has a block for the stream
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(B.DDError) as e:
            B.dd_rms_norm_grad(dy, h, None, rstd, dx, dw, stream=side)
        assert e.value.code == B.DD_EINVAL and "work" in str(e.value)
        B.dd_rms_norm_grad(dy, h, None, rstd, dx, stream=side)       # without dw there is nothing to keep
        B.dd_rms_norm_grad(dy, h, None, rstd, dx, dw, work=work, stream=side)
    dw.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert bool((dw == float(rows)).all())


@pytest.mark.parametrize("kind", ["bfloat16", "float32"])
def test_training_step(kind):
    """Gradients, norm and update of an optimizer that was made on the capture's
    stream; the same steps taken eagerly."""
    import torch
    from paper_2006_03318_amd.training import Adam, add_rms_norm
    require_gpu()
    gen = torch.Generator("cuda").manual_seed(5)
    t = getattr(torch, kind)
    x = torch.randn(300, 520, generator=gen, device="cuda").to(t)
    dy = torch.randn(300, 520, generator=gen, device="cuda").to(t)
    start = (1 + 0.1 * torch.randn(520, generator=gen, device="cuda")).to(t)

    def make():
        w = torch.nn.Parameter(start.clone())
        return w, Adam([w], lr=0.01, weight_decay=0.1, max_norm=1.0)

    def step(w, opt):
        opt.zero_grad()
        add_rms_norm(x, None, w).backward(dy)
        opt.step()

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        w, opt = make()
        step(w, opt)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(w, opt)
    w2, opt2 = make()
    step(w2, opt2)
    for k in range(4):
        x.mul_(-1.25)
        step(w2, opt2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, w2) and torch.equal(opt.stats, opt2.stats) and int(opt.steps) == int(opt2.steps) == k + 2
        assert all(torch.equal(a, b) for a, b in zip(opt.masters + opt.m + opt.v, opt2.masters + opt2.m + opt2.v))
    del graph
    opt.close()
    opt2.close()
