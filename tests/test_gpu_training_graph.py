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
