"""Lists of tensors used on other streams than the one they were loaded on."""
import pytest

from paper_2006_03318_amd import binding as B
from tests.gpu_common import require_gpu
from tests.test_gpu_update import List

pytestmark = pytest.mark.gpu


def test_capture_on_another_stream():
    """Clipping is captured on any stream; the calls with working memory are
    refused there, and the capture goes on."""
    import torch
    require_gpu()
    g = torch.randn(100_000, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    out = torch.empty_like(g)
    src, dst = List([dict(grad=g)]), List([dict(grad=out)])
    stats = torch.empty(3, device="cuda")
    B.dd_grad_norm(src.h, stats, max_norm=1.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(B.DDError) as e:
            B.dd_grad_norm(src.h, stats, max_norm=1.0, stream=side)
        assert e.value.code == B.DD_EINVAL
        B.dd_grad_clip(src.h, dst.h, stats, stream=side)
    for k in range(4):
        g.mul_(1.5)
        B.dd_grad_norm(src.h, stats, max_norm=1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, g * stats[1]), k
    del graph, src, dst
    torch.cuda.synchronize()


def test_the_default_stream_as_the_other():
    import torch
    require_gpu()
    side = torch.cuda.Stream()
    g = torch.ones(1 << 20, device="cuda")
    w, m, v = (torch.zeros_like(g) for _ in range(3))
    torch.cuda.synchronize()
    li = List([dict(grad=g, param=w, m=m, v=v)], side)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    stats = [torch.empty(3, device="cuda") for _ in range(6)]
    torch.cuda.synchronize()
    for k in range(6):
        s = None if k % 2 else side
        B.dd_grad_norm(li.h, stats[k], max_norm=4.0, stream=s)
        B.dd_adam_step(li.h, step, stats[k], lr=0.5, stream=s)
    torch.cuda.synchronize()
    assert int(step) == 6 and all(s.tolist() == [1024.0, 4.0 / 1024, 0.0] for s in stats)
    assert bool((w == w[0]).all()) and abs(float(w[0]) + 3.0) <= 1e-4
