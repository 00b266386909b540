"""What the functions for torch programs hand to the library, with the calls
themselves replaced: on the CPU."""
import pytest
import torch

from paper_2006_03318_amd import training


class Calls:
    """Records the library's calls, and does nothing in them."""

    def __init__(self, monkeypatch):
        self.made = []
        for name in ("dd_rms_norm", "dd_rms_norm_grad", "dd_grad_norm", "dd_adam_step", "dd_tensors_free"):
            monkeypatch.setattr(training.B, name, self._recorder(name))
        monkeypatch.setattr(training.B, "dd_tensors_load", lambda tensors, stream=None: None)
        monkeypatch.setattr(training, "_stream", lambda: 0)

    def _recorder(self, name):
        def call(*args, **kw):
            self.made.append((name, args, kw))
        return call

    def last(self, name):
        return [c for c in self.made if c[0] == name][-1][1:]


@pytest.fixture
def calls(monkeypatch):
    return Calls(monkeypatch)


@pytest.mark.parametrize("shape", [(5, 64), (3, 700, 32), (40,)])
def test_gradient_brings_its_working_memory(calls, shape):
    """From torch's allocator, which knows graphs: a block of the library's own
    cache would go back to it while a graph still writes there."""
    x = torch.ones(shape, requires_grad=True)
    w = torch.ones(shape[-1], requires_grad=True)
    training.add_rms_norm(x, None, w).sum().backward()
    args, kw = calls.last("dd_rms_norm_grad")
    need = training.B.dd_rms_norm_grad_work(x.numel() // shape[-1], shape[-1])
    assert kw["work"].numel() * kw["work"].element_size() >= need > 0
    x = torch.ones(shape, requires_grad=True)
    training.add_rms_norm(x, None, None).sum().backward()         # no gradient of a weight: none needed
    assert calls.last("dd_rms_norm_grad")[1].get("work") is None


def _params(kind, *sizes):
    gen = torch.Generator().manual_seed(1)
    return [torch.nn.Parameter(torch.randn(n, generator=gen).to(kind)) for n in sizes]


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
def test_weights_written_between_steps_reach_the_masters(calls, kind):
    """Whatever writes them: only the elements that were written lose the bits
    that a master has beside its weight."""
    model = torch.nn.Module()
    model.a, model.b, model.c = _params(kind, 40, 30, 20)
    opt = training.Adam(model.parameters())
    for w in opt.masters:
        w.mul_(1 + 2.0 ** -13)                  # as steps leave them: bits beside the rounding
    with torch.no_grad():
        for p, w in zip(opt.params, opt.masters):
            p.copy_(w)
    opt.step()
    fine = [w.clone() for w in opt.masters]
    state = {k: v.clone() for k, v in model.state_dict().items()}
    state["a"][3:7] += 1.0
    model.load_state_dict(state)
    with torch.no_grad():
        model.c.mul_(2.0)
    opt.step()
    assert torch.equal(opt.masters[0][3:7], model.a[3:7].float())
    assert torch.equal(opt.masters[0][7:], fine[0][7:]) and torch.equal(opt.masters[0][:3], fine[0][:3])
    assert torch.equal(opt.masters[1], fine[1])
    assert torch.equal(opt.masters[2], model.c.float())
    model.b.data.copy_(torch.full((30,), 5.0))  # behind torch's back: said, not seen
    opt.read_weights()
    assert torch.equal(opt.masters[1], torch.full((30,), 5.0)) and torch.equal(opt.masters[2], model.c.float())


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_a_step_counts_as_a_write(calls, kind):
    """A backward pass through a graph kept from before the step is refused, as
    with any other optimizer: its weights are gone."""
    p, = _params(kind, 40)
    opt = training.Adam([p])
    x = torch.ones(40, dtype=kind, requires_grad=True)
    loss = (p * x).sum()
    loss.backward(retain_graph=True)
    loss.backward(retain_graph=True)
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    fine = opt.masters[0].clone()
    (p * x).sum().backward()
    opt.step()                                  # its own writes are no one else's
    assert torch.equal(opt.masters[0], fine)


def test_a_parameter_given_twice_is_refused(calls):
    """Two tensors of the list would update it, one from a gradient that no one
    writes."""
    a, b = _params(torch.float32, 40, 30)
    with pytest.raises(ValueError, match="twice"):
        training.Adam([a, b, a])
    assert a.grad is None and b.grad is None
    training.Adam([a, b])


def test_gradients_that_are_there_stay(calls):
    """The optimizer's buffers take over gradients from before it was made."""
    a, b, c = _params(torch.bfloat16, 40, 30, 20)
    ((a * 3).sum() + (b[:4] * 2).sum()).backward()
    want = [a.grad.clone(), b.grad.clone()]
    opt = training.Adam([a, b, c])
    assert torch.equal(a.grad, want[0]) and torch.equal(b.grad, want[1]) and not bool(c.grad.any())
    (a * 1).sum().backward()                            # and add to them
    assert torch.equal(a.grad, want[0] + 1)
    opt.zero_grad()
    assert not any(bool(p.grad.any()) for p in opt.params)


def test_calls_are_made_on_the_tensors_device(calls, monkeypatch):
    """The library works on the current device: it is the tensors' own while a
    call is made, whatever it is outside."""
    import contextlib
    where = []

    @contextlib.contextmanager
    def on(*tensors):
        where.append([t for t in tensors if t is not None])
        calls.made.append(("enter", (), {}))
        yield
        calls.made.append(("leave", (), {}))

    monkeypatch.setattr(training, "_on", on)
    x, w = torch.ones(4, 8, requires_grad=True), torch.ones(8, requires_grad=True)
    y, h = training.add_rms_norm(x, x.detach(), w)
    (y.sum() + h.sum()).backward()
    opt = training.Adam([w])
    opt.step(inv_scale=torch.ones(1))
    for name in ("dd_rms_norm", "dd_rms_norm_grad", "dd_grad_norm", "dd_adam_step"):
        names = [c[0] for c in calls.made]
        before = names[:names.index(name)]
        assert before.count("enter") == before.count("leave") + 1, name
    assert [len(t) for t in where] == [3, 4, 1, 2]


def test_tensors_of_several_devices_are_refused(monkeypatch):
    class On:
        is_cuda = True

        def __init__(self, device):
            self.device = torch.device(device)

    assert training._on(On("cuda:1"), None, On("cuda:1")).idx == 1
    with pytest.raises(ValueError, match="cuda:1 and cuda:2"):
        training._on(On("cuda:1"), None, On("cuda:2"))
    monkeypatch.setattr(training, "_stream", lambda: 0)
    with pytest.raises(ValueError, match="GPU"):                  # as the library says it
        training.add_rms_norm(torch.ones(4, 8))


def test_an_optimizer_that_lives_to_the_end_of_the_program():
    """Its handle is freed without a word when the interpreter takes the modules
    apart."""
    import os
    import subprocess
    import sys
    code = ("import torch\n"
            "from paper_2006_03318_amd import training\n"
            "training.B.dd_tensors_load = lambda tensors, stream=None: 7\n"
            "training.B.dd_tensors_free = lambda handle: None\n"
            "training._stream = lambda: 0\n"
            "opt = training.Adam([torch.nn.Parameter(torch.zeros(4))])\n"
            "step = opt.step\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "Exception" not in r.stderr, r.stderr
