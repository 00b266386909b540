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
        monkeypatch.setattr(training.B, "dd_tensors_load", lambda tensors, stream=None: list(tensors))
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
