"""What the differentiable layers for torch programs hand to the library, with the calls themselves
replaced: on the CPU."""
import contextlib

import pytest
import torch

from paper_2006_03318_amd import training


@pytest.fixture
def calls(monkeypatch):
    """The arguments by name of every call of the library, which do nothing."""
    made = []
    for name in ("dd_linear", "dd_linear_grad", "dd_act_grad"):
        monkeypatch.setattr(training.B, name, lambda *args, _name=name, **kw: made.append((_name, args, kw)))
    monkeypatch.setattr(training, "_stream", lambda: 0)
    return made


def leaves(wanted, *shapes):
    return [torch.ones(s, dtype=torch.bfloat16, requires_grad=i in wanted) for i, s in enumerate(shapes)]


def kept(calls):
    """Whether each forward product was told to keep what its activation takes."""
    return [kw["z"] is not None for name, _, kw in calls if name == "dd_linear"]


@pytest.mark.parametrize("mode", [torch.enable_grad, torch.no_grad, torch.inference_mode])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_nothing_is_kept_without_gradients(calls, act, mode):
    """Weights that require a gradient, where gradients are off: nothing will ask for it."""
    x, w, b, v = leaves({1, 2, 3}, (5, 8), (8, 16), (16,), (16, 8))
    with mode():
        y = training.linear(x, w, b, act)
        z = training.mlp(x, w, v, b, act=act)
    on = mode is torch.enable_grad
    assert kept(calls) == [on and act != "none", on and act != "none", False]
    assert y.requires_grad == z.requires_grad == on


@pytest.mark.parametrize("wanted", [{0}, {1}, {2}, {3}, {4}, {5}, {1, 2}, set()])
def test_mlp_keeps_what_its_gradients_read(calls, wanted):
    """The activation's argument is read for the gradients of what comes before it alone; those asked for
    all come."""
    x, up, down, bu, bd, r = ins = leaves(wanted, (5, 8), (8, 16), (16, 8), (16,), (8,), (5, 8))
    y = training.mlp(x, up, down, bu, bd, "silu", r)
    assert kept(calls) == [bool(wanted & {0, 1, 3}), False]
    if wanted:
        y.backward(torch.ones_like(y))
    assert [t.grad is not None for t in ins] == [i in wanted for i in range(6)]
    second = [kw for name, _, kw in calls if name == "dd_linear_grad" and kw["in_act"] == "silu"]
    assert all((kw["dx"] is None) or kw["in_z"] is not None for kw in second)


@pytest.mark.parametrize("wanted", [{0}, {1}, {2}, {3}, set()])
def test_linear_keeps_what_its_gradients_read(calls, wanted):
    x, w, b, r = ins = leaves(wanted, (5, 8), (8, 16), (16,), (5, 16))
    y = training.linear(x, w, b, "gelu", r)
    assert kept(calls) == [bool(wanted & {0, 1, 2})]
    if wanted:
        y.backward(torch.ones_like(y))
    assert [t.grad is not None for t in ins] == [i in wanted for i in range(4)]


@pytest.mark.parametrize("reentrant", [True, False])
def test_checkpointed_passes(calls, reentrant):
    """A forward pass that is run again for its gradient: the first of a reentrant one keeps nothing."""
    from torch.utils.checkpoint import checkpoint
    x, w, b = leaves({0, 1, 2}, (5, 8), (8, 16), (16,))
    with contextlib.ExitStack() as s:
        s.enter_context(torch.autograd.set_multithreading_enabled(False))
        checkpoint(lambda t: training.linear(t, w, b, "gelu"), x, use_reentrant=reentrant, preserve_rng_state=False).sum().backward()
    assert kept(calls) == [not reentrant, True]
    assert x.grad is not None and w.grad is not None and b.grad is not None
