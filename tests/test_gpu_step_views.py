"""Tensors whose values are not what their memory holds (torch's lazily negated views, and zeros without memory), and rows millions of values
apart."""
import pytest
import torch

from paper_2605_04478_amd import step
from tests.test_step_calls import _arguments

BF = torch.bfloat16
DEV = "cuda:0"


def _negated(t):
    """The same values in a tensor whose memory holds the opposite ones."""
    return torch._neg_view(t.neg())


def _negated_imag(t):
    """The same for 32-bit vectors, as automatic differentiation makes them: every other value of complex numbers."""
    return torch.complex(torch.zeros_like(t), t.neg()).conj().imag


@pytest.mark.parametrize("shape", [(4,), (4, 6), (3, 4, 6), (1,)])
def test_layouts_are_of_plain_tensors(shape):
    t = torch.randn(shape)
    for form in (_negated, _negated_imag):
        for out in (step._rows(form(t)), step._vector(form(t)), step._plain(form(t))):
            assert not out.is_neg() and torch.equal(out, t)
    zero = torch._efficientzerotensor(shape)
    for out in (step._rows(zero), step._vector(zero), step._plain(zero)):
        assert out.data_ptr() and not out.any()
    assert step._plain(t) is t and step._rows(t) is t and step._vector(t).data_ptr() == t.data_ptr()
    spaced = torch.stack([t, t], -1)[..., 0]
    assert step._plain(spaced) is spaced and step._vector(spaced).is_contiguous()


def _with_values(device, name):
    """Arguments of a call whose values differ everywhere."""
    g = torch.Generator().manual_seed(4)
    args = [(torch.randn(a.shape, generator=g).to(a.dtype) if a.is_floating_point() else a.cpu()).to(device) if isinstance(a, torch.Tensor) else a
            for a in _arguments("cpu")[name]]
    if name.startswith("vocab_loss"):
        args[1 + name.endswith("grad") + 1] = torch.tensor([0, 9, -1, 3, 3, 5], device=device)
    return args


def _results(name, args):
    out = getattr(step, name)(*args)
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(_arguments("cpu")))
def test_negated_tensors_count_with_their_values(name):
    args = _with_values(DEV, name)
    want = _results(name, args)
    for i, t in enumerate(args):
        if not isinstance(t, torch.Tensor):
            continue
        forms = [_negated(t)] + ([_negated_imag(t)] if t.dtype == torch.float32 else [])
        for other in forms:
            assert other.is_neg() and torch.equal(other, t)
            assert getattr(step._native(), name)(*args[:i], other, *args[i + 1:]) is None
            got = _results(name, [*args[:i], other, *args[i + 1:]])
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (name, i)


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(_arguments("cpu")))
def test_zeros_without_memory_count_as_zeros(name):
    args = _with_values(DEV, name)
    for i, t in enumerate(args):
        if not isinstance(t, torch.Tensor):
            continue
        want = _results(name, [*args[:i], torch.zeros_like(t), *args[i + 1:]])
        zero = torch._efficientzerotensor(t.shape, dtype=t.dtype, device=DEV)
        assert getattr(step._native(), name)(*args[:i], zero, *args[i + 1:]) is None
        got = _results(name, [*args[:i], zero, *args[i + 1:]])
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want)), (name, i)


@pytest.mark.gpu
def test_a_loss_that_became_complex():
    """The backward pass of a conjugate hands the loss a gradient with torch's negative bit."""
    h, w, labels = (t for t in _with_values(DEV, "vocab_loss"))
    grads = []
    for through_complex in (False, True):
        leaves = [h.clone().requires_grad_(), w.clone().requires_grad_()]
        loss = step.VocabLoss.apply(*leaves, labels)
        if through_complex:
            loss = (torch.complex(torch.zeros_like(loss), loss).conj() * torch.tensor([1j], device=DEV)).real
        loss.sum().backward()
        grads.append([t.grad for t in leaves])
    assert all(torch.equal(a, b) and a.any() for a, b in zip(*grads))


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(_arguments("cpu")))
def test_rows_that_are_far_apart(name):
    args = _with_values(DEV, name)
    want = _results(name, args)
    for i, t in enumerate(args):
        if not isinstance(t, torch.Tensor) or t.dim() < 2:
            continue
        for apart in (step.MAX_LD - 8, step.MAX_LD, 5_000_008):
            wide = torch.empty(*t.shape[:-1], apart, dtype=t.dtype, device=DEV)[..., :t.shape[-1]]
            wide.copy_(t)
            got = _results(name, [*args[:i], wide, *args[i + 1:]])
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (name, i, apart)
