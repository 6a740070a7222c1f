"""The calls in native code take tensors that are as they should be and leave all others, and every wrong argument, to Python."""
import pytest
import torch

from paper_2605_04478_amd import step

BF = torch.bfloat16
DEV = "cuda:0"


def _arguments(device, rows=6):
    z = lambda *shape, dtype=BF: torch.zeros(shape, dtype=dtype, device=device)
    x, w, offsets = z(rows, 8), z(2, 16, 8), torch.tensor([0, 2, rows], dtype=torch.int32, device=device)
    h, v, labels, f = z(rows, 8), z(10, 8), z(rows, dtype=torch.int64), z(rows, dtype=torch.float32)
    g, p = z(3, 8), z(8)
    return {"expert_product": [x, w, offsets], "expert_product_grad": [z(rows, 16), x, w, offsets, True, True],
            "vocab_loss": [h, v, labels], "vocab_loss_grad": [f, h, v, labels, f, True, True],
            "norm_residual": [h, h, g, p, p, 1.0, 1e-6], "norm_residual_grad": [h, h, h, h, g, p, p, f, f, 1.0]}


@pytest.mark.parametrize("name", list(_arguments("cpu")))
def test_declines_without_a_gpu(name):
    call, args = getattr(step._native(), name), _arguments("cpu")[name]
    assert call(*args) is None and call() is None and call(*args, 1) is None
    for i in range(len(args)):
        for wrong in (None, 7, "x", [1.0]):
            assert call(*args[:i], wrong, *args[i + 1:]) is None


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(_arguments("cpu")))
def test_takes_ordinary_tensors_and_declines_others(name):
    call, args = getattr(step._native(), name), _arguments(DEV)[name]
    assert call(*args) is not None
    for i, t in enumerate(args):
        if not isinstance(t, torch.Tensor):
            continue
        spaced = torch.stack([t, t], -1)[..., 0]
        for wrong in (t.cpu(), t.double(), t[..., :-1], t[None], 1.5, "x",
                      None if (name, i) not in (("norm_residual", 2), ("norm_residual_grad", 0), ("norm_residual_grad", 1), ("norm_residual_grad", 4)) else 0):
            assert call(*args[:i], wrong, *args[i + 1:]) is None, (i, wrong)
        if not (name == "vocab_loss_grad" and i == 0):                     # (dloss may have any stride)
            assert call(*args[:i], spaced, *args[i + 1:]) is None, i
    if name == "norm_residual":
        assert call(*args[:6], -1.0) is None


@pytest.mark.gpu
def test_both_ways_give_the_same(monkeypatch):
    g = torch.Generator(device=DEV).manual_seed(1)
    n = lambda *shape, dtype=BF: torch.randn(shape, device=DEV, generator=g).to(dtype)
    off = torch.tensor([0, 40, 40, 100], dtype=torch.int64, device=DEV)
    labels = torch.randint(-3, 50, (100,), device=DEV, generator=g)
    x, w, dy, v, f = n(100, 72), n(3, 40, 72), n(100, 40), n(50, 72), n(100, dtype=torch.float32).abs()
    gate, p = n(5, 72), n(72)

    def calls():
        loss, lse = step.vocab_loss(x, v, labels)
        h_out, u, r1, r2 = step.norm_residual(x, x, gate, p, p, 0.5, 1e-5)
        return [step.expert_product(x, w, off), *step.expert_product_grad(dy, x, w, off), loss, lse,
                *step.vocab_loss_grad(f, x, v, labels, lse), h_out, u, r1, r2,
                *step.norm_residual_grad(u, h_out, x, x, gate, p, p, r1, r2, 0.5), *step.norm_residual_grad(None, x, x, x, gate, p, p, r1, r2)]

    class Declines:
        def __getattr__(self, _):
            return lambda *a: None
    native = calls()
    monkeypatch.setattr(step, "_calls", Declines())
    assert all(torch.equal(a, b) for a, b in zip(native, calls()))


@pytest.mark.gpu
def test_another_current_stream_is_used():
    x, w, off = torch.ones(4, 8, dtype=BF, device=DEV), torch.ones(1, 16, 8, dtype=BF, device=DEV), torch.tensor([0, 4], device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        y = step.expert_product(x, w, off)
        end = side.record_event()
    end.synchronize()
    assert (y == 8).all()
