"""A call's work goes to the current stream of its tensors' device: it waits for what that stream is still writing."""
import pytest
import torch

from paper_2605_04478_amd import step

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
DEV = "cuda:0"


class Declines:
    def __getattr__(self, _):
        return lambda *a: None


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_the_current_stream_is_waited_for(native, monkeypatch):
    g = torch.Generator(device=DEV).manual_seed(1)
    n = lambda *shape, dtype=BF: torch.randn(shape, device=DEV, generator=g).to(dtype)
    off = torch.tensor([0, 40, 40, 100], dtype=torch.int64, device=DEV)
    labels = torch.randint(-3, 50, (100,), device=DEV, generator=g)
    w, dy, v, f, gate, p = n(3, 40, 72), n(100, 40), n(50, 72), n(100, dtype=torch.float32).abs(), n(5, 72), n(72)
    calls = {
        "expert_product": lambda x: [step.expert_product(x, w, off)],
        "expert_product_grad": lambda x: list(step.expert_product_grad(dy, x, w, off)),
        "vocab_loss": lambda x: list(step.vocab_loss(x, v, labels)),
        "vocab_loss_grad": lambda x: list(step.vocab_loss_grad(f, x, v, labels, f)),
        "norm_residual": lambda x: list(step.norm_residual(x, x, gate, p, p)),
        "norm_residual_grad": lambda x: list(step.norm_residual_grad(x, x, x, x, gate, p, p, f, f)),
    }
    if not native:
        step._native()
        monkeypatch.setattr(step, "_calls", Declines())
    old, new = n(100, 72), n(100, 72)
    work = torch.zeros(1 << 28, device=DEV)          # 1 GB: an addition takes 0.3 ms
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                    # (first uses load their kernels, which takes its time)
        work.add_(1.0)
        old.clone().copy_(new)
        side.record_event().query()
    for name, call in calls.items():
        want, x = call(new), old.clone()
        assert not all(torch.equal(a, b) for a, b in zip(want, call(x))), name
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(60):                      # 20 ms before x has its new values
                work.add_(1.0)
            x.copy_(new)
            got = call(x)
            end = side.record_event()
        assert not end.query(), name                 # the call returned before its work was done
        end.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
