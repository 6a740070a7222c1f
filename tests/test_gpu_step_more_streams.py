"""The calls around a step's products go to the current stream of their tensors' device, and wait for what that stream is still writing."""
import pytest
import torch

from paper_2605_04478_amd import step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Declines:
    def __getattr__(self, _):
        return lambda *a: None


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_the_current_stream_is_waited_for(native, monkeypatch):
    g = torch.Generator(device=DEV).manual_seed(1)
    n = lambda *shape: torch.randn(shape, device=DEV, generator=g)
    z, w, y, dout, dlogp = n(300, 40), n(300, 3), n(900, 64), n(300, 64), n(300)
    tokens = torch.randint(0, 40, (300,), device=DEV, generator=g)
    experts, weights = step.route(z, 3)
    places, offsets = step.expert_order(experts, 40)
    _, entropy, lse, _, _ = step.token_logprobs(z, tokens)

    def stepped(x):
        params = [torch.ones(300, 40, device=DEV)]
        state = step.adamw_state(params, 8)
        step.adamw(params, [x], state, 1e-2)
        return params + [state["m"].view(torch.uint8), state["m_scale"]]
    calls = {
        "route": (z, lambda x: list(step.route(x, 3))),
        "route_grad": (w, lambda x: [step.route_grad(x, z, experts, weights)]),
        "expert_order": (experts, lambda x: list(step.expert_order(x, 40))),
        "dispatch": (dout, lambda x: [step.dispatch(x, places, offsets)]),
        "dispatch_grad": (y, lambda x: [step.dispatch_grad(x, places)]),
        "combine": (y, lambda x: [step.combine(x, places, weights)]),
        "combine_grad": (dout, lambda x: list(step.combine_grad(x, y, places, weights, offsets))),
        "token_logprobs": (z, lambda x: list(step.token_logprobs(x, tokens, 1.0, 4))),
        "token_logprobs_grad": (dlogp, lambda x: [step.token_logprobs_grad(x, None, z, tokens, lse, entropy)]),
        "adamw": (z, stepped),
    }
    if not native:
        step._native()
        monkeypatch.setattr(step, "_calls", Declines())
    work = torch.zeros(1 << 28, device=DEV)          # 1 GB: an addition takes 0.3 ms
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                    # (first uses load their kernels, which takes its time)
        work.add_(1.0)
        for new, call in calls.values():
            new.clone().copy_(new)
            call(new)
        side.record_event().query()
    torch.cuda.synchronize()
    for name, (new, call) in calls.items():
        want, x = call(new), new.flip(0).contiguous()
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
