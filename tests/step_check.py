"""What the tests of a training step's operators share: bounds on their errors, and a comparison that names the worst value."""
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
SMALLEST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}   # spacing next to zero
F32 = 2.0 ** -24


def rounding(want, dtype):
    """Most that one rounding of `want` to `dtype` changes it by."""
    return want.abs() * HALF_STEP[dtype] + SMALLEST[dtype]


def close(got, want, bound, what=""):
    """|got - want| <= bound everywhere; all in 64 bits on the CPU.  Infinities and NaN have to agree."""
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    if not want.numel():
        return
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)]), what
    over = torch.where(finite, (got - want).abs() - bound, torch.full_like(want, -1.0))
    at = int(over.argmax())
    assert float(over.flatten()[at]) <= 0, (what, at, float(got.flatten()[at]), float(want.flatten()[at]),
                                            float(bound.expand_as(want).flatten()[at]))
