"""What the optimizer of a whole step does with its routers."""
import pytest
import torch

from paper_2605_04478_amd import rankstep, step

pytestmark = pytest.mark.gpu
SPEC = rankstep.StepSpec(d=96, hidden=128, experts=5, layers=2, vocab=300)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("choices", [1, 2, 5])
def test_a_router_learns_from_its_gradient_or_stays(choices, bits):
    """One choice: no gradient, and no decay either.  More: its masters move by up to lr in the first step, with the decay."""
    work = rankstep.RoutedStep(SPEC, choices, bits=bits)
    batch = work.batch([50, 0, 10, 3, 1], masked=0.2)

    def held():
        """The routers' and another weight's masters: what 16 bits would hide."""
        at, out = 0, {}
        for k, w in enumerate(work.weights()):
            out[k] = work.optimizer.state["master"][at:at + w.numel()].clone()
            at += -(-w.numel() // step.ADAMW_BLOCK) * step.ADAMW_BLOCK
        return out
    before = held()
    _, grads = work.gradients(*batch)
    routers = [g for w, g in zip(work.weights(), grads) if any(w is layer["router"] for layer in work.layers)]
    assert len(routers) == SPEC.layers and all(bool(g.any()) == (choices > 1) for g in routers)
    for _ in range(3):
        work.take(*batch)
    assert int(work.optimizer.state["count"]) == 3
    after = held()
    for k, w in enumerate(work.weights()):
        router = any(w is layer["router"] for layer in work.layers)
        assert torch.equal(before[k], after[k]) == (router and choices == 1), k


def test_another_weight_of_one_choice_would_be_undone():
    """A block multiplied by any number is normed to the same, but for eps: the weights over all experts would teach a router of one choice no more."""
    g = torch.Generator(device="cuda:0").manual_seed(1)
    h, b = (torch.randn(64, 96, device="cuda:0", generator=g) for _ in range(2))
    w = torch.ones(96, device="cuda:0")
    du = torch.randn(64, 96, device="cuda:0", generator=g)
    _, _, r1, r2 = step.norm_residual(h, b, None, w, w, 0.9, 1e-6)
    _, db, *_ = step.norm_residual_grad(du, du, h, b, None, w, w, r1, r2, 0.9)
    along = (db.double() * b.double()).sum(1)
    # db b = (1 - mean(b^2) r^2) ... = eps r^2 times du's part along b, and roundings: 96 products of a dozen roundings each
    assert float(along.abs().max()) <= (2e-6 + 96 * 12 * 2.0 ** -24) * float((db.double().abs() * b.double().abs()).sum(1).max())
