"""Experts of equal scores get equal weights."""
import pytest
import torch

from paper_2605_04478_amd import step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("experts,k", [(16, 16), (40, 20), (64, 64), (128, 32), (256, 64), (500, 64), (1024, 64)])
@pytest.mark.parametrize("over_all", [False, True])
def test_equal_scores_have_equal_weights(experts, k, over_all):
    g = torch.Generator(device=DEV).manual_seed(experts)
    z = torch.randn(2000, experts, device=DEV, generator=g)
    z[:, ::2] = z[:, 1:2]                              # half of the experts share a score
    chosen, weights = step.route(z, k, over_all)
    score = z.gather(1, chosen.long())
    same = score[:, 1:] == score[:, :-1]
    assert int(same.sum()) > 1000
    assert torch.equal(weights[:, 1:][same], weights[:, :-1][same])
    # and the gradient of equal weights is equal
    d = step.route_grad(torch.ones_like(weights), z, chosen, weights, over_all)
    mine = d.gather(1, chosen.long())
    assert torch.equal(mine[:, 1:][same], mine[:, :-1][same])
