"""More rows than workgroups: every output of every row, by its own bound."""
import pytest
import torch

from paper_2605_04478_amd import step
from tests.step_check import F32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("v,top", [(8, 2), (8, 8), (5, 3)])
def test_more_rows_than_workgroups(v, top):
    """A workgroup's rows one after another use the same LDS: alternatives in their order, words exactly (all values of a row differ: consecutive multiples of a number modulo a
    larger prime)."""
    rows = (1 << 20) + 70001
    z = (torch.arange(rows * v, device=DEV).view(rows, v) * 2654435761 % 1009).float() / 128
    assert bool((z.sort(1).values.diff(dim=1) > 0).all())
    tokens = torch.arange(rows, device=DEV) % v
    logp, entropy, lse, ids, best = step.token_logprobs(z, tokens, 1.0, top)
    q = torch.log_softmax(z.double(), 1)
    order = z.sort(dim=1, descending=True, stable=True)[1][:, :top]
    assert torch.equal(ids.long(), order)
    # a dozen roundings of values below 8 + log 8
    bound = 12 * 16 * F32
    assert float((best - q.gather(1, order)).abs().max()) < bound
    assert float((lse - torch.logsumexp(z.double(), 1)).abs().max()) < bound
    assert float((logp - q.gather(1, tokens[:, None])[:, 0]).abs().max()) < bound
    assert float((entropy + (q.exp() * q).sum(1)).abs().max()) < 2 * bound


def test_parts_are_joined_to_their_rows():
    """Rows in parts: each row has its largest word in a place of its own."""
    rows, v = 300, 33001
    z = torch.zeros(rows, v, device=DEV)
    at = torch.arange(rows, device=DEV) * 97 % v
    second = (at + 16501) % v
    z[torch.arange(rows), at] = 20.0 + torch.arange(rows, device=DEV) / 64
    z[torch.arange(rows), second] = 19.0 + torch.arange(rows, device=DEV) / 64
    logp, entropy, lse, ids, best = step.token_logprobs(z, second, 1.0, 2)
    q = torch.log_softmax(z.double(), 1)
    assert torch.equal(ids.long(), torch.stack([at, second], 1))
    bound = 12 * 32 * F32                              # values below 32
    assert float((best - q.gather(1, ids.long())).abs().max()) < bound
    assert float((lse - torch.logsumexp(z.double(), 1)).abs().max()) < bound
    assert float((logp - q.gather(1, second[:, None])[:, 0]).abs().max()) < bound
    assert float((entropy + (q.exp() * q).sum(1)).abs().max()) < 2 * bound
