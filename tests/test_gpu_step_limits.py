"""More rows than one launch has threads for: 2^26 wavefronts of 64 threads are 2^32 threads."""
import pytest
import torch

from paper_2605_04478_amd import step

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
DEV = "cuda:0"
ROWS = (1 << 26) + 8


def test_norms_of_more_rows_than_a_launch_has():
    g = torch.Generator(device=DEV).manual_seed(1)
    h = torch.empty(ROWS, 8, dtype=BF, device=DEV).normal_(generator=g)
    b = torch.empty(ROWS, 8, dtype=BF, device=DEV).normal_(generator=g)
    gate = torch.empty(8, 8, dtype=BF, device=DEV).normal_(generator=g)
    w1, w2 = (1 + 0.1 * torch.randn(2, 8, device=DEV, generator=g)).to(BF)
    got = step.norm_residual(h, b, gate, w1, w2, 0.5, 1e-6)
    half = ROWS // 2
    for rows, gates in ((slice(0, half), slice(0, 4)), (slice(half, ROWS), slice(4, 8))):
        want = step.norm_residual(h[rows], b[rows], gate[gates], w1, w2, 0.5, 1e-6)
        assert all(torch.equal(t[rows], w) for t, w in zip(got, want))


def test_losses_of_more_rows_than_a_launch_has():
    g = torch.Generator(device=DEV).manual_seed(2)
    h = torch.empty(ROWS, 8, dtype=BF, device=DEV).normal_(generator=g)
    w = torch.randn(16, 8, device=DEV, generator=g).to(BF)
    labels = torch.randint(0, 16, (ROWS,), device=DEV, generator=g, dtype=torch.int32)
    loss, lse = step.vocab_loss(h, w, labels)
    half = ROWS // 2
    for rows in (slice(0, half), slice(half, ROWS)):
        want = step.vocab_loss(h[rows], w, labels[rows])
        assert torch.equal(loss[rows], want[0]) and torch.equal(lse[rows], want[1])
    tail = slice(ROWS - 1000, ROWS)
    z = h[tail].double() @ w.double().t().contiguous()
    # 16 additions of products of magnitude 8 at most, and of exponentials
    assert (lse[tail].double() - torch.logsumexp(z, 1)).abs().max() < 1e-4
