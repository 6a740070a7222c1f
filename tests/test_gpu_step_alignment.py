"""Operands that do not start on 16 bytes, at sizes that aligned ones compute in the largest tiles."""
import pytest
import torch

from tests.step_check import F32, close, rounding
from tests.test_gpu_vocab_precision import _check_gradients

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
DEV = "cuda:0"


def _shifted(t):
    """The same values, starting on an odd multiple of 2 bytes."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.flatten()
    return flat[1:].view(t.shape)


@pytest.mark.parametrize("which", ["x", "w", "dy", "all"])
def test_expert_products_of_shifted_operands(which):
    """8 experts of 2,048 x 2,048, 1,000 rows each."""
    from paper_2605_04478_amd import step
    e, n, k, each = 8, 2048, 2048, 1000
    g = torch.Generator(device=DEV).manual_seed(3)
    normal = lambda *shape: torch.randn(shape, device=DEV, generator=g).to(BF)
    x, w, dy = normal(e * each, k), normal(e, n, k), normal(e * each, n)
    off = torch.arange(e + 1, device=DEV) * each
    sx, sw, sdy = (_shifted(t) if which in (name, "all") else t for name, t in (("x", x), ("w", w), ("dy", dy)))
    y = step.expert_product(sx, sw, off)
    dx, dw = step.expert_product_grad(sdy, sx, sw, off)
    for i in (0, 3, e - 1):
        rows = slice(i * each, (i + 1) * each)
        xd, wd, gd = x[rows].double(), w[i].double(), dy[rows].double()
        # as in the products' other tests: an addition for each product, cut, and one rounding
        for got, a, b, terms in ((y[rows], xd, wd.t().contiguous(), k), (dx[rows], gd, wd, n), (dw[i], gd.t().contiguous(), xd, each)):
            want = torch.mm(a, b)
            close(got, want, rounding(want, BF) + 2 * F32 * (terms + 8) * torch.mm(a.abs(), b.abs()), which)


def test_the_loss_of_a_shifted_vocabulary():
    """4,096 rows x 4,096 x 8,192 words."""
    from paper_2605_04478_amd import step
    rows, d, vocab = 4096, 4096, 8192
    g = torch.Generator(device=DEV).manual_seed(4)
    w = (torch.randn(vocab, d, device=DEV, generator=g) * d ** -0.5).to(BF)
    h = torch.randn(rows, d, device=DEV, generator=g).to(BF)
    labels = torch.randint(-800, vocab, (rows,), device=DEV, generator=g)
    dloss = 0.25 + torch.rand(rows, device=DEV, generator=g)
    loss, lse = step.vocab_loss(h, w, labels)
    for sh, sw in ((h, _shifted(w)), (_shifted(h), _shifted(w)), (_shifted(h), w)):
        other = step.vocab_loss(sh, sw, labels)
        for a, b in zip(other, (loss, lse)):
            # the same products, joined to sums over tiles of another width: 300 roundings of sums of one
            assert (a - b).abs().max() <= 300 * F32 + 4 * F32 * float(lse.max())
        _check_gradients(h, w, labels, dloss, step.vocab_loss_grad(dloss, sh, sw, labels, other[1]), vocab + 16)
