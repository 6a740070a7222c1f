"""What rounding dz to 16 bits may leave of the vocabulary loss's gradients, what reaches dh from every piece of a huge vocabulary, and rows
whose gradient is infinite."""
import pytest
import torch

from tests.step_check import F32, HALF_STEP, close, rounding

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16
DEV = "cuda:0"


def _mm(a, b):
    return torch.mm(a.contiguous(), b.contiguous())


def _run(h, w, labels, dloss):
    from paper_2605_04478_amd import step
    h, w, labels, dloss = (t.to(DEV) for t in (h, w, labels, dloss))
    loss, lse = step.vocab_loss(h, w, labels)
    return step.vocab_loss_grad(dloss, h, w, labels, lse)


def _inputs(rows, d, vocab, dtype, labels, seed):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(vocab, d, generator=g) * d ** -0.5).to(dtype)
    h = torch.randn(rows, d, generator=g).to(dtype)
    return h, w, labels(rows, vocab, g), 0.25 + torch.rand(rows, generator=g)


def _once(rows, vocab, g):
    return torch.randperm(vocab, generator=g)[:rows]


def _any(rows, vocab, g):
    return torch.randint(0, vocab, (rows,), generator=g)


def _three_words(rows, vocab, g):
    return torch.tensor([1, vocab // 2, vocab - 1])[torch.randint(0, 3, (rows,), generator=g)]


def _few_kept(rows, vocab, g):
    labels = torch.full((rows,), -100)
    labels[[0, rows // 2, rows - 1]] = torch.tensor([5, 5, vocab - 1])
    return labels


def _check_gradients(h, w, labels, dloss, got, steps):
    """Against 64 bits.  Up to 128 kept rows all of dz has the bits of two parts, beyond that the target's dz has them, and any other
    value is rounded once.  steps: additions that a product passes in dh's sum."""
    dtype, (rows, d), vocab = h.dtype, h.shape, w.shape[0]
    h, w, labels, g = h.to(DEV).double(), w.to(DEV).double(), labels.to(DEV), dloss.to(DEV).double()
    used = (labels >= 0) & (labels < vocab)
    at = torch.where(used, labels, 0)[:, None]
    z = _mm(h, w.t())
    p = torch.exp(z - torch.logsumexp(z, 1)[:, None])
    g = (g * used)[:, None]
    dz = (p - torch.zeros_like(p).scatter_(1, at, 1.0)) * g
    # logits: d + 8 additions of the sum of magnitudes, cut instead of rounded; lse: that of its row, and its own sum; exponentials; p - 1
    # at the target; subnormal parts
    size = 2 * F32 * (d + 8) * _mm(h.abs(), w.abs().t())
    d_dz = g * p * (size + size.amax(1, keepdim=True) + 1000 * F32) + 2.0 ** -38 * float(g.max())
    d_dz = d_dz.scatter_add(1, at, 4 * F32 * g)
    twice = 2 * HALF_STEP[dtype] ** 2 * dz.abs()
    once = HALF_STEP[dtype] * dz.abs()
    d_dz += twice if int(used.sum()) <= 128 else once.scatter(1, at, twice.gather(1, at))
    bounds = {}
    for k, want, off, there, other, terms, value in (
            ("dh", _mm(dz, w), d_dz, dz.abs(), w.abs(), steps, got[0]),
            ("dw", _mm(dz.t(), h), d_dz.t(), dz.abs().t(), h.abs(), 2 * rows + 16, got[1])):
        bounds[k] = rounding(want, dtype) + _mm(off, other) + 2 * F32 * terms * _mm(there, other)
        close(value, want, bounds[k], k)
    return dz, w, bounds


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("labels", [_once, _any, _three_words, _few_kept], ids=lambda f: f.__name__[1:])
@pytest.mark.parametrize("rows,d,vocab", [(128, 72, 700), (129, 72, 700), (250, 33, 4001), (1000, 200, 5003), (1100, 264, 1300), (2000, 64, 12000)])
def test_a_targets_gradient_rounds_once(rows, d, vocab, labels, dtype):
    h, w, labels, dloss = _inputs(rows, d, vocab, dtype, labels, seed=rows + d)
    _check_gradients(h, w, labels, dloss, _run(h, w, labels, dloss), vocab + 16)


@pytest.mark.parametrize("d,vocab", [(40, 300), (520, 2100)])
def test_targets_of_many_rows(d, vocab):
    """More rows than a workgroup looks through at once, most of them with the same few targets."""
    g = torch.Generator().manual_seed(7)
    w = (torch.randn(vocab, d, generator=g) * d ** -0.5).to(BF)
    h = torch.randn(17000, d, generator=g).to(BF)
    labels = (vocab ** torch.rand(17000, generator=g)).long() - 1
    labels[torch.rand(17000, generator=g) < 0.05] = -1
    dloss = 0.25 + torch.rand(17000, generator=g)
    got = _run(h, w, labels, dloss)
    _check_gradients(h, w, labels, dloss, got, vocab + 16)
    for _ in range(3):               # the order in which workgroups end decides nothing
        assert all(torch.equal(a, b) for a, b in zip(got, _run(h, w, labels, dloss)))


@pytest.mark.parametrize("rows", [24, 40])
def test_every_piece_of_a_huge_vocabulary_reaches_dh(rows):
    """5 million words in three pieces, each with words of its own mean: dh without any one piece would be far off.  A product passes the
    additions of its part's steps of 32 (all of a piece's at most), 32 within a step, 64 parts and 3 pieces."""
    vocab, d = 5_000_003, 8
    piece = -(-vocab // 3 // 256) * 256
    g = torch.Generator().manual_seed(rows)
    mean = torch.randint(0, 2, (3, d), generator=g).float() * 2 - 1
    mean = (0.5 + torch.rand(3, d, generator=g)) * mean
    word = torch.arange(vocab) // piece
    w = (mean[word.clamp(max=2)] + 0.1 * torch.randn(vocab, d, generator=g)).to(BF)
    h = (0.05 * torch.randn(rows, d, generator=g)).to(BF)
    labels = torch.randint(0, vocab, (rows,), generator=g)
    dloss = 0.25 + torch.rand(rows, generator=g)
    dz, wd, bounds = _check_gradients(h, w, labels, dloss, _run(h, w, labels, dloss), (1 << 21) // 32 + 32 + 64 + 3)
    for i in range(3):
        share = _mm(dz[:, i * piece:(i + 1) * piece], wd[i * piece:(i + 1) * piece])
        assert (share.abs() > 2 * bounds["dh"]).all(), i


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows", [20, 300])
def test_an_infinite_gradient_stays_with_its_row(rows, dtype):
    """A row whose dloss is infinite (a loss scale that overflowed) leaves the other rows' dh as they are without it, and is infinite, not
    NaN, in dw."""
    h, w, labels, dloss = _inputs(rows, 64, 400, dtype, _any, seed=rows)
    h = torch.where(h == 0, torch.ones_like(h), h)
    for scale in (1.0, 1e-6):
        g = dloss * scale
        g[3] = 0
        clean = _run(h, w, labels, g)
        for value in (float("inf"), -float("inf")):
            g[3] = value
            dh, dw = _run(h, w, labels, g)
            rest = torch.arange(rows) != 3
            assert torch.equal(dh[rest.to(DEV)], clean[0][rest.to(DEV)])
            sign = torch.ones(400, 1)
            sign[labels[3]] = -1
            assert torch.equal(dw.cpu(), sign.to(dtype) * h[3:4] * value)
