"""Sums over long rows of logits do not lose bits with their length, wherever a thread's reference lies."""
import math

import pytest
import torch

from paper_2605_04478_amd import step
from tests.step_check import F32, close, rounding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rows(rows, v, dtype, low):
    """Nearly flat rows; with `low` a row's first values, one vector to each of 256 threads, are up to 2^-7.9 of the others: less than makes a thread measure from
    the others instead."""
    g = torch.Generator(device=DEV).manual_seed(v + rows)
    flat = torch.rand(rows, 1, device=DEV, generator=g)
    z = flat.expand(rows, v).clone()
    z[1::3] += 0.02 * torch.randn(z[1::3].shape, device=DEV, generator=g)
    if low:
        n = 16 // torch.empty(0, dtype=dtype).element_size()
        z[:, :256 * n] -= 4.5 + 0.9 * torch.rand(rows, 1, device=DEV, generator=g)
    return z.to(dtype)


def _exact(z, temperature):
    q = torch.log_softmax(z.double() / temperature, 1)
    return q, -(q.exp() * q).sum(1), torch.logsumexp(z.double() / temperature, 1)


# rows in parts of registers, in parts that are read again, whole
SHAPES = [(3, 128000), (1, 300001), (2, 1200007), (700, 131072), (600, 200003), (1100, 40000)]


@pytest.mark.parametrize("low", [False, True])
@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_entropy_and_lse(rows, v, dtype, low):
    z = _rows(rows, v, dtype, low)
    tokens = torch.randint(0, v, (rows,), device=DEV)
    logp, entropy, lse, _, _ = step.token_logprobs(z, tokens)
    for at in range(0, rows, 100):                      # (64 bits of a hundred rows at a time)
        part = slice(at, at + 100)
        q, h, want = _exact(z[part], 1.0)
        # Exponents are up to 8 in magnitude: their difference, factor and power of two are off by 3 half steps of 8, by which terms change, and the entropy by as much
        # (terms at one distance from the reference change alike, which changes nothing).  The entropy's terms are 8 times their exponentials at most: a vector's
        # eight sums, a thread's sum with its rest and its last move, and a dozen sums over threads and parts round 22 times.
        s = F32 * (3 * 8 + 22) * math.log(2)
        close(lse[part], want, s + F32 * 2 * (want.abs() + math.log(v)), "lse")
        close(entropy[part], h, s + F32 * 8 * math.log(2) * 22 + F32 * 4 * (h + math.log(v)), "entropy")
        exact = q.gather(1, tokens[part, None])[:, 0]
        close(logp[part], exact, s + F32 * 4 * (exact.abs() + math.log(v)), "logp")


@pytest.mark.parametrize("rows,v", [(3, 65536), (3, 128000), (520, 100003), (5, 262147)])
def test_gradient(rows, v):
    """A probability's relative error is that of the sum and of its own exponent, which is at most log V."""
    z = _rows(rows, v, torch.float32, False)
    tokens = torch.full((rows,), -1, device=DEV)
    _, entropy, lse, _, _ = step.token_logprobs(z, tokens)
    tokens[:] = 7
    got = step.token_logprobs_grad(torch.ones(rows, device=DEV), None, z, tokens, lse, entropy)
    for at in range(0, rows, 100):
        part = slice(at, at + 100)
        q, _, want = _exact(z[part], 1.0)
        d = -q.exp()
        # exponents, which are log V from lse: difference and factor in the sum's terms and in the value, and the value's step to the sum; then powers, products; sums as above
        relative = F32 * (5 * math.log2(v) * math.log(2) + 22 + 8)
        d[:, 7] += 1
        bound = q.exp() * relative + rounding(d, torch.float32)
        close(got[part], d, bound, "dlogits")
