"""AdamW with an eps that is small beside the roots of 32-bit numbers, or none, against its formulas in 64 bits."""
import pytest
import torch

from paper_2605_04478_amd import step
from tests.step_check import F32, close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LEAST = 2.0 ** -149                     # spacing of 32-bit numbers next to zero


def _check(g, m0, v0, count, eps, betas, bits=32, lr=0.5):
    """A step of parameters that are zero."""
    n = g.numel()
    p = torch.zeros(n, device=DEV)
    state = step.adamw_state([p], bits)
    if bits == 32:
        state["m"][:n], state["v"][:n] = m0, v0
    state["count"].fill_(count)
    step.adamw([p], [g], state, lr, betas=betas, eps=eps)
    (b1, b2), t = betas, count + 1
    g, m0, v0 = g.double().cpu(), m0.double().cpu(), v0.double().cpu()
    m, v = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
    # products and factors round by a half step each, subnormal ones by half of their spacing; what is below it may be nothing
    em, ev = F32 * (2 * b1 * m0.abs() + 3 * (1 - b1) * g.abs() + m.abs()) + 2 * LEAST, F32 * (2 * b2 * v0 + 4 * (1 - b2) * g * g + v) + 2 * LEAST
    den = (v / (1 - b2 ** t)).sqrt() + eps
    # (the root's error: of v + ev and of v - ev, not by its slope, which is steep next to zero; eps itself rounds too)
    root = lambda x: (x.clamp(min=0) / (1 - b2 ** t)).sqrt()
    eden = torch.maximum(root(v + ev) - root(v), root(v) - root(v - ev)) + LEAST * (eps > 0)
    ratio = torch.where(m == 0, m, m / den)
    er = (em / (1 - b1 ** t) + ratio.abs() / (1 - b1 ** t) * eden) / (den - eden).clamp(min=1e-300) + 16 * F32 * ratio.abs() / (1 - b1 ** t)
    want = -lr * ratio / (1 - b1 ** t)
    er = torch.where((m0 == 0) & (g == 0), torch.zeros_like(er), er)         # a parameter that never had a gradient stays
    # (the parameter itself is a 32-bit number)
    close(p, want, lr * er + 4 * F32 * want.abs() + LEAST, (eps, betas, bits))


def _first(g, eps, betas, bits, lr=0.5):
    g = torch.tensor(g, device=DEV)
    _check(g, torch.zeros_like(g), torch.zeros_like(g), 0, eps, betas, bits, lr)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-19, 1e-18])
def test_large_gradients_beside_a_small_eps(eps, bits):
    """Squares up to the end of 32 bits."""
    _first([1e18, -3e15, 2e12, 1e10, -5.0, 1e-6], eps, (0.9, 0.999), bits)
    _first([1.8e19, -1e19], eps, (0.9, 0.5), bits)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps,betas", [(1e-18, (0.9, 0.999)), (1e-17, (0.9, 0.999)), (1e-15, (0.9, 0.9999)), (1e-12, (0.9, 0.999999)), (1e-11, (0.9, 1 - 1e-7))], ids=str)
def test_small_gradients_beside_a_small_eps(eps, betas, bits):
    """Squares that are subnormal in 32 bits, whose roots over sqrt(1 - b2^t) are as large as eps, or not nothing beside it."""
    top = 1e-19 / (1 - betas[1]) ** 0.5          # v = 1e-38
    _first([3e-18, -1e-18, 1e-17, 1e-16, 1e-12, 1.0, top, -0.5 * top, 0.1 * top, 3 * top], eps, betas, bits)


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-18, 1e-12, 1e-8])
def test_later_steps(eps):
    """Moments anywhere, many steps on."""
    e = torch.linspace(-125, 124, 300, device=DEV)
    v0 = torch.ldexp(1 + torch.rand(300, device=DEV), e.round().int())
    v0[:20] = torch.ldexp(torch.ones(20, device=DEV), torch.arange(-148, -128, device=DEV).int())
    m0 = v0.sqrt() * torch.randn(300, device=DEV)
    _check(torch.zeros(300, device=DEV), m0, v0, 10 ** 6, eps, (0.9, 0.999))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-30, 1e-38, 1e-40, 1e-45, 1e-60, 5e-324])
def test_what_never_had_a_gradient_stays(eps, bits):
    """m = v = 0: the ratio is 0 / eps, whatever 32 bits have of eps and its reciprocal."""
    _first([0.0, -0.0, 1.0, 1e-18, 0.0, -1e10], eps, (0.9, 0.999), bits)


@pytest.mark.parametrize("eps", [1e-37, 1e-38, 1e-39, 1e-40])
def test_quotients_by_a_subnormal_eps(eps):
    m0 = torch.tensor([1e-33, -1e-36, 1e-38, 0.0, 3e-35], device=DEV)
    _check(torch.zeros_like(m0), m0, torch.zeros_like(m0), 10 ** 6, eps, (0.9, 0.999))


@pytest.mark.parametrize("eps", [1e20, 1e38, 1.5e38, 1e300])
def test_a_large_eps(eps):
    """A step of 10^18 by ratios of 10^-18: a reciprocal that is subnormal is no zero."""
    _first([1e18, -3e18, 1.0], eps, (0.0, 0.999), 32, lr=1e20)
