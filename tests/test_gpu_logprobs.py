"""Log probabilities of tokens, entropy, alternatives and the gradient against plain computations in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2605_04478_amd import step
from tests.step_check import F32, close, rounding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MOST = torch.finfo(torch.float32).max
INF, NAN = float("inf"), float("nan")
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _exact(logits, tokens, temperature, top):
    raw = logits.double().cpu()
    v, m = raw.shape[1], raw.amax(1)
    none = m == -INF
    # relative to the largest: beside the lowest value of a type even 64 bits lose the sum's logarithm
    z = (raw - torch.where(none, torch.zeros_like(m), m)[:, None]) / temperature
    rest = torch.where(none, torch.zeros_like(m), torch.logsumexp(z, 1))
    lse = m / temperature + rest
    lse = torch.where(none, lse, lse.clamp(-MOST, MOST))          # 32 bits have no more
    logp = z - rest[:, None]
    p = torch.exp(logp)
    h = -(p * torch.where(p > 0, logp, torch.zeros_like(logp))).sum(1)
    tokens = tokens.long().cpu()
    used = (tokens >= 0) & (tokens < v)
    mine = torch.where(used, logp.gather(1, tokens.clamp(0, v - 1)[:, None])[:, 0], torch.zeros(()))
    raw = raw.numpy()
    order = np.argsort(-raw, axis=1, kind="stable")[:, :top]
    ids = np.where(np.take_along_axis(raw, order, 1) > -INF, order, -1)
    ids = np.concatenate([ids, np.full((ids.shape[0], top - ids.shape[1]), -1)], 1)
    best = torch.where(torch.from_numpy(ids) >= 0, logp.gather(1, torch.from_numpy(ids).clamp(min=0)), torch.full((), -INF, dtype=torch.float64))
    beyond = lambda x: torch.where(x < -MOST * (1 + F32 / 2), torch.full_like(x, -INF), x)      # what 32 bits round to infinity
    return beyond(mine), h, lse, ids, beyond(best), p, logp, used


def _bounds(logits, temperature, h, lse, v):
    """Errors of the values.  S, a sum of exponentials relative to the largest: an exponent x is off by 6 F32 |x| (difference, factor, product, and once more where the
    sum moves to a larger maximum), whose mean under p is below log V; a thread adds V / 256 terms and one per sum that is joined, each move rounds three times, and there
    are 60 of both at most but for one row in millions."""
    z = logits.double().cpu()
    m = torch.where(torch.isfinite(z.amax(1)), z.amax(1), torch.zeros(())).abs() / temperature
    log_v = math.log(v) + 1
    s = F32 * (6 * log_v + v / 256 + 200)
    return dict(s=s, lse=s + F32 * (4 * m + 4 * log_v + lse.abs()), entropy=s * (1 + 2 * h) + 8 * F32 * (h + 1 + log_v),
                logp=lambda logp: s + F32 * (4 * logp.abs() + 4 * log_v) + F32 * 2 * logp.abs())


def _check(logits, tokens, temperature, top, gradient=True):
    v, dtype = logits.shape[1], logits.dtype
    logp, entropy, lse, ids, best = step.token_logprobs(logits, tokens, temperature, top)
    want, h, wlse, wids, wbest, p, logs, used = _exact(logits, tokens, temperature, top)
    assert ids.dtype == torch.int32 and all(t.dtype == torch.float32 for t in (logp, entropy, lse, best))
    b = _bounds(logits, temperature, h, wlse, v)
    close(lse, wlse, b["lse"], "lse")
    close(entropy, h, b["entropy"], "entropy")
    close(logp, want, b["logp"](want), "logp")
    assert np.array_equal(ids.cpu().numpy(), wids)
    close(best, wbest, b["logp"](wbest), "top")
    if not gradient:
        return
    g = torch.Generator(device=DEV).manual_seed(logits.numel())
    dlogp, dentropy = torch.randn(len(logits), device=DEV, generator=g), torch.randn(len(logits), device=DEV, generator=g)
    dlogp[tokens.to(DEV) < 0] = NAN                              # does not matter
    d, de = torch.where(used, dlogp.double().cpu(), torch.zeros(()))[:, None], dentropy.double().cpu()[:, None]
    safe = torch.where(p > 0, logs, torch.zeros_like(logs))
    hot = torch.zeros_like(p).scatter_(1, tokens.long().cpu().clamp(0, v - 1)[:, None], used[:, None].double())
    alive = (wlse > -INF)[:, None]
    at_t = torch.where(alive, hot, torch.zeros(()))
    wantd = (at_t * d - p * (d + de * (safe + h[:, None]))) / temperature
    # p's exponent: the logit's product and lse, or, far from zero, S and the difference to the largest
    z = torch.where(p > 0, logits.double().cpu(), torch.zeros(())) / temperature
    near = F32 * (4 * z.abs() + 4 * wlse.abs()[:, None]) + b["lse"][:, None]
    relative = torch.where((wlse.abs() < 63)[:, None], near, F32 * 6 * safe.abs() + 2 * b["s"]) + 8 * F32
    relative = torch.where((wlse.abs() >= 63)[:, None] & (wlse.abs() < 65)[:, None], torch.maximum(near, relative), relative)
    size = p * (d.abs() + de.abs() * (safe.abs() + h[:, None]))
    bound = torch.where(p > 0, size * (relative + 8 * F32) + p * de.abs() * (relative + b["entropy"][:, None]), torch.zeros(())) / temperature
    got = step.token_logprobs_grad(dlogp, dentropy, logits, tokens, lse, entropy, temperature)
    assert got.dtype == dtype
    # (exponentials below the smallest normal value are zero)
    close(got, wantd, torch.nan_to_num(bound, posinf=0.0) + 4 * F32 * wantd.abs() + 2.0 ** -118 * (d.abs() + 200 * de.abs()) / temperature + rounding(wantd, dtype), "dlogits")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,v,top,temperature", [(1, 1, 1, 1.0), (3, 7, 7, 0.7), (4, 5, 9, 1.0), (5, 1000, 20, 2.0), (2, 1025, 64, 1.0), (9, 4099, 5, 0.3), (511, 2000, 3, 1.0),
                                                    (700, 1537, 10, 1.0), (513, 64, 64, 1.5), (4, 128000, 20, 1.0), (3, 50021, 1, 0.7), (2, 300001, 0, 1.0), (2, 1200007, 5, 1.0), (90, 40000, 20, 1.0), (300, 33001, 2, 0.6),
                                                    (1500, 9001, 2, 1.0), (280, 70003, 1, 1.0)])
def test_rows(rows, v, top, temperature, dtype):
    g = torch.Generator(device=DEV).manual_seed(rows + v)
    z = torch.randn(rows, v, device=DEV, generator=g) * (0.2 + 6 * torch.rand(rows, 1, device=DEV, generator=g))
    z[::2] = z[::2].round()                                      # ties
    z[torch.rand(rows, v, device=DEV, generator=g) < 0.1] = -INF
    z[:, 0] = z[:, 0].clamp(min=-50)
    tokens = torch.randint(0, v, (rows,), device=DEV, generator=g)
    tokens[torch.rand(rows, device=DEV, generator=g) < 0.2] = -100
    _check(z.to(dtype), tokens if rows % 2 else tokens.int(), temperature, top)


@pytest.mark.parametrize("v", [9000, 45003])                       # whole rows; parts
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_masks(dtype, v):
    """Rows of nothing, of one word, of the type's lowest value, with it as a mask, far from zero, with more equal logits than the candidates have room for."""
    low = torch.finfo(dtype).min
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randn(12, v, device=DEV, generator=g)
    z[0] = -INF
    z[1] = -INF
    z[1, 8999] = 3.0
    z[2] = low
    z[3] = low
    z[3, 5000:5003] = torch.tensor([1.0, 2.0, 1.0], device=DEV)
    z[4] += 300
    z[5] -= 5000
    z[6] = 0
    z[7] = torch.where(z[7] > 0, torch.ones(()).cuda(), torch.zeros(()).cuda())
    z[8, 100:] = -INF
    z[9, ::512] += 40                                             # candidates that fall to few threads
    z[10, :4096] = 2.0
    tokens = torch.tensor([3, 8999, 17, 5001, 4, 5, 8999, 0, 50, 512, 0, v], device=DEV)
    for top in (0, 1, 5, 64):
        for temperature in (1.0, 0.25):
            _check(z.to(dtype), tokens, temperature, top)
    if v == 9000:
        many = z.repeat(60, 1).to(dtype)
        _check(many, tokens.repeat(60), 1.0, 20)


def test_a_token_that_is_ruled_out():
    z = torch.tensor([[0.0, -INF, 1.0]], device=DEV)
    tokens = torch.tensor([1], device=DEV)
    logp, entropy, lse, ids, best = step.token_logprobs(z, tokens, 1.0, 3)
    assert logp.tolist() == [-INF] and ids.tolist() == [[2, 0, -1]] and best[0, 2] == -INF
    got = step.token_logprobs_grad(torch.ones(1, device=DEV), None, z, tokens, lse, entropy)
    p = torch.softmax(z.double().cpu(), 1)
    close(got, torch.tensor([[0.0, 1.0, 0.0]]).double() - p, torch.full((1, 3), 2.0 ** -20))


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("rows,v", [(2, 3000), (600, 3000), (2, 60000)])
def test_rows_that_are_not_finite_are_nan_and_alone(rows, v, bad):
    z = torch.randn(rows, v, device=DEV)
    z[1, 2000] = bad
    z[1, 4] = 50.0
    tokens = torch.full((rows,), 7, device=DEV)
    want = step.token_logprobs(torch.cat([z[:1], z[:1]]), tokens[:2], 1.0, 4)
    out = step.token_logprobs(z, tokens, 1.0, 4)
    for a, b in zip(out, want):
        if rows == 2:
            assert torch.equal(a[0], b[0])
    assert all(torch.isnan(t[1]).all() for t in (out[0], out[1], out[2], out[4])) and torch.isfinite(out[0][[0, -1 if rows > 2 else 0]]).all()
    assert out[3][1].tolist()[:1] == [4 if bad != bad else 2000]
    d = step.token_logprobs_grad(out[2] * 0 + 1, None, z, tokens, out[2], out[1])
    assert torch.isnan(d[1]).all() and torch.isfinite(d[0]).all()
    alone = torch.full((1, 40), -INF, device=DEV)
    alone[0, 3] = bad
    assert all(torch.isnan(t).all() for t in step.token_logprobs(alone, torch.tensor([3], device=DEV))[:3])


def test_gradient_by_itself_and_against_differences():
    g = torch.Generator(device=DEV).manual_seed(3)
    z = torch.randn(3, 11, device=DEV, generator=g)
    tokens = torch.tensor([2, 10, -1], device=DEV)
    a, b = torch.randn(3, device=DEV, generator=g), torch.randn(3, device=DEV, generator=g)
    _, h, lse, _, _ = step.token_logprobs(z, tokens, 0.8)
    both = step.token_logprobs_grad(a, b, z, tokens, lse, h, 0.8)
    one, two = step.token_logprobs_grad(a, None, z, tokens, lse, h, 0.8), step.token_logprobs_grad(None, b, z, tokens, lse, h, 0.8)
    assert torch.allclose(one + two, both, atol=1e-6) and not one[2].any() and two[2].any()
    assert not step.token_logprobs_grad(None, None, z, tokens, lse, h, 0.8).any()
    value = lambda x: (lambda o: float((o[0].double() * a + o[1].double() * b).sum()))(step.token_logprobs(x, tokens, 0.8))
    for r, c in ((0, 2), (1, 3), (2, 7), (0, 0)):
        d = torch.zeros_like(z)
        d[r, c] = 2.0 ** -6
        # the third derivatives are below 8 / 0.8^3 |a, b|, the values off by 2^-20
        bound = (2.0 ** -12 * 16 + 2 * 2.0 ** -20 * 2.0 ** 5 * 12) * float(a.abs().max() + b.abs().max())
        assert abs((value(z + d) - value(z - d)) * 2.0 ** 5 - float(both[r, c])) < bound


def test_automatic_differentiation():
    g = torch.Generator(device=DEV).manual_seed(4)
    z = torch.randn(6, 500, device=DEV, generator=g).requires_grad_()
    tokens = torch.randint(0, 500, (6,), device=DEV, generator=g)
    logp, entropy = step.TokenLogprobs.apply(z, tokens, 1.3)
    wide = z.detach().double().cpu().requires_grad_()
    q = torch.log_softmax(wide / 1.3, 1)
    want = q.gather(1, tokens.cpu()[:, None]).sum() * 0.5 - 0.01 * (q.exp() * q).sum()
    for out, ref in (((0.5 * logp + 0.01 * entropy).sum(), want), (0.5 * logp.sum(), q.gather(1, tokens.cpu()[:, None]).sum() * 0.5), (entropy.sum(), -(q.exp() * q).sum())):
        got, = torch.autograd.grad(out, z, retain_graph=True)
        exact, = torch.autograd.grad(ref, wide, retain_graph=True)
        assert float((got.double().cpu() - exact).abs().max()) < 500 * F32


def test_layouts_and_both_ways_of_calling(monkeypatch):
    g = torch.Generator(device=DEV).manual_seed(5)
    z = torch.randn(7, 1001, device=DEV, generator=g).bfloat16()
    tokens = torch.randint(0, 1001, (7,), device=DEV, generator=g)
    dl = torch.randn(7, device=DEV, generator=g)
    apart = lambda t: torch.stack([t, t], -1)[..., 0]

    def calls(z, tokens, dl):
        out = step.token_logprobs(z, tokens, 0.9, 6)
        return [*out, step.token_logprobs_grad(dl, dl, z, tokens, out[2], out[1], 0.9), step.token_logprobs_grad(dl[:1].expand(7), None, z, tokens, out[2], out[1], 0.9)]

    class Declines:
        def __getattr__(self, _):
            return lambda *a: None
    want = calls(z, tokens, dl)
    same = lambda got: all(torch.equal(a, b) for a, b in zip(got, want))
    for f in (apart, lambda t: t.t().contiguous().t(), lambda t: torch.cat([t, t], -1)[..., :t.shape[-1]]):
        assert same(calls(f(z), tokens, dl)) and same(calls(z, apart(tokens), apart(dl)))
    lse, h = want[2], want[1]
    for name, args in dict(token_logprobs=(z, tokens, 0.9, 6), token_logprobs_grad=(dl, dl, z, tokens, lse, h, 0.9)).items():
        call = getattr(step._native(), name)
        assert call(*args) is not None
        for i, a in enumerate(args):
            for wrong in ((a.cpu(), a[None], a.double(), "x") if isinstance(a, torch.Tensor) else ("x", -1, None)):
                assert call(*args[:i], wrong, *args[i + 1:]) is None, (name, i, wrong)
    monkeypatch.setattr(step, "_calls", Declines())
    assert same(calls(z, tokens, dl)) and same(calls(z, tokens.int(), dl))


def test_without_rows():
    z, t, f = torch.zeros(0, 9, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, device=DEV)
    out = step.token_logprobs(z, t, 1.0, 3)
    assert [tuple(o.shape) for o in out] == [(0,), (0,), (0,), (0, 3), (0, 3)] and step.token_logprobs_grad(f, f, z, t, f, f).shape == (0, 9)


def test_captured_and_replayed():
    g = torch.Generator(device=DEV).manual_seed(6)
    z, tokens, dl = torch.randn(40, 30000, device=DEV, generator=g), torch.randint(0, 30000, (40,), device=DEV, generator=g), torch.randn(40, device=DEV, generator=g)

    def calls():
        out = step.token_logprobs(z, tokens, 1.0, 8)
        return [*out, step.token_logprobs_grad(dl, dl, z, tokens, out[2], out[1])]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = calls()
    for _ in range(3):
        z.normal_(generator=g)
        want = calls()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_more_rows_than_workgroups():
    rows = (1 << 20) + 70001
    z = (torch.arange(rows * 8, device=DEV).view(rows, 8) * 2654435761 % 1009).float() / 128
    tokens = torch.arange(rows, device=DEV) % 8
    logp, entropy, lse, ids, best = step.token_logprobs(z, tokens, 1.0, 2)
    q = torch.log_softmax(z.double(), 1)
    # 8 terms: a dozen roundings of values below 8 + log 8
    assert float((logp - q.gather(1, tokens[:, None])[:, 0]).abs().max()) < 12 * 16 * F32
    assert float((entropy + (q.exp() * q).sum(1)).abs().max()) < 24 * 16 * F32
    assert torch.equal(ids[:, 0].long(), z.argmax(1)) or float((best[:, 0] - q.amax(1)).abs().max()) < 12 * 16 * F32
    got = step.token_logprobs_grad(torch.ones(rows, device=DEV), None, z, tokens, lse, entropy)
    want = -q.exp()
    want.scatter_add_(1, tokens[:, None], torch.ones(rows, 1, device=DEV, dtype=torch.float64))
    assert float((got - want).abs().max()) < 24 * 16 * F32


def test_logits_beyond_32_bits():
    rows, v = 34000, 65536                                        # 2.2 G values
    z = torch.zeros(rows, v, dtype=torch.bfloat16, device=DEV)
    z[:, 65000] = 30.0
    tokens = torch.full((rows,), 65000, device=DEV)
    logp, entropy, lse, ids, _ = step.token_logprobs(z, tokens, 1.0, 1)
    assert (ids == 65000).all() and float((lse - 30).abs().max()) < 1e-5
    d = step.token_logprobs_grad(torch.ones(rows, device=DEV), None, z, tokens, lse, entropy)
    assert float(d[:, 64000:66000].abs().max()) < 1e-6 and (d[::1000, 5] == d[0, 5]).all()
