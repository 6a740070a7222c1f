"""The choice of experts, and tokens sorted by expert and back, against plain computations in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2605_04478_amd import step
from tests.step_check import F32, close, rounding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _chosen(scores, k):
    """Experts by score, equal ones by number; those of -inf and NaN are none."""
    z = np.nan_to_num(scores.double().cpu().numpy(), nan=-INF, posinf=INF, neginf=-INF)
    order = np.argsort(-z, axis=1, kind="stable")[:, :k]
    return np.where(np.take_along_axis(z, order, 1) > -INF, order, -1)


def _weights(z, experts, over_all):
    """In 64 bits: weights of the chosen, and the softmax that they are part of."""
    z = torch.where(torch.isnan(z), torch.full_like(z, -INF), z)
    there = experts >= 0
    if not over_all:
        mask = torch.zeros(z.shape[0], z.shape[1] + 1, dtype=torch.bool).scatter_(1, torch.where(there, experts, z.shape[1]), True)[:, :-1]
        z = torch.where(mask, z, torch.full_like(z, -INF))
    m = z.amax(1, keepdim=True)
    e = torch.where(z == m, torch.ones_like(z), torch.exp(z - m))
    e = torch.where(m > -INF, e, torch.zeros_like(e))
    p = e / e.sum(1, keepdim=True).clamp(min=1)
    return torch.where(there, p.gather(1, experts.clamp(min=0)), torch.zeros(())), p


def _relative(z, experts):
    """Relative error of a weight: the difference to the largest score is off by 2^-24 of itself and expf by two steps; of the sum each term likewise, which
    makes at most 1/e of a term, and as many additions as there are terms; a division."""
    z = torch.where(torch.isfinite(z), z, torch.zeros_like(z))
    far = (z.amax(1, keepdim=True) - z).gather(1, experts.clamp(min=0))
    return F32 * (far + 2 * z.shape[1] + 16)


@pytest.mark.parametrize("over_all", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tokens,n,k", [(1, 1, 1), (3, 2, 2), (5, 8, 2), (257, 63, 6), (64, 64, 64), (33, 65, 4), (130, 128, 8), (9, 200, 7), (70, 256, 8), (1000, 500, 10),
                                        (17, 1000, 16), (6, 1024, 64)])
def test_route(tokens, n, k, dtype, over_all):
    g = torch.Generator(device=DEV).manual_seed(tokens + n)
    z = (2 * torch.randn(tokens, n, device=DEV, generator=g)).to(dtype)
    z[:, ::3] = z[:, ::3].round()                              # ties
    z[torch.rand(tokens, n, device=DEV, generator=g) < 0.1] = -INF
    z[0, n // 2] = float("nan")
    z[-1] = -INF                                               # a row of nothing
    experts, weights = step.route(z, k, over_all)
    assert experts.dtype == torch.int32 and weights.dtype == torch.float32
    want = _chosen(z, k)
    assert np.array_equal(experts.cpu().numpy(), want)
    wide, at = z.double().cpu(), torch.from_numpy(want)
    w, p = _weights(wide, at, over_all)
    rel = _relative(wide, at)
    close(weights, w, rel * w + 2.0 ** -149)
    dw = torch.randn(tokens, k, device=DEV, generator=g)
    dw[experts < 0] = float("nan")                             # does not matter
    dz = step.route_grad(dw, z, experts, weights, over_all)
    d = torch.where(at >= 0, dw.double().cpu(), torch.zeros(()))
    each = w * d
    full = torch.zeros(tokens, n + 1, dtype=torch.float64).scatter_add_(1, torch.where(at >= 0, at, n), each)[:, :-1]
    size = torch.zeros(tokens, n + 1, dtype=torch.float64).scatter_add_(1, torch.where(at >= 0, at, n), each.abs())[:, :-1] + p * each.abs().sum(1, keepdim=True)
    wantd = full - p * each.sum(1, keepdim=True)
    assert dz.dtype == dtype
    # twice the relative error of p and w, k additions
    far = torch.where(p > 0, (wide - torch.where(p > 0, wide, torch.full_like(wide, -INF)).amax(1, keepdim=True)).abs(), torch.zeros(()))
    close(dz, wantd, size * F32 * 2 * (torch.nan_to_num(far, posinf=0.0) + 2 * n + k + 20) + 2.0 ** -140 + rounding(wantd, dtype))


def test_gradient_of_the_choice_against_differences():
    z = torch.tensor([[0.3, -1.0, 0.9, 0.1, -0.4]], device=DEV)
    dw = torch.tensor([[0.7, -1.3]], device=DEV)
    for over_all in (False, True):
        grad = step.route_grad(dw, z, *step.route(z, 2, over_all), over_all)
        for e in range(5):
            h = torch.zeros_like(z)
            h[0, e] = 2.0 ** -8
            up, down = ((step.route(z + s * h, 2, over_all)[1].double() * dw).sum() for s in (1, -1))
            # the third derivative is below 4, the weights are off by 2^-20 at most
            assert abs(float(up - down) * 2.0 ** 7 - float(grad[0, e])) < 4 * 2.0 ** -16 + 4 * 2.0 ** -20 * 2.0 ** 7


def test_infinite_scores_share_the_weight():
    z = torch.tensor([[1.0, INF, 2.0, INF], [INF, 0.0, 1.0, 2.0]], device=DEV)
    for over_all in (False, True):
        experts, weights = step.route(z, 3, over_all)
        assert experts.tolist() == [[1, 3, 2], [0, 3, 2]] and weights.tolist() == [[0.5, 0.5, 0.0], [1.0, 0.0, 0.0]]


def test_lowest_values_are_scores():
    low = torch.finfo(torch.bfloat16).min
    z = torch.full((2, 70), low, dtype=torch.bfloat16, device=DEV)
    z[1, 69] = 0
    experts, weights = step.route(z, 2)
    assert experts.tolist() == [[0, 1], [69, 0]] and weights.tolist() == [[0.5, 0.5], [1.0, 0.0]]


@pytest.mark.parametrize("bits", [torch.int32, torch.int64], ids=str)
@pytest.mark.parametrize("tokens,k,n", [(0, 2, 3), (1, 1, 1), (5, 4, 16), (63, 1, 7), (100, 3, 12), (1024, 1, 40), (1025, 1, 40), (4096, 1, 9), (4097, 1, 9), (2048, 4, 64), (8193, 1, 5), (3001, 3, 1024), (40000, 8, 128), (300001, 1, 256),
                                        (150000, 2, 2)])
def test_expert_order(tokens, k, n, bits):
    rng = np.random.default_rng(tokens + n)
    e = rng.integers(0, n, (tokens, k))
    e = np.where(rng.random((tokens, k)) < 0.6, e // 2, e)                      # uneven
    e = np.where(rng.random((tokens, k)) < 0.1, rng.choice([-1, n, -2 ** 31, 2 ** 31 - 1], (tokens, k)), e)
    places, offsets = step.expert_order(torch.from_numpy(e).to(bits).to(DEV), n)
    flat = e.reshape(-1)
    valid = (flat >= 0) & (flat < n)
    key = np.where(valid, flat, n)
    order = np.argsort(key, kind="stable")
    want = np.empty(tokens * k, dtype=np.int64)
    want[order] = np.arange(tokens * k)
    want[~valid] = -1
    assert places.dtype == offsets.dtype == torch.int32
    assert np.array_equal(offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(np.bincount(key, minlength=n + 1)[:n])]))
    assert np.array_equal(places.cpu().numpy().reshape(-1), want)


def test_entries_of_far_numbers_have_no_place():
    e = torch.tensor([[0, 1 << 32], [(1 << 32) + 1, 1]], device=DEV)
    places, offsets = step.expert_order(e, 2)
    assert places.tolist() == [[0, -1], [-1, 1]] and offsets.tolist() == [0, 1, 2]


def test_one_expert_takes_all():
    places, offsets = step.expert_order(torch.full((20000, 2), 3, device=DEV, dtype=torch.int32), 9)
    assert torch.equal(places.view(-1), torch.arange(40000, device=DEV, dtype=torch.int32)) and offsets.tolist() == [0] * 4 + [40000] * 6


def _both_ways(tokens, k, n, d, dtype, dropped, seed=0, spread=0):
    g = torch.Generator(device=DEV).manual_seed(seed + tokens + d)
    experts = torch.rand(tokens, max(n, k), device=DEV, generator=g).topk(k, dim=1).indices.to(torch.int32)
    experts[torch.rand(tokens, k, device=DEV, generator=g) < dropped] = -1
    matrix = lambda rows: torch.randn(rows, d + spread, device=DEV, generator=g).to(dtype)[:, :d]
    x, y, dout, drows = matrix(tokens), matrix(tokens * k), matrix(tokens), matrix(tokens * k)
    weights = torch.rand(tokens, k, device=DEV, generator=g)
    places, offsets = step.expert_order(experts, max(n, k))
    return places, offsets, x, y, dout, drows, weights


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tokens,k,n,d,dropped,spread", [(1, 1, 1, 1, 0, 0), (1, 4, 16, 2048, 0, 0), (3, 2, 4, 7, 0.5, 0), (5, 64, 64, 130, 0.2, 3), (40, 9, 12, 1001, 0.1, 0),
                                                         (33, 3, 8, 1024, 1.0, 0), (70, 8, 16, 4096, 0, 8), (9, 3, 4, 5003, 0.1, 1), (50, 3, 4, 1000, 0.1, 0), (50, 3, 4, 72, 0.1, 8), (4, 2, 3, 20011, 0, 0), (257, 2, 5, 515, 0.3, 1), (18000, 1, 4, 24, 0.05, 0)])
def test_dispatch_and_combine(tokens, k, n, d, dropped, spread, dtype):
    places, offsets, x, y, dout, drows, weights = _both_ways(tokens, k, n, d, dtype, dropped, spread=spread)
    used, at = int(offsets[-1]), places.long().cpu()
    there = at >= 0
    xs, ys, ws = x.double().cpu(), y.double().cpu(), weights.double().cpu()
    rows = step.dispatch(x, places, offsets)
    want = torch.zeros(tokens * k, d, dtype=torch.float64)
    want[at[there]] = xs.repeat_interleave(k, 0)[there.view(-1)]
    assert rows.dtype == dtype and torch.equal(rows.double().cpu(), want) and not rows[used:].any()
    pick = lambda m: torch.where(there[..., None], m[at.clamp(min=0)], torch.zeros((), dtype=torch.float64))       # [tokens, k, d]
    terms = ws[..., None] * pick(ys)
    # k products, each rounded, and as many additions
    close(step.combine(y, places, weights), terms.sum(1), 2 * k * F32 * terms.abs().sum(1) + rounding(terms.sum(1), dtype))
    terms = pick(drows.double().cpu())
    close(step.dispatch_grad(drows, places), terms.sum(1), k * F32 * terms.abs().sum(1) + rounding(terms.sum(1), dtype))
    dy, dw = step.combine_grad(dout, y, places, weights, offsets)
    ds = dout.double().cpu()
    want = torch.zeros(tokens * k, d, dtype=torch.float64)
    want[at[there]] = (ws[..., None] * ds[:, None, :])[there]
    close(dy, want, F32 * want.abs() + rounding(want, dtype))
    assert not dy[used:].any()
    terms = ds[:, None, :] * pick(ys)
    # a thread adds d / 64 + 16 products at most, then 6 + 4 sums of threads
    close(dw, terms.sum(2), (d / 64 + 30) * F32 * terms.abs().sum(2) + 2.0 ** -140)
    same, none = step.combine_grad(dout, y, places, weights, offsets, False)
    assert none is None and torch.equal(same, dy)


def test_without_tokens():
    e = torch.zeros(0, 2, dtype=torch.int32, device=DEV)
    places, offsets = step.expert_order(e, 3)
    x, w = torch.zeros(0, 8, device=DEV), torch.zeros(0, 2, device=DEV)
    assert offsets.tolist() == [0] * 4 and step.dispatch(x, places, offsets).shape == (0, 8) and step.combine(x, places, w).shape == (0, 8)
    dy, dw = step.combine_grad(x, x, places, w, offsets)
    assert dy.shape == (0, 8) and dw.shape == (0, 2) and step.dispatch_grad(x, places).shape == (0, 8)
    experts, weights = step.route(torch.zeros(0, 5, device=DEV), 2)
    assert experts.shape == weights.shape == (0, 2) and step.route_grad(weights, torch.zeros(0, 5, device=DEV), experts, weights).shape == (0, 5)


def test_places_outside_the_rows_are_not_followed():
    places = torch.tensor([[0, 1 << 30], [-5, 3]], dtype=torch.int32, device=DEV)
    offsets = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    x, y, w = torch.ones(2, 40, device=DEV), torch.arange(4.0, device=DEV)[:, None].expand(4, 40), torch.ones(2, 2, device=DEV)
    rows = step.dispatch(x, places, offsets)
    assert (rows[[0, 3]] == 1).all()
    assert step.combine(y, places, w)[:, 0].tolist() == [0.0, 3.0]
    assert step.combine_grad(x, y, places, w, offsets)[1].tolist() == [[0.0, 0.0], [0.0, 120.0]]
    # a number of used rows that is not one
    for used in (-7, 1 << 30):
        step.dispatch(x, places, torch.tensor([0, used], dtype=torch.int32, device=DEV))


def test_what_dropped_entries_hold_does_not_matter():
    places = torch.tensor([[0, -1]], dtype=torch.int32, device=DEV)
    y = torch.tensor([[2.0] * 33, [float("nan")] * 33], device=DEV)
    w = torch.tensor([[0.5, float("nan")]], device=DEV)
    assert (step.combine(y, places, w) == 1).all() and (step.dispatch_grad(y, places) == 2).all()
    dy, dw = step.combine_grad(torch.ones(1, 33, device=DEV), y, places, w, torch.tensor([0, 1], dtype=torch.int32, device=DEV))
    assert dy[0].tolist() == [0.5] * 33 and not dy[1].any() and dw.tolist() == [[66.0, 0.0]]


@pytest.mark.parametrize("over_all", [False, True])
def test_a_layer_of_experts_as_a_whole(over_all):
    """Choice, order, dispatch, product, combine and all gradients, in one step of automatic differentiation."""
    g = torch.Generator(device=DEV).manual_seed(5)
    t, d, n, k = 150, 64, 6, 3
    bf = torch.bfloat16
    leaf = lambda *shape, std=1.0: (std * torch.randn(shape, device=DEV, generator=g)).to(bf).requires_grad_()
    x, gate, w = leaf(t, d), leaf(n, d, std=0.2), leaf(n, d, d, std=d ** -0.5)
    dout = torch.randn(t, d, device=DEV, generator=g).to(bf)
    scores = x @ gate.t()
    experts, weights = step.Route.apply(scores, k, over_all)
    places, offsets = step.expert_order(experts, n)
    y = step.ExpertProduct.apply(step.Dispatch.apply(x, places, offsets), w, offsets)
    out = step.Combine.apply(y, places, weights, offsets)
    grads = torch.autograd.grad(out, (x, gate, w), dout)
    wide = [v.detach().double().cpu().requires_grad_() for v in (x, gate, w)]
    xs, gs, ws = wide
    at = experts.long().cpu()
    z = xs @ gs.t()
    p = torch.softmax(z, 1).gather(1, at) if over_all else torch.softmax(z.gather(1, at), 1)
    each = torch.stack([torch.stack([xs[i] @ ws[at[i, c]].t() for c in range(k)]) for i in range(t)])
    res = (p[..., None] * each).sum(1)
    want = torch.autograd.grad(res, wide, dout.double().cpu())
    # 8 roundings to 8 bits on the longest way, each at most half a step of what it is part of, in norm
    bound = 8 * 2.0 ** -8
    assert float((out.detach().double().cpu() - res.detach()).norm()) <= bound * float(res.detach().norm())
    for got, x64 in zip(grads, want):
        assert float((got.double().cpu() - x64).norm()) <= bound * float(x64.norm())


def test_captured_and_replayed():
    g = torch.Generator(device=DEV).manual_seed(9)
    t, d, n, k = 3000, 200, 16, 4
    z, x, dout = torch.randn(t, n, device=DEV, generator=g), torch.randn(t, d, device=DEV, generator=g), torch.randn(t, d, device=DEV, generator=g)

    def all_of_it():
        experts, weights = step.route(z, k)
        places, offsets = step.expert_order(experts, n)
        rows = step.dispatch(x, places, offsets)
        out = step.combine(rows, places, weights)
        dy, dw = step.combine_grad(dout, rows, places, weights, offsets)
        return [experts, weights, places, offsets, rows, out, dy, dw, step.dispatch_grad(dy, places), step.route_grad(dw, z, experts, weights)]
    all_of_it()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        all_of_it()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = all_of_it()
    for _ in range(3):
        z.copy_(torch.randn(t, n, device=DEV, generator=g))
        x.copy_(torch.randn(t, d, device=DEV, generator=g))
        want = all_of_it()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_views_and_other_layouts():
    g = torch.Generator(device=DEV).manual_seed(2)
    n = lambda *shape: torch.randn(shape, device=DEV, generator=g)
    z = n(20, 9)
    want = step.route(z, 3)
    for same in (z.t().contiguous().t(), torch.stack([z, z], -1)[..., 0], torch.cat([z, z], 1)[:, :9]):
        assert all(torch.equal(a, b) for a, b in zip(step.route(same, 3), want))
    lazily = torch.complex(z, -z).conj().imag
    assert lazily.is_neg() and torch.equal(step.route(lazily, 3)[0], want[0])
    experts, weights = want
    places, offsets = step.expert_order(experts, 9)
    apart = lambda m: torch.stack([m, m], -1)[..., 0]
    assert torch.equal(step.expert_order(apart(experts), 9)[0], places)
    x, y = n(20, 33), n(60, 33)
    base = step.dispatch(x, places, offsets), step.combine(y, places, weights), *step.combine_grad(x, y, places, weights, offsets), step.dispatch_grad(y, places)
    for f in (apart, lambda m: m.t().contiguous().t()):
        again = (step.dispatch(f(x), f(places), offsets), step.combine(f(y), f(places), f(weights)),
                 *step.combine_grad(f(x), f(y), f(places), f(weights), offsets), step.dispatch_grad(f(y), f(places)))
        assert all(torch.equal(a, b) for a, b in zip(again, base))
    one = torch.ones(33, device=DEV).expand(20, 33)                # the gradient of a sum
    assert torch.equal(step.combine_grad(one, y, places, weights, offsets)[0], step.combine_grad(one.contiguous(), y, places, weights, offsets)[0])
    dw = torch.ones(1, device=DEV).expand(20, 3)
    assert torch.equal(step.route_grad(dw, z, experts, weights), step.route_grad(dw.contiguous(), z, experts, weights))


def test_both_ways_of_calling_give_the_same(monkeypatch):
    g = torch.Generator(device=DEV).manual_seed(4)
    z = torch.randn(50, 20, device=DEV, generator=g)
    x, y = torch.randn(50, 40, device=DEV, generator=g), torch.randn(150, 40, device=DEV, generator=g)

    def calls():
        experts, weights = step.route(z, 3, True)
        places, offsets = step.expert_order(experts, 20)
        return [experts, weights, places, offsets, step.dispatch(x, places, offsets), step.combine(y, places, weights), step.dispatch_grad(y, places),
                *step.combine_grad(x, y, places, weights, offsets), step.route_grad(weights, z, experts, weights, True)]

    class Declines:
        def __getattr__(self, _):
            return lambda *a: None
    native = calls()
    e, w = native[:2]
    p, o = native[2:4]
    for name, args in dict(route=(z, 3, True), route_grad=(w, z, e, w, True), expert_order=(e, 20), dispatch=(x, p, o), dispatch_grad=(y, p), combine=(y, p, w),
                           combine_grad=(x, y, p, w, o, True)).items():
        assert getattr(step._native(), name)(*args) is not None, name            # ordinary tensors are native code's
        for i, a in enumerate(args):
            for wrong in ((a.cpu(), a[None], a.double(), 1.5) if isinstance(a, torch.Tensor) else ("x", 1.5, None)):
                assert getattr(step._native(), name)(*args[:i], wrong, *args[i + 1:]) is None, (name, i)
    monkeypatch.setattr(step, "_calls", Declines())
    assert all(torch.equal(a, b) for a, b in zip(native, calls()))


@pytest.mark.parametrize("n", [10, 200])
def test_more_tokens_than_workgroups(n):
    """300,001 tokens: every workgroup takes several."""
    t, k = 300001, 3
    z = (torch.arange(t, device=DEV)[:, None] * 7919 + torch.arange(n, device=DEV) * 104729) % 8191 / 1024.0
    experts, weights = step.route(z, k)
    top, want = z.sort(dim=1, descending=True, stable=True)
    assert torch.equal(experts.long(), want[:, :k])
    w = torch.softmax(top[:, :k].double(), 1)
    assert float((weights - w).abs().max()) < 64 * F32               # differences below 8, three terms
    dw = torch.randn(t, k, device=DEV)
    each = w * dw
    full = torch.zeros(t, n, device=DEV, dtype=torch.float64).scatter_(1, want[:, :k], each - w * each.sum(1, keepdim=True))
    assert float((step.route_grad(dw, z, experts, weights) - full).abs().max()) < 256 * F32 * float(dw.abs().max())


@pytest.mark.parametrize("d", [20, 520])
def test_more_rows_than_workgroups(d):
    """70,001 tokens of whole numbers, whose sums are exact."""
    t, k, n = 70001, 2, 7
    experts = (torch.arange(t * k, device=DEV) * 48271 % (n + 1)).view(t, k).int()          # n: dropped
    places, offsets = step.expert_order(experts, n)
    used, there, at = int(offsets[-1]), places >= 0, places.long().clamp(min=0)
    number = lambda rows: (torch.arange(rows, device=DEV)[:, None] * 31 + torch.arange(d, device=DEV) * 17) % 61 - 30.0
    x, y, w = number(t), number(t * k), (torch.arange(t * k, device=DEV).view(t, k) % 5).float()
    rows = step.dispatch(x, places, offsets)
    want = torch.zeros_like(rows)
    want[at[there]] = x.repeat_interleave(k, 0)[there.view(-1)]
    assert torch.equal(rows, want) and not rows[used:].any()
    keep = there[..., None]
    assert torch.equal(step.combine(y, places, w), (torch.where(keep, y[at], 0.0) * w[..., None]).sum(1))
    assert torch.equal(step.dispatch_grad(y, places), torch.where(keep, y[at], 0.0).sum(1))
    dy, dw = step.combine_grad(x, y, places, w, offsets)
    want[at[there]] = (x[:, None, :] * w[..., None])[there]
    assert torch.equal(dy, want) and torch.equal(dw, (torch.where(keep, y[at], 0.0) * x[:, None, :]).sum(2))


def test_rows_beyond_32_bits():
    """Rows whose elements lie beyond 2^31 of the first."""
    t, d = 70000, 32768                                     # 2.3 G values
    places, offsets = step.expert_order((torch.arange(t, device=DEV, dtype=torch.int32) * 7919 % 5)[:, None], 5)
    x = (torch.arange(t, device=DEV)[:, None] % 251).to(torch.bfloat16).expand(t, d).contiguous()
    rows = step.dispatch(x, places, offsets)
    assert torch.equal(rows[places[:, 0].long(), ::4001], x[:, ::4001])
    assert torch.equal(step.combine(rows, places, torch.ones(t, 1, device=DEV)), x)
