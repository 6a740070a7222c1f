"""AdamW over many tensors at once against its formulas in 64 bits, with states in 32 and in 8 bits."""
import pytest
import torch

from paper_2605_04478_amd import step
from tests.step_check import F32, close, rounding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BLOCK = 256
M, V = torch.float8_e4m3fn, torch.float8_e5m2
MOST = {"m": 448.0, "v": 57344.0}
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-7, weight_decay=0.1, scale=0.25, seed=3)


def _mix(x):
    x = (x ^ (x >> 16)) * 0x9E3779B1 & 0xFFFFFFFF
    x = (x ^ (x >> 15)) * 0xBB67AE85 & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(seed, count, i):
    """The bits that round element i (int64 tensor) at this step."""
    key = _mix(seed & 0xFFFFFFFF)
    for word in (seed >> 32 & 0xFFFFFFFF, count & 0xFFFFFFFF, count >> 32):
        key = _mix(key ^ word)
    return _mix((_mix(key ^ (i >> 32)) + i) & 0xFFFFFFFF)


def _decoded(state, name):
    x = state[name].double().cpu()
    return x if state["m"].dtype == torch.float32 else (x.view(-1, BLOCK) * state[name + "_scale"].double().cpu()[:, None]).view(-1)


def _starts(params):
    at = 0
    for p in params:
        yield at
        at += -(-p.numel() // BLOCK) * BLOCK


def _check_step(params, grads, state, hyper=HYPER, scale=None):
    """Takes a step and compares every output with the formulas, each by the roundings that lead to it."""
    before = {n: t.clone() for n, t in state.items()}
    old = [p.detach().double().cpu() for p in params]
    step.adamw(params, grads, state, **{**hyper, **({} if scale is None else {"scale": scale})})
    t = int(before["count"]) + 1
    assert int(state["count"]) == t
    (b1, b2), lr, eps = hyper["betas"], hyper["lr"], hyper["eps"]
    s = float(scale) if scale is not None else hyper["scale"]
    bits8 = state["m"].dtype == M
    om, ov = _decoded(before, "m"), _decoded(before, "v")
    if bits8:
        nm, nv = _decoded(state, "m"), _decoded(state, "v")
    for p, g, o, at in zip(params, grads, old, _starts(params)):
        n, end = p.numel(), at + -(-p.numel() // BLOCK) * BLOCK
        if g is None:
            assert torch.equal(p.detach().double().cpu(), o)
            assert all(torch.equal(state[k][at:end].view(torch.uint8), before[k][at:end].view(torch.uint8)) for k in ("m", "v"))
            continue
        g = torch.cat([g.double().cpu().reshape(-1) * s, torch.zeros(end - at - n, dtype=torch.float64)])
        m0, v0 = om[at:end], ov[at:end]
        m, v = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
        # (decoding rounds once)
        em, ev = F32 * (4 * (b1 * m0).abs() + 5 * ((1 - b1) * g).abs() + m.abs()) + 2.0 ** -140, F32 * (4 * b2 * v0 + 8 * (1 - b2) * g * g + v) + 2.0 ** -140
        den = (v / (1 - b2 ** t)).sqrt() + eps
        ratio = m / (1 - b1 ** t) / den
        # the root halves v's relative error; root, its factor, their product, the sum with eps, the quotient and the step's factor round once or twice each
        er = em / (1 - b1 ** t) / den + ratio.abs() * (ev / (2 * v).clamp(min=1e-300) + 16 * F32)
        if state.get("master") is not None:
            x = before["master"][at:at + n].double().cpu()
        else:
            x = o.reshape(-1)
        want = x - lr * hyper["weight_decay"] * x - lr * ratio[:n]
        bound = F32 * (3 * x.abs() + want.abs()) + lr * (er + 4 * F32 * ratio.abs())[:n]
        if state.get("master") is not None:
            close(state["master"][at:at + n], want, bound)
            assert not state["master"][at + n:end].any()
            assert torch.equal(p.detach().reshape(-1), state["master"][at:at + n].to(p.dtype))
        else:
            close(p.detach().reshape(-1), want, bound + rounding(want, p.dtype))
        if not bits8:
            close(state["m"][at:end], m, em)
            close(state["v"][at:end], v, ev)
            continue
        i = torch.arange(at, end)
        random = _random(hyper["seed"], t, i)
        for name, x, e, r, form, least in (("m", m, em, random & 0xFFFF, M, 0.0), ("v", v, ev, random >> 16, V, 2.0 ** -16)):
            largest = x.abs().view(-1, BLOCK).amax(1)
            scale_64 = largest.clamp(min=2.0 ** -80) / MOST[name]
            got = state[name + "_scale"][at // BLOCK:end // BLOCK]
            close(got, scale_64, F32 * 3 * scale_64 + e.view(-1, BLOCK).amax(1) / MOST[name])
            per = scale_64[:, None].expand(-1, BLOCK).reshape(-1)
            q, eq = x.abs() / per, 2 * e / per + 8 * F32 * x.abs() / per + 2.0 ** -30
            every = torch.arange(127 if form == M else 124, dtype=torch.uint8).view(form).double()
            low = (torch.searchsorted(every, q, right=True) - 1).clamp(0, every.numel() - 2)
            unit = every[low + 1] - every[low]
            sure = (q - every[low]) / unit + (r.double() + 0.5) / 65536
            slack = 2 * eq / unit + 2.0 ** -18
            code = state[name][at:end].float().double().cpu().abs()
            up, down = every[low + 1], every[low].clamp(min=least)
            down = torch.where(x == 0, torch.zeros_like(down), down)
            fits = torch.where(sure >= 1 + slack, code == up, torch.where(sure <= 1 - slack, code == down, (code == up) | (code == down)))
            # (next to one of the format's values the neighbour below may be the one that is meant)
            near = ((q - every[low]) <= eq) | ((every[low + 1] - q) <= eq)
            fits |= near & ((code == every[low]) | (code == every[(low - 1).clamp(min=0)]) | (code == up) | (code == every[(low + 2).clamp(max=every.numel() - 1)]))
            assert bool(fits.all()), (name, int((~fits).sum()), q[~fits][:3], code[~fits][:3], sure[~fits][:3])
            if t == 1:          # (later steps whose gradient is next to nothing scale values that were the format's)
                assert int((near & (q > 0) & (q < MOST[name] * 0.999)).sum()) <= 0.1 * q.numel()
            sign = torch.signbit(state[name][at:end].float().cpu())
            assert torch.equal(sign & (code > 0), (x < 0) & (code > 0))


def _tensors(sizes, dtype, grad_dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda size, std: std * torch.randn(size, device=DEV, generator=g)
    params = [n(s, 0.1).to(dtype) for s in sizes]
    return params, lambda: [(n(s, 1.0) * 10.0 ** float(torch.randint(-4, 1, (1,), generator=g, device=DEV))).to(grad_dtype or dtype) for s in sizes]


KINDS = [(torch.bfloat16, None, False), (torch.bfloat16, torch.float32, True), (torch.float16, None, True), (torch.float16, torch.float32, False), (torch.float32, None, False)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grad_dtype,masters", KINDS, ids=str)
def test_steps(dtype, grad_dtype, masters, bits):
    sizes = [(1,), (255,), (16, 16), (257,), (0,), (3, 7, 11), (4096,), (4097,), (100, 123), (8191,), (2,)]
    params, draw = _tensors(sizes, dtype, grad_dtype)
    state = step.adamw_state(params, bits, masters)
    for _ in range(3):
        _check_step(params, draw(), state)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 63, 64, 65, 112, 113, 300])
def test_many_tensors(count, bits):
    sizes = [((i * 37) % 700,) for i in range(count)]
    params, draw = _tensors(sizes, torch.bfloat16, None, seed=count)
    state = step.adamw_state(params, bits)
    grads = draw()
    grads[count // 2] = None
    _check_step(params, grads, state)


@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_at_odd_addresses(bits):
    base, grad = torch.randn(5000, device=DEV).bfloat16(), torch.randn(5000, device=DEV).bfloat16()
    params, grads = [base[1:1100], base[1101:3003], base[3004:3005]], [grad[3:1102], grad[1500:3402], grad[7:8]]
    rest = base[[0, 1100, 3003]].clone()
    state = step.adamw_state(params, bits)
    _check_step(params, grads, state)
    assert torch.equal(base[[0, 1100, 3003]], rest)


def test_scale_on_the_device_and_other_gradient_layouts():
    params, draw = _tensors([(40, 50), (300,)], torch.float32, None)
    state, grads = step.adamw_state(params), draw()
    _check_step(params, [grads[0].t().contiguous().t(), torch.stack([grads[1]] * 2, -1)[..., 0]], state, scale=torch.full((), 0.125, device=DEV))
    _check_step(params, [torch.ones(1, 1, device=DEV).expand(40, 50), torch.complex(grads[1], -grads[1]).conj().imag], state, scale=torch.full((1,), 2.0, device=DEV))


def test_zeros_stay_zeros_and_v_does_not_become_zero():
    p = torch.zeros(512, device=DEV)
    g = torch.zeros(512, device=DEV)
    g[0], g[1], g[300] = 1.0, 1e-9, -1e-30
    state = step.adamw_state([p], 8)
    for _ in range(20):
        step.adamw([p], [g], state, 1e-3, weight_decay=0.0)
    v = state["v"].float()
    assert v[0] > 0 and v[1] > 0 and not v[2:256].any() and not p[2:256].any() and not state["m"].float()[2:256].any()
    # a gradient whose square 32 bits do not have
    assert not v[301:].any() and torch.isfinite(p).all()


def test_without_eps():
    """Gradients whose squares are subnormal in 32 bits still step by lr."""
    g = torch.tensor([1e-3, -1e-18, 3e-19, 5.0, 1e10], device=DEV)
    p = torch.zeros(5, device=DEV)
    state = step.adamw_state([p])
    step.adamw([p], [g], state, 0.5, betas=(0.9, 0.5), eps=0.0)
    # v = 0.5 g^2 of 1e-37 has 23 bits, of 4.5e-38 too; m / sqrt(v) / (0.1 / sqrt(0.5)) is 1 to 2^-17 where v's spacing, 2^-149, is 2^-17 of it
    assert float((p + 0.5 * torch.sign(g)).abs().max()) < 0.5 * 2.0 ** -16
    tiny = torch.full((300,), 1e-20, device=DEV)
    p, state = torch.zeros(300, device=DEV), None
    state = step.adamw_state([p])
    step.adamw([p], [tiny], state, 0.5, betas=(0.9, 0.5), eps=0.0)          # v is 5e-41: 35,682 of its spacings
    assert float((p + 0.5).abs().max()) < 0.5 * 2.0 ** -14


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_gradients_that_are_not_finite(bad):
    for bits in (32, 8):
        params = [torch.ones(600, device=DEV), torch.ones(100, device=DEV)]
        grads = [torch.full((600,), 0.5, device=DEV), torch.full((100,), 0.5, device=DEV)]
        grads[0][300] = bad
        state = step.adamw_state(params, bits)
        step.adamw(params, grads, state, 1e-3)
        first = [p.clone() for p in params]
        grads[0][300] = 0.5
        step.adamw(params, grads, state, 1e-3)
        nan = torch.isnan(params[0])
        mine = torch.zeros_like(nan)
        mine[256:512 if bits == 8 else 0] = True
        mine[300] = True
        assert torch.equal(nan, mine) and not torch.isnan(params[1]).any(), bits
        assert not torch.isnan(first[0][torch.arange(600, device=DEV) != 300]).any()


def test_rounding_keeps_the_mean():
    """The first step's m is 0.1 g: what rounding adds is between -1 and 1 units of the format, zero on average; the mean of N such values is off by
    more than 6 times 0.5 / sqrt(N) once in 10^8."""
    n = 1 << 20
    g = torch.rand(n, device=DEV) + 0.5
    p = torch.zeros(n, device=DEV)
    for seed in (0, 1, (5 << 40) + 9):
        state = step.adamw_state([p], 8)
        step.adamw([p], [g], state, 1e-3, seed=seed)
        for name, want in (("m", (0.1 * g.double())), ("v", 0.001 * g.double() ** 2)):
            got = state[name].double().view(-1, BLOCK) * state[name + "_scale"].double()[:, None]
            scale = state[name + "_scale"].double()[:, None].expand(-1, BLOCK).reshape(-1)
            unit = torch.ldexp(torch.ones_like(scale), torch.frexp(want / scale).exponent - 1 - (3 if name == "m" else 2)) * scale
            off = (got.view(-1) - want.cuda()) / unit
            assert float(off.abs().max()) < 1.001 and abs(float(off.mean())) < 3 / n ** 0.5, (name, seed)
            # neighbours' roundings have nothing to do with one another
            assert abs(float((off[1:] * off[:-1]).mean())) < 6 * 0.25 / n ** 0.5
            if name == "m":
                first = off
            else:
                assert abs(float((off * first).mean())) < 6 * 0.25 / n ** 0.5


def test_eight_bits_follow_a_constant_gradient():
    """v of a constant gradient is (1 - b2^t) g^2.  Each of 8,192 elements walks at random around it: a step of its two bits of mantissa is a quarter of v at most,
    taken with odds of (1 - b2) / 0.125 at most each step and decaying with b2, so its variance is v^2 0.25 / 2 at most; the mean is off by 6 sigma
    of 0.36 / sqrt(8192) = 0.024 once in 10^8."""
    n, steps = 8192, 1500
    g, p = torch.full((n,), 0.7, device=DEV), torch.zeros(n, device=DEV)
    state = step.adamw_state([p], 8)
    for _ in range(steps):
        step.adamw([p], [g], state, 1e-4, betas=(0.9, 0.999))
    v, m = _decoded(state, "v"), _decoded(state, "m")
    want = 0.49 * (1 - 0.999 ** steps)
    assert abs(float(v.mean()) / want - 1) < 0.024
    # m's three bits: an eighth of m, decaying ten times a hundred faster
    assert abs(float(m.mean()) / 0.7 - 1) < 6 * 0.25 / n ** 0.5


def test_class_and_its_state():
    torch.manual_seed(0)
    model = [torch.nn.Parameter(torch.randn(30, 20, device=DEV)), torch.nn.Parameter(torch.randn(20, device=DEV))]
    twin = [torch.nn.Parameter(p.detach().clone()) for p in model]
    a, b = step.AdamW(model, 1e-2, weight_decay=0.1), torch.optim.AdamW(twin, 1e-2, weight_decay=0.1)
    x = torch.randn(50, 30, device=DEV)
    for _ in range(5):
        for params in (model, twin):
            for p in params:
                p.grad = None
            (torch.tanh(x @ params[0]) @ params[1]).square().mean().backward()
        a.step()
        b.step()
    # steps of 0.01, each by a ratio that 32 bits hold to 2^-18 where neither moment is next to zero
    for p, q in zip(model, twin):
        assert float((p - q).detach().abs().max()) < 5 * 1e-2 * 2.0 ** -10
    kept = a.state_dict()
    saved = [p.detach().clone() for p in model]
    a.step()
    after = [p.detach().clone() for p in model]
    with torch.no_grad():
        for p, s in zip(model, saved):
            p.copy_(s)
    a.load_state_dict(kept)
    a.step()
    assert all(torch.equal(p, q) for p, q in zip(model, after))
    with pytest.raises(ValueError, match="the state has"):
        a.load_state_dict({"m": kept["m"]})


def test_a_saved_parameter_is_known_to_have_changed():
    for native in (True, False):
        p = torch.ones(10, device=DEV, requires_grad=True)
        y = (p * p).sum()
        g = torch.ones(10, device=DEV)
        step.adamw([p], [g if native else torch.stack([g, g], -1)[..., 0]], step.adamw_state([p]), 1e-3)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def test_parameters_of_inference_mode():
    with torch.inference_mode():
        p, g = torch.ones(10, device=DEV), torch.ones(10, device=DEV)
        for grad in (g, torch.stack([g, g], -1)[..., 0]):
            state = step.adamw_state([p])
            step.adamw([p], [grad], state, 0.5)
        # two first steps of 0.5, each by a ratio of 1 that passes 16 roundings of 2^-24 (and eps, 2^-26): off by 2 (0.5 (16 + 1) + 1) 2^-24 < 2^-19
        assert float(p.abs().max()) < 2.0 ** -19


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_and_replayed(bits):
    make = lambda: _tensors([(3000,), (77, 13), (5,)], torch.bfloat16, None, seed=4)
    (params, draw), (twin, _) = make(), make()
    grads = draw()
    state, other = step.adamw_state(params, bits, True), step.adamw_state(twin, bits, True)
    by = torch.ones(1, device=DEV)
    run = lambda p, s: step.adamw(p, grads, s, 1e-2, weight_decay=0.01, scale=by, seed=5)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run(params, state)
    side.synchronize()
    run(twin, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(params, state)
    for k in range(4):
        for g, new in zip(grads, draw()):
            g.copy_(new)
        by.fill_(0.5 + k)
        torch.cuda.synchronize()
        graph.replay()
        run(twin, other)
        torch.cuda.synchronize()
        assert int(state["count"]) == k + 2
        assert all(torch.equal(a, b) for a, b in zip(params, twin)) and all(torch.equal(state[n].view(torch.uint8), other[n].view(torch.uint8)) for n in state)


def test_native_code_and_python_do_the_same(monkeypatch):
    class Declines:
        def __getattr__(self, _):
            return lambda *a: None
    outs = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(step, "_calls", Declines())
        params, draw = _tensors([(700,), (3, 5), (0,), (129,)], torch.float16, torch.float32, seed=6)
        state, grads = step.adamw_state(params, 8, True), draw()
        grads[1] = None
        if native:
            assert step._native().adamw(params, grads, state, 1e-3, (0.9, 0.99), 1e-8, 0.1, 1.0, 5) is True
        else:
            step.adamw(params, grads, state, 1e-3, (0.9, 0.99), 1e-8, 0.1, 1.0, 5)
        outs.append([*params, *(state[n].view(torch.uint8) for n in sorted(state))])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_native_code_declines_what_is_out_of_the_ordinary():
    p, g = torch.ones(300, device=DEV), torch.ones(300, device=DEV)
    state = step.adamw_state([p])
    args = lambda **c: [c.get("params", [p]), c.get("grads", [g]), c.get("state", state), 1e-3, c.get("betas", (0.9, 0.99)), 1e-8, 0.1, c.get("scale", 1.0), 0]
    call = step._native().adamw
    assert call(*args()) is True
    for change in (dict(params=[p.cpu()]), dict(params=[p.double()]), dict(params=[p, p], grads=[g, g]), dict(params=[p, p[10:20]], grads=[g, g[:10]]), dict(params=[p[::2]], grads=[g[::2]]),
                   dict(grads=[]), dict(grads=[g[:4]]), dict(grads=[g.cpu()]), dict(grads=[g.half()]), dict(state={}), dict(state={**state, "v": state["v"][:256]}),
                   dict(state={**state, "count": state["count"].int()}), dict(state={**state, "m": state["m"].to(M)}), dict(state={**state, "master": state["m"]}), dict(betas=(1.0, 0.9)),
                   dict(betas=(0.9,)), dict(scale=torch.ones(2, device=DEV)), dict(scale=torch.ones(1)), dict(scale=float("inf")), dict(params=None)):
        assert call(*args(**change)) is None, change
    assert int(state["count"]) == 1


def test_states_beyond_32_bits():
    """A tensor whose last elements' places do not fit 32 bits, and one behind it."""
    n = (1 << 32) + 1000
    params = [torch.zeros(n, dtype=torch.bfloat16, device=DEV), torch.zeros(300, dtype=torch.bfloat16, device=DEV)]
    grads = [torch.ones(n, dtype=torch.bfloat16, device=DEV), torch.ones(300, dtype=torch.bfloat16, device=DEV)]
    state = step.adamw_state(params, 8)
    step.adamw(params, grads, state, 0.5, weight_decay=0.0)
    # m = 0.1, v = 0.001: one step of lr
    for x in (params[0][:9], params[0][n // 2:n // 2 + 9], params[0][-1001:], params[1]):
        assert (x == -0.5).all()
    m = state["m"].view(torch.uint8)
    assert (m[[0, 1 << 31, n - 1, -1024, -725]] == 0x7E).all() and not m[n:-512].any() and not m[-212:].any()
