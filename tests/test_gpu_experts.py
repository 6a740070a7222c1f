"""Products grouped by expert and their gradients against products in 64 bits."""
import pytest
import torch

from tests.step_check import F32, close, rounding

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16
DEV = "cuda:0"


def _inputs(rows, offsets, k, n, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    e = len(offsets) - 1
    x = torch.randn(rows, k, generator=g).to(dtype)
    w = (torch.randn(e, n, k, generator=g) * k ** -0.5).to(dtype)
    dy = torch.randn(rows, n, generator=g).to(dtype)
    return x, w, dy


def _want(x, w, dy, offsets):
    """Results, and of each the sum of its products' magnitudes."""
    xd, wd, dyd = x.double(), w.double(), dy.double()
    out = [torch.zeros(x.shape[0], w.shape[1]).double(), torch.zeros_like(xd), torch.zeros_like(wd)]
    size = [torch.zeros_like(t) for t in out]
    for e, (a, b) in enumerate(zip(offsets, offsets[1:])):
        for o, f in ((out, lambda t: t), (size, torch.abs)):
            o[0][a:b] = f(xd[a:b]) @ f(wd[e]).t()
            o[1][a:b] = f(dyd[a:b]) @ f(wd[e])
            o[2][e] = f(dyd[a:b]).t() @ f(xd[a:b])
    return out, size


def _compare(got, want, size, terms, dtype, what):
    # every product is exact in 32 bits; each of the additions rounds once, by at most a step of the sum of magnitudes (matrix
    # instructions may cut instead of rounding to nearest: a whole step), and the result once more
    close(got, want, rounding(want, dtype) + 2 * F32 * (terms + 8) * size, what)


def _check(x, w, dy, offsets, bits=32, dev=lambda t: t.to(DEV)):
    from paper_2605_04478_amd import step
    want, size = _want(x, w, dy, offsets)
    off = torch.tensor(offsets, dtype=torch.int32 if bits == 32 else torch.int64, device=DEV)
    gx, gw, gdy = dev(x), dev(w), dev(dy)
    y = step.expert_product(gx, gw, off)
    dx, dw = step.expert_product_grad(gdy, gx, gw, off)
    longest = max(b - a for a, b in zip(offsets, offsets[1:]))
    for name, got, i, terms in (("y", y, 0, w.shape[2]), ("dx", dx, 1, w.shape[1]), ("dw", dw, 2, longest)):
        assert got.dtype == w.dtype and got.is_contiguous()
        _compare(got, want[i], size[i], terms, w.dtype, name)
    return y, dx, dw


CASES = [
    # rows, offsets, k, n
    (0, [0, 0, 0], 64, 64),
    (1, [0, 0, 1], 64, 128),
    (1, [0, 1], 8, 8),
    (5, [0, 0, 5, 5], 72, 136),
    (37, [0, 1, 1, 20, 37], 128, 256),
    (64, [0, 64], 64, 64),
    (130, [0, 129, 130], 200, 392),
    (300, [0, 33, 33, 33, 290, 300], 264, 120),
    (1023, [0, 1023], 512, 264),                       # one expert: its rows in several parts
    (1500, [0, 700, 1500], 320, 640),
    (2050, [0, 1025, 2050], 256, 512),                 # the largest tiles
    (40, [0, 40], 4096, 64),                           # a long contraction with few tiles: in several parts
    (200, sorted([0] + [(i * 37) % 201 for i in range(150)] + [200]), 64, 72),   # more experts than a wavefront has lanes
]


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,offsets,k,n", CASES, ids=lambda v: str(v) if isinstance(v, int) else f"e{len(v) - 1}")
def test_against_64_bits(rows, offsets, k, n, dtype):
    _check(*_inputs(rows, offsets, k, n, dtype), offsets)


@pytest.mark.parametrize("k,n", [(1, 1), (63, 65), (100, 7), (129, 64), (64, 129), (1001, 40)])
@pytest.mark.parametrize("rows,offsets", [(3, [0, 3]), (150, [0, 20, 20, 150]), (1300, [0, 1290, 1300])], ids=["few", "some", "many"])
def test_odd_sizes(rows, offsets, k, n):
    """Rows that do not start on 16 bytes take the path that loads single values."""
    _check(*_inputs(rows, offsets, k, n, BF), offsets, bits=64)


def test_strides_and_orders():
    offsets = [0, 50, 120]
    x, w, dy = _inputs(120, offsets, 96, 80, BF)

    def padded(t):              # every row followed by something else
        big = torch.full(t.shape[:-1] + (t.shape[-1] + 24,), float("nan"), dtype=t.dtype, device=DEV)
        big[..., :t.shape[-1]] = t.to(DEV)
        return big[..., :t.shape[-1]]

    def transposed(t):
        return t.to(DEV).transpose(-1, -2).contiguous().transpose(-1, -2)

    def shifted(t):             # aligned to 2 bytes only
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        flat[1:] = t.to(DEV).flatten()
        return flat[1:].view(t.shape)

    plain = _check(x, w, dy, offsets)
    for dev in (padded, transposed, shifted):
        for a, b in zip(_check(x, w, dy, offsets, dev=dev), plain):
            assert torch.equal(a, b)
    # a gradient that is one value everywhere, as that of a sum comes
    ones = torch.ones(1, 1, dtype=BF).expand(120, 80)
    _check(x, w, ones, offsets, dev=lambda t: t.to(DEV) if t is not ones else torch.ones(1, 1, dtype=BF, device=DEV).expand(120, 80))


@pytest.mark.parametrize("size", [64, 61], ids=["direct", "single"])
def test_rows_of_nobody(size):
    """Rows before the first and after the last expert's: zeros come out, and what they hold reaches nothing."""
    offsets = [9, 9, 40, 100]
    x, w, dy = _inputs(200, offsets, size, 72, BF)
    x[:9], x[100:] = float("nan"), float("inf")
    dy[:9], dy[100:] = float("inf"), float("nan")
    y, dx, dw = _check(x, w, dy, offsets)
    for t in (y, dx):
        assert not t[:9].any() and not t[100:].any()
    assert not dw[0].any()


def test_infinities_stay_with_their_rows():
    offsets = [0, 30, 70]
    x, w, dy = _inputs(70, offsets, 64, 64, BF)
    x[3, 5] = float("inf")
    dy[60, 2] = float("nan")
    from paper_2605_04478_amd import step
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    y = step.expert_product(x.to(DEV), w.to(DEV), off)
    dx, dw = step.expert_product_grad(dy.to(DEV), x.to(DEV), w.to(DEV), off)
    assert torch.isfinite(y[torch.arange(70) != 3]).all() and not torch.isfinite(y[3]).any()
    assert torch.isfinite(dx[torch.arange(70) != 60]).all() and torch.isnan(dx[60]).all()
    assert torch.isnan(dw[1, 2]).all() and torch.isfinite(dw[1][torch.arange(64) != 2]).all()
    assert not torch.isfinite(dw[0, :, 5]).any() and torch.isfinite(dw[0][:, torch.arange(64) != 5]).all()


@pytest.mark.parametrize("offsets", [[-5, 20, 50], [0, 20, 1000], [-1 << 30, 0, 1 << 30], [60, 70, 80]], ids=str)
def test_offsets_beyond_the_rows_are_clamped(offsets):
    x, w, dy = _inputs(50, offsets, 64, 64, BF)
    from paper_2605_04478_amd import step
    clamped = [min(max(o, 0), 50) for o in offsets]
    gx, gw, gdy = x.to(DEV), w.to(DEV), dy.to(DEV)
    res = []
    for o in (offsets, clamped):
        off = torch.tensor(o, dtype=torch.int32, device=DEV)
        res.append([step.expert_product(gx, gw, off), *step.expert_product_grad(gdy, gx, gw, off)])
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_weights_beyond_four_gigabytes():
    """Element offsets pass 32 bits: the last experts' weights start beyond 2^32 elements."""
    from paper_2605_04478_amd import step
    e, n, k = 36, 8192, 16384
    w = torch.empty(e, n, k, dtype=BF, device=DEV)
    assert w.numel() > 1 << 32
    g = torch.Generator(device=DEV).manual_seed(1)
    used = (0, 33, 35)
    for i in used:
        w[i].normal_(0, k ** -0.5, generator=g)
    x = torch.randn(6, k, device=DEV, generator=g).to(BF)
    counts = [2 if i in used else 0 for i in range(e)]
    off = torch.tensor([0] + counts, device=DEV).cumsum(0)
    y = step.expert_product(x, w, off)
    for i, u in enumerate(used):
        xs, ws = x[2 * i:2 * i + 2].double().cpu(), w[u].double().cpu()
        _compare(y[2 * i:2 * i + 2], xs @ ws.t(), xs.abs() @ ws.abs().t(), k, BF, u)


def test_automatic_differentiation_and_differences():
    """The gradients of a sum of squares through ExpertProduct: the formulas', and those that differences of the result give."""
    from paper_2605_04478_amd import step
    offsets = [0, 10, 10, 33]
    x, w, _ = _inputs(33, offsets, 40, 24, FP)
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    gx, gw = x.to(DEV).requires_grad_(), w.to(DEV).requires_grad_()
    y = step.ExpertProduct.apply(gx, gw, off)
    (y.float() ** 2).sum().backward()
    dy = (2 * y.float()).to(FP).cpu()
    want, size = _want(x, w, dy.detach(), offsets)
    _compare(gx.grad, want[1], size[1], 24, FP, "dx")
    _compare(gw.grad, want[2], size[2], 23, FP, "dw")

    def value(xd, wd):
        return sum(((xd[a:b] @ wd[e].t()) ** 2).sum() for e, (a, b) in enumerate(zip(offsets, offsets[1:])))
    g = torch.Generator().manual_seed(5)
    for leaf, grad in ((0, gx.grad), (1, gw.grad)):
        d = torch.randn(grad.shape, generator=g).double()
        h = 1e-4
        args = [x.double(), w.double()]
        hi, lo = list(args), list(args)
        hi[leaf] = args[leaf] + h * d
        lo[leaf] = args[leaf] - h * d
        slope = float(value(*hi) - value(*lo)) / (2 * h)
        got = float((grad.double().cpu() * d).sum())
        # each of the gradient's values is off by at most two roundings to 16 bits (dy and itself) of its size
        bound = float((d.abs() * 2 * rounding(want[1 + leaf].abs() + size[1 + leaf], FP)).sum())
        assert abs(got - slope) <= bound + 1e-6 * abs(slope)
    only = step.ExpertProduct.apply(gx.detach(), gw, off)
    assert torch.autograd.grad(only.sum(), gw)[0].shape == gw.shape


def test_replayed_graph_and_another_stream():
    from paper_2605_04478_amd import step
    offsets = [0, 100, 300, 411]
    x, w, dy = (t.to(DEV) for t in _inputs(411, offsets, 512, 136, BF))
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)

    def call():
        return (step.expert_product(x, w, off), *step.expert_product_grad(dy, x, w, off))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(4):
        x.normal_()
        off.copy_(torch.tensor([0, 30 * i, 200 + i, 411 - i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, call()):
            assert torch.equal(a, b), i
    assert all(torch.isfinite(t).all() for t in on_side)


def test_same_results_again():
    """The order in which workgroups end decides nothing."""
    from paper_2605_04478_amd import step
    offsets = [0, 37, 2000]
    x, w, dy = (t.to(DEV) for t in _inputs(2000, offsets, 2048, 96, BF))
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    first = (step.expert_product(x, w, off), *step.expert_product_grad(dy, x, w, off))
    for _ in range(3):
        again = (step.expert_product(x, w, off), *step.expert_product_grad(dy, x, w, off))
        assert all(torch.equal(a, b) for a, b in zip(first, again))
