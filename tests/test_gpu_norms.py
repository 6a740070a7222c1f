"""The norms around a block with its gate and the residual scale, and their gradients, against the formulas in 64 bits."""
import pytest
import torch

from tests.step_check import F32, close, rounding

pytestmark = pytest.mark.gpu
BF, FP, FF = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda:0"
SCALE, EPS = 0.875, 1e-6
OUT = ("h_out", "u", "dh", "db", "dgate", "dw_post", "dw_pre")


def _inputs(rows, d, groups, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dtype)
    return dict(h=n(rows, d, std=2.0), b=n(rows, d, std=0.5), gate=n(groups, d, std=0.3) if groups else None,
                w_post=(1 + 0.1 * torch.randn(d, generator=g)).to(dtype), w_pre=(1 + 0.1 * torch.randn(d, generator=g)).to(dtype),
                dh_out=n(rows, d), du=n(rows, d))


def _want(s, scale=SCALE, eps=EPS):
    """Results in 64 bits, each with the bound that 32-bit arithmetic and one rounding to the type leave: a value's own roundings,
    and what the errors of the values before it become.  A sum's longest chain has no more than 128 additions within a row."""
    dtype, chain = s["h"].dtype, 128 * F32
    f = {k: None if v is None else v.double() for k, v in s.items()}
    h, b, w1, w2, a = f["h"], f["b"], f["w_post"], f["w_pre"], scale
    rows, d = h.shape
    groups = f["gate"].shape[0] if f["gate"] is not None else 1
    gate = f["gate"].repeat_interleave(rows // groups, 0) if f["gate"] is not None and rows else torch.ones(1, d).double().expand(rows, d)
    dh_out = f["dh_out"] if f["dh_out"] is not None else torch.zeros_like(h)
    du = f["du"] if f["du"] is not None else torch.zeros_like(h)
    mean = lambda t: t.mean(1, keepdim=True)
    r1 = torch.rsqrt(mean(b * b) + eps)
    e1 = chain + 4 * F32
    n = b * r1 * w1
    x = a * h + gate * n
    bx = (a * h).abs() * 3 * F32 + (gate * n).abs() * (e1 + 5 * F32) + x.abs() * F32
    ms = mean(x * x) + eps
    r2 = torch.rsqrt(ms)
    e2 = mean(x.abs() * bx) / ms + chain + 4 * F32
    u = x * r2 * w2
    out = {"h_out": (x, bx), "u": (u, (r2 * w2).abs() * bx + u.abs() * (e2 + 3 * F32))}
    e = du * w2
    m2 = mean(e * x) * r2 * r2
    b_m2 = (mean(e.abs() * bx) + (chain + 3 * F32) * mean((e * x).abs())) * r2 * r2 + m2.abs() * (2 * e2 + 4 * F32)
    dx = dh_out + r2 * (e - x * m2)
    part = r2 * (e.abs() + (x * m2).abs())
    b_dx = part * (e2 + 5 * F32) + r2 * (bx * m2.abs() + x.abs() * b_m2) + dx.abs() * 2 * F32
    out["dh"] = (a * dx, abs(a) * b_dx + (a * dx).abs() * F32)
    b_n = n.abs() * (e1 + 3 * F32)
    per_gate = lambda t: t.view(groups, rows // groups, d).sum(1) if rows else torch.zeros(groups, d).double()
    if f["gate"] is not None:
        out["dgate"] = (per_gate(dx * n), per_gate(b_dx * n.abs() + dx.abs() * b_n + (rows + 8) * F32 * (dx * n).abs()))
    dn, b_dn = dx * gate, b_dx * gate.abs() + (dx * gate).abs() * F32
    fv, b_f = dn * w1, (b_dn * w1.abs()) + (dn * w1).abs() * F32
    m1 = mean(fv * b) * r1 * r1
    b_m1 = (mean(b_f * b.abs()) + (chain + 3 * F32) * mean((fv * b).abs())) * r1 * r1 + m1.abs() * (2 * e1 + 4 * F32)
    db = r1 * (fv - b * m1)
    out["db"] = (db, r1 * (b_f + b.abs() * b_m1) + r1 * (fv.abs() + (b * m1).abs()) * (e1 + 4 * F32))
    t = dn * b * r1
    out["dw_post"] = (t.sum(0), (b_dn * (b * r1).abs() + t.abs() * (e1 + (rows + 8) * F32)).sum(0))
    t = du * x * r2
    out["dw_pre"] = (t.sum(0), (du.abs() * r2 * bx + t.abs() * (e2 + (rows + 8) * F32)).sum(0))
    # halved exponents of products near the smallest numbers: one more step next to zero
    return {k: (v, bound + rounding(v.abs() + bound, dtype) + 1e-37) for k, (v, bound) in out.items()}


def _run(s, scale=SCALE, eps=EPS):
    from paper_2605_04478_amd import step
    h_out, u, r1, r2 = step.norm_residual(s["h"], s["b"], s["gate"], s["w_post"], s["w_pre"], scale=scale, eps=eps)
    grads = step.norm_residual_grad(s["dh_out"], s["du"], s["h"], s["b"], s["gate"], s["w_post"], s["w_pre"], r1, r2, scale=scale)
    return {k: v for k, v in zip(OUT, (h_out, u, *grads)) if v is not None}


def _on(s, form=lambda t: t.to(DEV)):
    return {k: None if v is None else form(v) for k, v in s.items()}


def _check(s, got=None, **kw):
    got = got or _run(_on(s), **kw)
    want = _want(s, **kw)
    assert set(got) == set(want)
    for k, (v, bound) in want.items():
        assert got[k].dtype == s["h"].dtype
        close(got[k], v, bound, k)
    return got


@pytest.mark.parametrize("dtype", [BF, FP, FF], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,d,groups", [(1, 1, 1), (1, 4096, 1), (2, 8, 2), (7, 64, 7), (6, 500, 3), (1030, 512, 1), (300, 520, 4),
                                           (64, 1024, 2), (33, 1025, 1), (600, 2048, 6), (21, 2500, 7), (700, 4096, 1), (12, 4104, 12),
                                           (530, 8192, 2), (9, 8191, 3), (5, 16384, 1), (4, 12345, 2), (1100, 24, 1100)])
def test_against_64_bits(rows, d, groups, dtype):
    _check(_inputs(rows, d, groups, dtype))


@pytest.mark.parametrize("d", [40, 3001])
def test_no_gate_and_missing_gradients(d):
    _check(_inputs(50, d, 0, BF))
    for gone in (("dh_out",), ("du",), ("dh_out", "du")):
        s = _inputs(50, d, 5, BF)
        for k in gone:
            s[k] = None
        got = _check(s)
        if len(gone) == 2:
            assert not any(got[k].any() for k in OUT[2:])


def test_no_rows():
    s = _on(_inputs(0, 96, 3, BF))
    got = _run(s)
    assert got["h_out"].shape == (0, 96) and got["dgate"].shape == (3, 96)
    assert not any(got[k].any() for k in ("dgate", "dw_post", "dw_pre"))


@pytest.mark.parametrize("dtype", [BF, FF], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,groups", [(4096, 2048), (4096, 3 * 512 // 3), (5000, 1000), (3000, 1), (2049, 1), (70000, 70000)])
def test_rows_in_chunks(rows, groups, dtype):
    """Gates of one row, of two, of several chunks: sums over rows are the same however rows are divided."""
    _check(_inputs(rows, 24, groups, dtype))


def test_zero_and_tiny_rows():
    """A block that returns zeros has a finite norm: eps decides."""
    s = _inputs(40, 300, 2, FF)
    s["b"][:10] = 0
    s["b"][10:20] *= 1e-12
    s["h"][5:15] = 0
    _check(s)
    _check(s, eps=1e-3, scale=0.0)
    _check(s, scale=-1.5)


def test_infinities_stay_with_their_rows():
    s = _inputs(60, 200, 3, BF)
    clean = _run(_on(s))
    s["b"][7, 3], s["h"][30, 0], s["du"][50, 10] = float("nan"), float("inf"), float("nan")
    got = _run(_on(s))
    rest = torch.ones(60, dtype=torch.bool)
    rest[[7, 30, 50]] = False
    for k in ("h_out", "u", "dh", "db"):
        assert torch.equal(got[k][rest.to(DEV)], clean[k][rest.to(DEV)]), k
    assert torch.isnan(got["u"][7]).all() and torch.isnan(got["db"][50]).all()
    assert torch.isfinite(got["h_out"][50]).all()


def test_strides_and_orders():
    s = _inputs(90, 136, 3, BF)
    plain = _check(s)

    def padded(t):
        if t.dim() == 1:
            return torch.stack([t, torch.zeros_like(t)], 1).to(DEV)[:, 0]
        big = torch.full((t.shape[0], t.shape[1] + 24), float("nan"), dtype=t.dtype, device=DEV)
        big[:, :t.shape[1]] = t.to(DEV)
        return big[:, :t.shape[1]]

    def transposed(t):
        return t.to(DEV).t().contiguous().t()
    for form in (padded, transposed):
        got = _run(_on(s, form))
        assert all(torch.equal(got[k], plain[k]) for k in plain), form.__name__

    def shifted(t):             # aligned to 2 bytes: columns one by one, summed in another order
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        flat[1:] = t.to(DEV).flatten()
        return flat[1:].view(t.shape)
    _check(s, got=_run(_on(s, shifted)))
    s["du"] = torch.full((1, 1), 0.5, dtype=BF).expand(90, 136)
    _check(s, got=_run({**_on(s), "du": torch.full((1, 1), 0.5, dtype=BF, device=DEV).expand(90, 136)}))


def test_rows_beyond_four_gigabytes():
    from paper_2605_04478_amd import step
    rows, d = (1 << 31) // 8192 + 5, 8192
    h = torch.zeros(rows, d, dtype=BF, device=DEV)
    b = torch.zeros(rows, d, dtype=BF, device=DEV)
    assert h.numel() > 1 << 31
    small = _inputs(4, d, 1, BF)
    h[-4:], b[-4:] = small["h"].to(DEV), small["b"].to(DEV)
    gate, w1, w2 = (small[k].to(DEV) for k in ("gate", "w_post", "w_pre"))
    h_out, u, r1, r2 = step.norm_residual(h, b, gate, w1, w2, scale=SCALE, eps=EPS)
    want = _want({**small})
    close(h_out[-4:], *want["h_out"], "h_out")
    close(u[-4:], *want["u"], "u")
    assert not u[:-4].any()


def test_automatic_differentiation_and_differences():
    from paper_2605_04478_amd import step
    s = _inputs(24, 40, 4, FF)
    leaves = [s[k].to(DEV).requires_grad_() for k in ("h", "b", "gate", "w_post", "w_pre")]
    h_out, u = step.NormResidual.apply(*leaves, SCALE, EPS)
    grads = torch.autograd.grad([h_out, u], leaves, [s["dh_out"].to(DEV), s["du"].to(DEV)])
    want = _want(s)
    for k, g in zip(OUT[2:], grads):
        close(g, *want[k], k)

    def value(h, b, gate, w1, w2):
        n = b / torch.sqrt((b * b).mean(1, keepdim=True) + EPS) * w1
        x = SCALE * h + gate.repeat_interleave(6, 0) * n
        return float((x * s["dh_out"].double()).sum() + (x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * w2 * s["du"].double()).sum())
    gen = torch.Generator().manual_seed(2)
    args = [t.detach().cpu().double() for t in leaves]
    for i, (k, g) in enumerate(zip(OUT[2:], grads)):
        d = torch.randn(g.shape, generator=gen).double()
        hi, lo = list(args), list(args)
        hi[i], lo[i] = args[i] + 1e-5 * d, args[i] - 1e-5 * d
        slope = (value(*hi) - value(*lo)) / 2e-5
        got = float((g.double().cpu() * d).sum())
        assert abs(got - slope) <= float((want[k][1] * d.abs()).sum()) + 1e-6 * abs(slope) + 1e-7, k
    # one output alone: the other's gradient is absent
    only = torch.autograd.grad(step.NormResidual.apply(*leaves, SCALE, EPS)[1], leaves, s["du"].to(DEV))
    want = _want({**s, "dh_out": None})
    for k, g in zip(OUT[2:], only):
        close(g, *want[k], k)


def test_replayed_graph_and_another_stream():
    s = _on(_inputs(900, 264, 9, BF))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = _run(s)
    torch.cuda.current_stream().wait_stream(side)
    here = _run(s)
    assert all(torch.equal(here[k], on_side[k]) for k in here)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _run(s)
    for i in range(4):
        for k in ("h", "b", "du"):
            s[k].normal_()
        graph.replay()
        torch.cuda.synchronize()
        eager = _run(s)
        assert all(torch.equal(out[k], eager[k]) for k in eager), i
