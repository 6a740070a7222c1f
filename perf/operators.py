"""The computation of a training step between its collectives, as cases that can be timed.

Three operators, forward and with their gradients: the matrix products of a rank's experts (ragged row counts), the
softmax cross entropy over a large vocabulary whose logits are never kept, and the norms before and after a block fused
with its gate and residual scale.  `run` computes a case in its plain form, elementary torch operations in 32 bits, or
(`own`) with the calls that a user makes of `paper_2605_04478_amd.step`; `exact` computes it in 64 bits.

A case is a dict of plain values; "kind" names the operator, "train" whether the gradients are taken too.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6
NO_TARGET = -100
LOSS_SCALE = 65536.0         # of half-precision gradients, as programs that train in that type scale them


def listed():
    return [
        # the last rows of a batch: a few rows for each expert, bound by reading the experts' weights
        experts("experts_few_rows", rows=37, n_experts=16, k=2048, n=4096),
        # an ordinary layer's up projection in half precision, 128 rows for an expert on average, with gradients
        experts("experts_train_fp16", rows=8192, n_experts=64, k=2048, n=1024, dtype="fp16", train=True),
        # sizes that are no multiples of a tile, a third of the experts without any row
        experts("experts_train_ragged", rows=5003, n_experts=12, k=1000, n=1336, idle=4, train=True),
        # the largest layer: 1,024 rows for an expert on average
        experts("experts_train_large", rows=32768, n_experts=32, k=4096, n=4096, train=True),
        # the loss of a handful of positions: bound by reading the vocabulary's weights
        loss("loss_few_rows", rows=5, d=2048, v=32000),
        # the evaluation of a batch: no gradients
        loss("loss_eval", rows=4096, d=2048, v=65536),
        # a fine-tuning batch: a vocabulary of odd size, four rows of ten without a target, half precision
        loss("loss_train_masked_fp16", rows=2000, d=1536, v=50021, masked=0.4, dtype="fp16", train=True),
        # a pre-training micro-batch on the last pipeline stage
        loss("loss_train_large", rows=8192, d=4096, v=128000, train=True),
        # one position
        norm("norm_one_row", rows=1, d=4096),
        # a layer's forward pass over the longest batch
        norm("norm_large", rows=32768, d=8192, groups=1),
        # a layer's gradients over an ordinary batch
        norm("norm_train", rows=16384, d=4096, groups=1, train=True),
        # one gate for each of 7 sequences, a width that is no multiple of a wavefront, in 32 bits
        norm("norm_train_fp32", rows=3003, d=2500, groups=7, dtype="fp32", train=True),
    ]


def experts(name=None, *, rows, n_experts, k, n, idle=0, dtype="bf16", train=False):
    return _case(name, kind="experts", rows=rows, n_experts=n_experts, k=k, n=n, idle=idle, dtype=dtype, train=train)


def loss(name=None, *, rows, d, v, masked=0.0, dtype="bf16", train=False):
    return _case(name, kind="loss", rows=rows, d=d, v=v, masked=masked, dtype=dtype, train=train)


def norm(name=None, *, rows, d, groups=1, dtype="bf16", train=False):
    return _case(name, kind="norm", rows=rows, d=d, groups=groups, dtype=dtype, train=train)


def _case(name, **fields):
    return fields if name is None else dict(name=name, **fields)


# ---- further cases of the same ranges --------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A feature size: mostly whole vectors of 8, now and then an odd one."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.15 else max(8, w // 8 * 8)


def draw(rng):
    kind = rng.choice(("experts", "loss", "norm"))
    train = rng.random() < 0.6
    if kind == "experts":
        k, n, n_experts = _width(rng, 128, 4096), _width(rng, 128, 4096), _log_int(rng, 1, 128)
        return experts(rows=_log_int(rng, 1, 32768), n_experts=n_experts, k=k, n=n,
                       idle=rng.randint(0, n_experts // 3), dtype=rng.choice(("bf16", "bf16", "fp16")), train=train)
    if kind == "loss":
        return loss(rows=_log_int(rng, 1, 8192), d=_width(rng, 256, 4096), v=_log_int(rng, 1000, 128000),
                    masked=rng.choice((0.0, 0.0, round(rng.uniform(0.05, 0.95), 2))),
                    dtype=rng.choice(("bf16", "bf16", "fp16")), train=train)
    rows = _log_int(rng, 1, 32768)
    groups = rng.choice([g for g in (1, 2, 3, 4, 8, rows) if rows % g == 0])
    return norm(rows=rows, d=_width(rng, 64, 8192), groups=groups, dtype=rng.choice(("bf16", "fp16", "fp32")), train=train)


# ---- what a pass cannot do without -------------------------------------------------------------------------
def work(case):
    size, train = DTYPES[case["dtype"]].itemsize, case["train"]
    if case["kind"] == "experts":
        r, k, n = case["rows"], case["k"], case["n"]
        busy = min(r, case["n_experts"] - case["idle"])
        weights, x, y = busy * n * k, r * k, r * n
        moved = x + weights + y
        if train:                                   # dy read, dx and the gradients of all experts written
            moved += y + x + case["n_experts"] * n * k
        return {"bytes": size * moved, "flops": (3 if train else 1) * 2 * r * k * n}
    if case["kind"] == "loss":
        r, d, v = case["rows"], case["d"], case["v"]
        used = max(1, round(r * (1 - case["masked"])))
        moved = size * (used * d + v * d) + 8 * r + 8 * r
        if train:
            moved += size * (r * d + v * d) + 4 * r
        return {"bytes": moved, "flops": (3 if train else 1) * 2 * used * d * v}
    r, d, g = case["rows"], case["d"], case["groups"]
    # forward: h, b, gate and weights read, two outputs written
    moved = 4 * r * d + g * d + 2 * d
    flops = 10 * r * d
    if train:                                       # two gradients read, two and those of gate and weights written
        moved += 4 * r * d + g * d + 2 * d
        flops += 30 * r * d
    return {"bytes": size * moved, "flops": flops}


# ---- inputs ---------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 12345)
    return g


def _normal(g, *shape, dtype, std=1.0):
    """Normal values; large tensors are drawn in their own type."""
    t = torch.empty(shape, device=DEV, dtype=dtype)
    return t.normal_(0.0, std, generator=g)


def prepare(case, seed):
    g = _generator(seed)
    dt = DTYPES[case["dtype"]]
    s = dict(case)
    if case["kind"] == "experts":
        r, k, n, e = case["rows"], case["k"], case["n"], case["n_experts"]
        s["x"] = _normal(g, r, k, dtype=dt)
        s["w"] = _normal(g, e, n, k, dtype=dt, std=k ** -0.5)
        # rows sorted by expert, as routing leaves them: uneven loads, some experts idle
        share = torch.exp(0.7 * torch.randn(e, device=DEV, generator=g))
        share[torch.randperm(e, device=DEV, generator=g)[:case["idle"]]] = 0
        chosen = torch.multinomial(share, r, replacement=True, generator=g)
        counts = torch.bincount(chosen, minlength=e)
        s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        if case["train"]:
            s["dy"] = _normal(g, r, n, dtype=dt)
    elif case["kind"] == "loss":
        r, d, v = case["rows"], case["d"], case["v"]
        s["w"] = _normal(g, v, d, dtype=dt, std=d ** -0.5)
        # frequent and rare tokens; a model that has learnt something: targets stand out by up to 12
        u = torch.rand(r, device=DEV, generator=g)
        target = (torch.exp(u * math.log(v + 1.0)) - 1.0).long().clamp_(0, v - 1)
        boost = 12.0 * torch.rand(r, 1, device=DEV, generator=g)
        s["h"] = (torch.randn(r, d, device=DEV, generator=g) + boost * s["w"][target].float()).to(dt)
        masked = torch.rand(r, device=DEV, generator=g) < case["masked"]
        s["labels"] = torch.where(masked, torch.full_like(target, NO_TARGET), target)
        if case["train"]:
            scale = LOSS_SCALE if case["dtype"] == "fp16" else 1.0
            s["dloss"] = (0.5 + torch.rand(r, device=DEV, generator=g)) * (scale / r)
    else:
        r, d, groups = case["rows"], case["d"], case["groups"]
        s["h"] = _normal(g, r, d, dtype=dt, std=2.0)
        s["b"] = _normal(g, r, d, dtype=dt, std=0.5)
        s["gate"] = _normal(g, groups, d, dtype=dt, std=0.3)
        s["w_post"] = (1.0 + 0.1 * torch.randn(d, device=DEV, generator=g)).to(dt)
        s["w_pre"] = (1.0 + 0.1 * torch.randn(d, device=DEV, generator=g)).to(dt)
        s["scale"] = 0.875
        if case["train"]:
            s["dh_out"] = _normal(g, r, d, dtype=dt)
            s["du"] = _normal(g, r, d, dtype=dt)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    return {"experts": _plain_experts, "loss": _plain_loss, "norm": _plain_norm}[s["kind"]](s)


def _run_own(s):
    from paper_2605_04478_amd import step
    if s["kind"] == "experts":
        out = {"y": step.expert_product(s["x"], s["w"], s["offsets"])}
        if s["train"]:
            out["dx"], out["dw"] = step.expert_product_grad(s["dy"], s["x"], s["w"], s["offsets"])
        return out
    if s["kind"] == "loss":
        value, lse = step.vocab_loss(s["h"], s["w"], s["labels"])
        out = {"loss": value, "lse": lse}
        if s["train"]:
            out["dh"], out["dw"] = step.vocab_loss_grad(s["dloss"], s["h"], s["w"], s["labels"], lse)
        return out
    h_out, u, rstd_post, rstd_pre = step.norm_residual(s["h"], s["b"], s["gate"], s["w_post"], s["w_pre"],
                                                       scale=s["scale"], eps=EPS)
    out = {"h_out": h_out, "u": u}
    if s["train"]:
        out["dh"], out["db"], out["dgate"], out["dw_post"], out["dw_pre"] = step.norm_residual_grad(
            s["dh_out"], s["du"], s["h"], s["b"], s["gate"], s["w_post"], s["w_pre"], rstd_post, rstd_pre,
            scale=s["scale"])
    return out


def _plain_experts(s):
    """One product for each expert that has rows, on the rows that are its own."""
    x, w, dt = s["x"], s["w"], s["x"].dtype
    ends = s["offsets"].tolist()
    out = {"y": torch.zeros(x.shape[0], w.shape[1], device=DEV, dtype=dt)}
    if s["train"]:
        out["dx"] = torch.zeros_like(x)
        out["dw"] = torch.zeros_like(w)
    for e, (a, b) in enumerate(zip(ends, ends[1:])):
        if a == b:
            continue
        xe, we = x[a:b].float(), w[e].float()
        out["y"][a:b] = (xe @ we.t()).to(dt)
        if s["train"]:
            dy = s["dy"][a:b].float()
            out["dx"][a:b] = (dy @ we).to(dt)
            out["dw"][e] = (dy.t() @ xe).to(dt)
    return out


def _plain_loss(s):
    """The whole matrix of logits, its softmax and its gradient, in 32 bits."""
    h, w, labels, dt = s["h"], s["w"], s["labels"], s["h"].dtype
    used = (labels >= 0) & (labels < w.shape[0])
    at = torch.where(used, labels, torch.zeros_like(labels))[:, None]
    hf, wf = torch.where(used[:, None], h.float(), torch.zeros((), device=DEV)), w.float()
    z = hf @ wf.t()
    top = z.max(dim=1, keepdim=True).values
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(dim=1))
    zero = torch.zeros_like(lse)
    out = {"loss": torch.where(used, lse - z.gather(1, at)[:, 0], zero), "lse": torch.where(used, lse, zero)}
    if s["train"]:
        z -= lse[:, None]
        p = z.exp_()
        p.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
        p *= torch.where(used, s["dloss"], zero)[:, None]
        out["dh"] = (p @ wf).to(dt)
        out["dw"] = (p.t() @ hf).to(dt)
    return out


def _plain_norm(s):
    h, b, gate = s["h"].float(), s["b"].float(), s["gate"].float()
    w1, w2, a, dt = s["w_post"].float(), s["w_pre"].float(), s["scale"], s["h"].dtype
    rows, d = h.shape
    groups = gate.shape[0]
    gate = gate.repeat_interleave(rows // groups, dim=0)
    r1 = torch.rsqrt((b * b).mean(dim=1, keepdim=True) + EPS)
    n = b * r1 * w1
    x = a * h + gate * n
    r2 = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)
    out = {"h_out": x.to(dt), "u": (x * r2 * w2).to(dt)}
    if s["train"]:
        du = s["du"].float()
        e = du * w2
        dx = s["dh_out"].float() + r2 * (e - x * (r2 * r2 * (e * x).mean(dim=1, keepdim=True)))
        dn = dx * gate
        f = dn * w1
        out["dh"] = (a * dx).to(dt)
        out["db"] = (r1 * (f - b * (r1 * r1 * (f * b).mean(dim=1, keepdim=True)))).to(dt)
        out["dgate"] = (dx * n).view(groups, rows // groups, d).sum(dim=1).to(dt)
        out["dw_post"] = (dn * b * r1).sum(dim=0).to(dt)
        out["dw_pre"] = (du * x * r2).sum(dim=0).to(dt)
    return out


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    wide = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    if case["kind"] == "experts":
        return _exact_experts(wide, s["offsets"], case["train"])
    if case["kind"] == "loss":
        return _exact_loss(wide, s["labels"], case["train"])
    return _exact_norm(wide, s["scale"], case["train"])


def _exact_experts(t, offsets, train):
    """Row by row the expert is the last one whose rows start at or before it: one masked product for each."""
    x, w = t["x"], t["w"]
    row = torch.arange(x.shape[0], device=DEV)
    owner = torch.searchsorted(offsets[1:].long().contiguous(), row, right=True)
    y = x.new_empty(x.shape[0], w.shape[1])
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    for e in range(w.shape[0]):
        mine = (owner == e).nonzero()[:, 0]
        y[mine] = torch.mm(x[mine], w[e].t().contiguous())
        if train:
            dy = t["dy"][mine]
            dx[mine] = torch.mm(dy, w[e])
            dw[e] = torch.mm(dy.t().contiguous(), x[mine])
    return {"y": y, "dx": dx, "dw": dw} if train else {"y": y}


def _exact_loss(t, labels, train):
    """Rows with a target alone, some hundred at a time."""
    h, w = t["h"], t["w"]
    keep = ((labels >= 0) & (labels < w.shape[0])).nonzero()[:, 0]
    value, lse = h.new_zeros(h.shape[0]), h.new_zeros(h.shape[0])
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    for rows in keep.split(1024):
        z = torch.mm(h[rows], w.t().contiguous())
        l = torch.logsumexp(z, dim=1)
        lse[rows] = l
        value[rows] = l - z[torch.arange(rows.numel(), device=DEV), labels[rows]]
        if train:
            dz = torch.exp(z - l[:, None])
            dz[torch.arange(rows.numel(), device=DEV), labels[rows]] -= 1.0
            dz *= t["dloss"][rows][:, None]
            dh[rows] = torch.mm(dz, w)
            dw += torch.mm(dz.t().contiguous(), h[rows])
    out = {"loss": value, "lse": lse}
    return dict(out, dh=dh, dw=dw) if train else out


def _exact_norm(t, scale, train):
    """The forward formulas, and their gradient by automatic differentiation."""
    rows, d = t["h"].shape
    groups = t["gate"].shape[0]
    leaves = [t[k].clone().requires_grad_(train) for k in ("h", "b", "gate", "w_post", "w_pre")]
    h, b, gate, w_post, w_pre = leaves
    normed = b / torch.sqrt(b.square().sum(dim=1, keepdim=True) / d + EPS) * w_post
    x = scale * h + (gate[:, None, :] * normed.view(groups, rows // groups, d)).view(rows, d)
    u = x / torch.sqrt(x.square().sum(dim=1, keepdim=True) / d + EPS) * w_pre
    out = {"h_out": x.detach(), "u": u.detach()}
    if train:
        grads = torch.autograd.grad([x, u], leaves, [t["dh_out"], t["du"]])
        out.update(zip(("dh", "db", "dgate", "dw_post", "dw_pre"), grads))
    return out
