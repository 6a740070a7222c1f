"""The computation of a training step between its collectives, on the GPU.

A rank that the analysis calls computation-slow (Section 2.2, S1) has a slow card, or was given more work than its peers.
These operators are the work to run on such a card, and the kinds of work that are uneven by design: the products of
a rank's experts, whose rows routing decides, and the loss over the vocabulary, which the last pipeline stage alone has; and the norms around a block, which only memory bounds.  Beside them
stands what a step needs around its products: the choice of experts, tokens sorted by expert and back, log probabilities of given tokens, and the optimizer.  The HIP library computes them; this module checks arguments and marshals them
(for ordinary tensors in native code), PyTorch supplies memory and the stream.  Every call goes to the current stream of its tensors' device and returns before it is
done; outputs and workspaces come from torch's allocator, so calls may be captured into a graph.  (Who captures a backward pass of
the classes below captures its forward pass with it, while no eager result of the same leaves is alive: torch would have the
captured pass wait for a stream that is not captured.)

Matrices have unit stride within a row and any row stride.  The functions named `*_grad` are the gradients by themselves;
the classes at the end of each section give the same to automatic differentiation.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from .ccld import CcldError, lib

DTYPES = {torch.bfloat16: 0, torch.float16: 1}
NORM_DTYPES = {**DTYPES, torch.float32: 2}
NORM_MAX = 16384
ROUTE_EXPERTS, ROUTE_MOST = 1024, 64                # most experts, and most of them for a token
ADAMW_BLOCK = 256                   # elements of 8-bit states that share a scale, and what a tensor's states start on a multiple of
ADAMW_WORKSPACE = 256
TOP_MOST = 64                       # most alternatives of a row
MAX_LD = (1 << 22) - (1 << 14)      # a product's operands have their rows closer than this many elements


class _ExpertArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("offsets_bits", C.c_int32), ("rows", C.c_int64), ("k", C.c_int64), ("n", C.c_int64),
                ("n_experts", C.c_int64), ("x", C.c_void_p), ("w", C.c_void_p), ("offsets", C.c_void_p), ("dy", C.c_void_p),
                ("y", C.c_void_p), ("dx", C.c_void_p), ("dw", C.c_void_p), ("ldx", C.c_int64), ("ldw", C.c_int64),
                ("expert_stride", C.c_int64), ("lddy", C.c_int64), ("ldy", C.c_int64), ("lddx", C.c_int64),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class _VocabArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("label_bits", C.c_int32), ("rows", C.c_int64), ("d", C.c_int64), ("vocab", C.c_int64),
                ("h", C.c_void_p), ("w", C.c_void_p), ("labels", C.c_void_p), ("dloss", C.c_void_p), ("loss", C.c_void_p),
                ("lse", C.c_void_p), ("dh", C.c_void_p), ("dw", C.c_void_p), ("ldh", C.c_int64), ("ldw", C.c_int64),
                ("dloss_stride", C.c_int64), ("lddh", C.c_int64), ("lddw", C.c_int64), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_uint64)]


class _NormArgs(C.Structure):
    _fields_ = ([("dtype", C.c_int32), ("scale", C.c_float), ("eps", C.c_float), ("reserved", C.c_int32), ("rows", C.c_int64),
                 ("d", C.c_int64), ("groups", C.c_int64)]
                + [(n, C.c_void_p) for n in ("h", "b", "gate", "w_post", "w_pre", "h_out", "u", "rstd_post", "rstd_pre", "dh_out",
                                             "du", "dh", "db", "dgate", "dw_post", "dw_pre")]
                + [(n, C.c_int64) for n in ("ldh", "ldb", "ldgate", "ldh_out", "ldu", "lddh_out", "lddu", "lddh", "lddb")]
                + [("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)])


class _RouteArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("over_all", C.c_int32), ("tokens", C.c_int64), ("n_experts", C.c_int64), ("k", C.c_int64),
                ("scores", C.c_void_p), ("experts", C.c_void_p), ("weights", C.c_void_p), ("dweights", C.c_void_p), ("dscores", C.c_void_p),
                ("ldscores", C.c_int64), ("lddscores", C.c_int64)]


class _OrderArgs(C.Structure):
    _fields_ = [("expert_bits", C.c_int32), ("reserved", C.c_int32), ("tokens", C.c_int64), ("k", C.c_int64), ("n_experts", C.c_int64),
                ("experts", C.c_void_p), ("places", C.c_void_p), ("offsets", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_uint64)]


class _ExchangeArgs(C.Structure):
    _fields_ = ([("dtype", C.c_int32), ("reserved", C.c_int32), ("tokens", C.c_int64), ("k", C.c_int64), ("d", C.c_int64)]
                + [(n, C.c_void_p) for n in ("places", "used", "weights", "x", "y", "x_out", "y_out", "dweights")]
                + [(n, C.c_int64) for n in ("ldx", "ldy", "ldx_out", "ldy_out")])


class _AdamwTensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("n", C.c_int64), ("start", C.c_int64)]


class _AdamwArgs(C.Structure):
    _fields_ = ([("dtype", C.c_int32), ("grad_dtype", C.c_int32), ("bits", C.c_int32), ("reserved", C.c_int32)]
                + [(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay", "scale")]
                + [("scale_by", C.c_void_p), ("seed", C.c_uint64), ("tensors", C.c_void_p), ("n_tensors", C.c_int64), ("total", C.c_int64)]
                + [(n, C.c_void_p) for n in ("count", "m", "v", "m_scale", "v_scale", "master", "workspace")]
                + [("workspace_bytes", C.c_uint64)])


class _LogprobArgs(C.Structure):
    _fields_ = ([("dtype", C.c_int32), ("token_bits", C.c_int32), ("temperature", C.c_float), ("top", C.c_int32), ("rows", C.c_int64), ("vocab", C.c_int64)]
                + [(n, C.c_void_p) for n in ("logits", "tokens", "logp", "entropy", "lse", "top_ids", "top_logp", "dlogp", "dentropy", "dlogits")]
                + [(n, C.c_int64) for n in ("ldlogits", "lddlogits", "dlogp_stride", "dentropy_stride")]
                + [("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)])


# ---- the calls from native code ---
_calls = None


def _native():
    """The module that makes a call of tensors that are as they should be, and returns None for all others."""
    global _calls
    if _calls is None:
        lib()
        try:
            from . import _step
        except ImportError as e:
            raise RuntimeError("_step.so is missing or of another build: build it with `python -m paper_2605_04478_amd.build`") from e
        _calls = _step
    return _calls


# ---- checks and marshalling -------------------------------------------------------------------------------------
def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _tensor(t, name: str, shape, dtypes):
    """A tensor of this shape (None: any size) and one of these types."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} is no tensor")
    if len(shape) != t.dim() or any(s != n and s is not None for s, n in zip(shape, t.shape)):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple('any' if s is None else s for s in shape)}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} has type {t.dtype}")


def _on_gpu(first, *others):
    """The GPU that all of these (None apart) are on."""
    device = first.device
    for t in (first, *others):
        if t is not None and t.device != device or device.type != "cuda":
            raise ValueError("a tensor is not on a GPU: there is no CPU path" if "cpu" in (device.type, t.device.type)
                             else f"tensors are on {device} and {t.device}")
    return device


def _plain(t):
    """The tensor itself where its memory holds its values, else a copy: torch negates lazily (the gradient of an imaginary part
    is a view with the negative bit), and keeps zeros that have no memory."""
    return t.clone() if t.is_neg() or t._is_zerotensor() else t


def _vector(t):
    return _plain(t).contiguous()


def _rows(t):
    """The tensor itself where its last dimension has unit stride and its rows do not overlap, else a copy that does so
    (expanded and transposed tensors: gradients of broadcast outputs come as the former)."""
    t = _plain(t)
    if t.is_contiguous():
        return t
    if t.stride(-1) != 1 and t.shape[-1] > 1 or any(st < t.shape[-1] and n > 1 for st, n in zip(t.stride()[:-1], t.shape[:-1])):
        return t.contiguous()
    return t


def _operand(t):
    """The same for an operand of a product, whose rows are not too far apart either."""
    t = _rows(t)
    return t.contiguous() if t.shape[-2] > 1 and t.stride(-2) >= MAX_LD else t


def _ld(t) -> int:
    """Elements between rows; that of a single row may be anything."""
    return max(t.stride(-2), t.shape[-1]) if t.shape[-2] > 1 else t.shape[-1]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise CcldError(status, where)


class _NoChange:
    def __enter__(self): pass
    def __exit__(self, *_): pass


_NO_CHANGE = _NoChange()


def _current(device):
    """Makes a GPU the current one, where it is not (which takes some microseconds)."""
    return _NO_CHANGE if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _workspace(query, args, device, *extra):
    """A buffer of the size that the query names, set in the arguments; torch's allocator starts buffers on 512 bytes."""
    need = C.c_uint64()
    _check(query(C.addressof(args), *extra, C.addressof(need)), query.__name__)
    if not need.value:
        return None
    ws = torch.empty(need.value, dtype=torch.uint8, device=device)
    args.workspace, args.workspace_bytes = ws.data_ptr(), need.value
    return ws


def _call(fn, args, device) -> None:
    _check(fn(C.addressof(args), torch._C._cuda_getCurrentRawStream(device.index)), fn.__name__)


# ---- products grouped by expert ---------------------------------------------------------------------------------------
INTEGERS = (torch.int32, torch.int64)


def _expert_inputs(x, w, offsets, *others):
    _tensor(w, "w", (None, None, None), DTYPES)
    e, n, k = w.shape
    _tensor(x, "x", (None, k), (w.dtype,))
    _tensor(offsets, "offsets", (e + 1,), INTEGERS)
    _require(e > 0 and n > 0 and k > 0, f"w has shape {tuple(w.shape)}: no size may be zero")
    for t in others:
        _tensor(t, "dy", (x.shape[0], n), (w.dtype,))
    device = _on_gpu(w, x, offsets, *others)
    return device, _operand(x), _operand(w), _vector(offsets), *map(_operand, others)


def _expert_args(x, w, offsets, dy, y, dx, dw):
    e, n, k = w.shape
    return _ExpertArgs(DTYPES[w.dtype], 8 * offsets.element_size(), x.shape[0], k, n, e, x.data_ptr(), w.data_ptr(), offsets.data_ptr(),
                       _ptr(dy), _ptr(y), _ptr(dx), _ptr(dw), _ld(x), _ld(w), w.stride(0) if e > 1 else 0,
                       n if dy is None else _ld(dy), n, k, None, 0)


def expert_product(x, w, offsets):
    """y[r] = x[r] w[e]^T for the rows offsets[e] .. offsets[e + 1) - 1 of every expert e.

    x [rows, k] and w [experts, n, k] in bfloat16 or float16, offsets [experts + 1] in int32 or int64 -> y [rows, n].
    Rows that belong to no expert are zero.  The offsets stay on the device; they must not decrease."""
    out = _native().expert_product(x, w, offsets)
    if out is not None:
        return out
    device, x, w, offsets = _expert_inputs(x, w, offsets)
    L = lib()
    with _current(device):
        y = torch.empty(x.shape[0], w.shape[1], dtype=w.dtype, device=device)
        a = _expert_args(x, w, offsets, None, y, None, None)
        ws = _workspace(L.ccld_expert_workspace, a, device, 0)      # (kept until the call has been enqueued)
        _call(L.ccld_expert_product, a, device)
    del ws
    return y


def expert_product_grad(dy, x, w, offsets, need_dx: bool = True, need_dw: bool = True):
    """Gradients of expert_product: (dx [rows, k], dw [experts, n, k]); None for one that is not needed."""
    out = _native().expert_product_grad(dy, x, w, offsets, need_dx, need_dw)
    if out is not None:
        return out
    device, x, w, offsets, dy = _expert_inputs(x, w, offsets, dy)
    L = lib()
    with _current(device):
        dx = torch.empty(x.shape, dtype=w.dtype, device=device) if need_dx else None
        dw = torch.empty(w.shape, dtype=w.dtype, device=device) if need_dw else None
        a = _expert_args(x, w, offsets, dy, None, dx, dw)
        ws = _workspace(L.ccld_expert_workspace, a, device, 1)
        _call(L.ccld_expert_product_grad, a, device)
    del ws
    return dx, dw


class ExpertProduct(torch.autograd.Function):
    """expert_product with its gradients: ExpertProduct.apply(x, w, offsets)."""

    @staticmethod
    def forward(ctx, x, w, offsets):
        ctx.save_for_backward(x, w, offsets)
        return expert_product(x, w, offsets)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        dx, dw = expert_product_grad(dy, *ctx.saved_tensors, need_dx=ctx.needs_input_grad[0], need_dw=ctx.needs_input_grad[1])
        return dx, dw, None


# ---- the choice of experts, and tokens sorted by expert and back -----------------------------------------------------------
def _integer(v, name: str, low: int, high: int) -> int:
    _require(isinstance(v, int) and not isinstance(v, bool) and low <= v <= high, f"{name} is {v!r}: {low} to {high} are possible")
    return v


def _route_inputs(scores, k, *others):
    _tensor(scores, "scores", (None, None), NORM_DTYPES)
    t, e = scores.shape
    _require(0 < e <= ROUTE_EXPERTS, f"scores has {e} columns: 1 to {ROUTE_EXPERTS} are possible")
    _integer(k, "k", 1, min(e, ROUTE_MOST))
    for (name, dtype), x in zip((("experts", torch.int32), ("weights", torch.float32), ("dweights", torch.float32)), others):
        _tensor(x, name, (t, k), (dtype,))
    return _on_gpu(scores, *others)


def _route_args(scores, k, over_all, experts, weights, dweights, dscores):
    t, e = scores.shape
    return _RouteArgs(NORM_DTYPES[scores.dtype], bool(over_all), t, e, k, scores.data_ptr(), experts.data_ptr(), weights.data_ptr(), _ptr(dweights),
                      _ptr(dscores), _ld(scores), e)


def route(scores, k: int, over_all: bool = False):
    """The k experts with the largest scores of every token, in descending order, equal ones by the lower expert, and their weights: a softmax
    over the chosen scores, or (over_all) their part of the softmax over all.

    scores [tokens, experts] in bfloat16, float16 or float32 -> (experts [tokens, k] int32, weights [tokens, k] float32).  A score of
    -infinity (or NaN) is never chosen; where fewer than k others are left, the rest of the row is expert -1 with weight 0."""
    out = _native().route(scores, k, over_all)
    if out is not None:
        return out
    device = _route_inputs(scores, k)
    scores = _rows(scores)
    with _current(device):
        experts = torch.empty(scores.shape[0], k, dtype=torch.int32, device=device)
        weights = torch.empty(scores.shape[0], k, dtype=torch.float32, device=device)
        _call(lib().ccld_route, _route_args(scores, k, over_all, experts, weights, None, None), device)
    return experts, weights


def route_grad(dweights, scores, experts, weights, over_all: bool = False):
    """Gradient of route for dweights [tokens, k] and what it returned: dscores [tokens, experts] in the type of scores.  What
    dweights holds for expert -1 does not matter."""
    out = _native().route_grad(dweights, scores, experts, weights, over_all)
    if out is not None:
        return out
    _tensor(experts, "experts", (None, None), (torch.int32,))
    device = _route_inputs(scores, experts.shape[1], experts, weights, dweights)
    scores, experts, weights, dweights = _rows(scores), _vector(experts), _vector(weights), _vector(dweights)
    with _current(device):
        dscores = torch.empty(scores.shape, dtype=scores.dtype, device=device)
        _call(lib().ccld_route_grad, _route_args(scores, experts.shape[1], over_all, experts, weights, dweights, dscores), device)
    return dscores


class Route(torch.autograd.Function):
    """route with its gradient: Route.apply(scores, k, over_all) -> (experts, weights)."""

    @staticmethod
    def forward(ctx, scores, k, over_all):
        experts, weights = route(scores, k, over_all)
        ctx.over_all = over_all
        ctx.save_for_backward(scores, experts, weights)
        ctx.mark_non_differentiable(experts)
        return experts, weights

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, _, dweights):
        return route_grad(dweights, *ctx.saved_tensors, over_all=ctx.over_all), None, None


def expert_order(experts, n_experts: int):
    """The places of entries sorted by expert, in the order of the tokens within an expert.

    experts [tokens, k] in int32 or int64 -> (places [tokens, k], offsets [n_experts + 1]), both int32: entry (t, j) is row places[t, j] of
    the sorted rows, and the rows of expert e are offsets[e] .. offsets[e + 1) - 1, as expert_product takes them.  An
    entry whose expert is outside [0, n_experts) has place -1."""
    out = _native().expert_order(experts, n_experts)
    if out is not None:
        return out
    _tensor(experts, "experts", (None, None), INTEGERS)
    t, k = experts.shape
    _require(k > 0, "experts has no columns")
    _integer(n_experts, "n_experts", 1, ROUTE_EXPERTS)
    device = _on_gpu(experts)
    experts = _vector(experts)
    L = lib()
    with _current(device):
        places = torch.empty(t, k, dtype=torch.int32, device=device)
        offsets = torch.empty(n_experts + 1, dtype=torch.int32, device=device)
        a = _OrderArgs(8 * experts.element_size(), 0, t, k, n_experts, experts.data_ptr(), places.data_ptr(), offsets.data_ptr(), None, 0)
        ws = _workspace(L.ccld_order_workspace, a, device)
        _call(L.ccld_expert_order, a, device)
    del ws
    return places, offsets


def _exchange_inputs(places, x=None, y=None, weights=None, offsets=None, names=("x", "y")):
    """Checks a side's rows against places; x [tokens, d] and y [tokens x k, d]."""
    _tensor(places, "places", (None, None), (torch.int32,))
    t, k = places.shape
    _require(0 < k <= ROUTE_MOST, f"places has {k} columns: 1 to {ROUTE_MOST} are possible")
    first = x if x is not None else y
    d = dtype = None
    for name, m, rows in ((names[0], x, t), (names[1], y, t * k)):
        if m is not None:
            _tensor(m, name, (rows, d), NORM_DTYPES if dtype is None else (dtype,))
            d, dtype = m.shape[1], m.dtype
            _require(d > 0, f"{name} has no columns")
    if weights is not None:
        _tensor(weights, "weights", (t, k), (torch.float32,))
    if offsets is not None:
        _tensor(offsets, "offsets", (None,), (torch.int32,))
        _require(offsets.shape[0] > 0, "offsets is empty")
    device = _on_gpu(first, places, x, y, weights, offsets)
    keep = lambda f, m: None if m is None else f(m)
    return device, _vector(places), keep(_rows, x), keep(_rows, y), keep(_vector, weights), keep(_vector, offsets)


def _exchange(fn, device, places, x, y, weights, offsets, x_out, y_out, dweights=None) -> None:
    t, k = places.shape
    m = next(v for v in (x, y) if v is not None)
    d = m.shape[1]
    used = None if offsets is None else offsets.data_ptr() + 4 * (offsets.shape[0] - 1)
    a = _ExchangeArgs(NORM_DTYPES[m.dtype], 0, t, k, d, places.data_ptr(), used, _ptr(weights), _ptr(x), _ptr(y), _ptr(x_out), _ptr(y_out),
                      _ptr(dweights), d if x is None else _ld(x), d if y is None else _ld(y), d, d)
    _call(fn, a, device)


def dispatch(x, places, offsets):
    """Rows of tokens sorted by expert: rows[places[t, j]] = x[t], for places and offsets of expert_order.

    x [tokens, d] in bfloat16, float16 or float32 -> rows [tokens k, d]; those from offsets[-1] on, which no entry has, are zero."""
    out = _native().dispatch(x, places, offsets)
    if out is not None:
        return out
    device, places, x, _, _, offsets = _exchange_inputs(places, x=x, offsets=offsets)
    with _current(device):
        rows = torch.empty(places.numel(), x.shape[1], dtype=x.dtype, device=device)
        _exchange(lib().ccld_dispatch, device, places, x, None, None, offsets, None, rows)
    return rows


def dispatch_grad(drows, places):
    """Gradient of dispatch for drows [tokens k, d]: dx [tokens, d], the sum of each token's rows."""
    out = _native().dispatch_grad(drows, places)
    if out is not None:
        return out
    device, places, _, drows, _, _ = _exchange_inputs(places, y=drows, names=("x", "drows"))
    with _current(device):
        dx = torch.empty(places.shape[0], drows.shape[1], dtype=drows.dtype, device=device)
        _exchange(lib().ccld_dispatch_grad, device, places, None, drows, None, None, dx, None)
    return dx


class Dispatch(torch.autograd.Function):
    """dispatch with its gradient: Dispatch.apply(x, places, offsets) -> rows."""

    @staticmethod
    def forward(ctx, x, places, offsets):
        ctx.save_for_backward(places)
        return dispatch(x, places, offsets)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, drows):
        return dispatch_grad(drows, *ctx.saved_tensors), None, None


def combine(y, places, weights):
    """The sorted rows back at their tokens, with weights: out[t] = sum over j of weights[t, j] y[places[t, j]].

    y [tokens k, d] in bfloat16, float16 or float32, weights [tokens, k] in float32 -> out [tokens, d].  Entries without a place have no part."""
    out = _native().combine(y, places, weights)
    if out is not None:
        return out
    device, places, _, y, weights, _ = _exchange_inputs(places, y=y, weights=weights)
    with _current(device):
        res = torch.empty(places.shape[0], y.shape[1], dtype=y.dtype, device=device)
        _exchange(lib().ccld_combine, device, places, None, y, weights, None, res, None)
    return res


def combine_grad(dout, y, places, weights, offsets, need_dweights: bool = True):
    """Gradients of combine for dout [tokens, d]: (dy [tokens k, d], dweights [tokens, k] float32, or None where it is not needed).
    Rows of dy from offsets[-1] on are zero, and so is dweights of an entry without a place."""
    out = _native().combine_grad(dout, y, places, weights, offsets, need_dweights)
    if out is not None:
        return out
    device, places, dout, y, weights, offsets = _exchange_inputs(places, x=dout, y=y, weights=weights, offsets=offsets, names=("dout", "y"))
    with _current(device):
        dy = torch.empty(y.shape, dtype=y.dtype, device=device)
        dweights = torch.empty(places.shape, dtype=torch.float32, device=device) if need_dweights else None
        _exchange(lib().ccld_combine_grad, device, places, dout, y, weights, offsets, None, dy, dweights)
    return dy, dweights


class Combine(torch.autograd.Function):
    """combine with its gradients: Combine.apply(y, places, weights, offsets) -> out."""

    @staticmethod
    def forward(ctx, y, places, weights, offsets):
        ctx.save_for_backward(y, places, weights, offsets)
        return combine(y, places, weights)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        dy, dweights = combine_grad(dout, *ctx.saved_tensors, need_dweights=ctx.needs_input_grad[2])
        return dy, None, dweights, None


# ---- softmax cross entropy over a vocabulary ----------------------------------------------------------------------------
def _vocab_inputs(h, w, labels, *others):
    _tensor(w, "w", (None, None), DTYPES)
    v, d = w.shape
    _tensor(h, "h", (None, d), (w.dtype,))
    _tensor(labels, "labels", (h.shape[0],), INTEGERS)
    _require(v > 0 and d > 0, f"w has shape {tuple(w.shape)}: no size may be zero")
    for name, t in zip(("dloss", "lse"), others):
        _tensor(t, name, (h.shape[0],), (torch.float32,))
    device = _on_gpu(w, h, labels, *others)
    return device, _rows(h), _operand(w), _vector(labels)


def _vocab_args(h, w, labels, dloss, loss, lse, dh, dw):
    v, d = w.shape
    return _VocabArgs(DTYPES[w.dtype], 8 * labels.element_size(), h.shape[0], d, v, h.data_ptr(), w.data_ptr(), labels.data_ptr(),
                      _ptr(dloss), _ptr(loss), lse.data_ptr(), _ptr(dh), _ptr(dw), _ld(h), _ld(w),
                      0 if dloss is None else dloss.stride(0), d, d, None, 0)


def vocab_loss(h, w, labels):
    """Softmax cross entropy of every row of h [rows, d] over the vocabulary w [vocab, d], whose logits h w^T are never kept.

    h and w in bfloat16 or float16, labels [rows] in int32 or int64 -> (loss [rows], lse [rows]) in float32, lse being the
    logarithm of the sum of the logits' exponentials.  A row whose label is outside [0, vocab) has no target: both are zero."""
    out = _native().vocab_loss(h, w, labels)
    if out is not None:
        return out
    device, h, w, labels = _vocab_inputs(h, w, labels)
    L = lib()
    with _current(device):
        loss = torch.empty(h.shape[0], dtype=torch.float32, device=device)
        lse = torch.empty(h.shape[0], dtype=torch.float32, device=device)
        a = _vocab_args(h, w, labels, None, loss, lse, None, None)
        ws = _workspace(L.ccld_vocab_workspace, a, device, 0)
        _call(L.ccld_vocab_loss, a, device)
    del ws
    return loss, lse


def vocab_loss_grad(dloss, h, w, labels, lse, need_dh: bool = True, need_dw: bool = True):
    """Gradients of vocab_loss for dloss [rows], the gradient of each row's loss, and the lse that it returned:
    (dh [rows, d], dw [vocab, d]) in the type of h and w; None for one that is not needed.  The logits are taken again, in
    pieces of the vocabulary.  Rows without a target have no gradient, whatever they hold."""
    out = _native().vocab_loss_grad(dloss, h, w, labels, lse, need_dh, need_dw)
    if out is not None:
        return out
    device, h, w, labels = _vocab_inputs(h, w, labels, dloss, lse)
    dloss, lse = _plain(dloss), _vector(lse)
    L = lib()
    with _current(device):
        dh = torch.empty(h.shape, dtype=w.dtype, device=device) if need_dh else None
        dw = torch.empty(w.shape, dtype=w.dtype, device=device) if need_dw else None
        a = _vocab_args(h, w, labels, dloss, None, lse, dh, dw)
        ws = _workspace(L.ccld_vocab_workspace, a, device, 1)
        _call(L.ccld_vocab_loss_grad, a, device)
    del ws
    return dh, dw


class VocabLoss(torch.autograd.Function):
    """vocab_loss with its gradients: VocabLoss.apply(h, w, labels) -> loss [rows]."""

    @staticmethod
    def forward(ctx, h, w, labels):
        loss, lse = vocab_loss(h, w, labels)
        ctx.save_for_backward(h, w, labels, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        h, w, labels, lse = ctx.saved_tensors
        dh, dw = vocab_loss_grad(dloss, h, w, labels, lse, need_dh=ctx.needs_input_grad[0], need_dw=ctx.needs_input_grad[1])
        return dh, dw, None


# ---- log probabilities of given tokens ------------------------------------------------------------------------------------
def _logprob_inputs(logits, tokens, temperature, *others):
    _tensor(logits, "logits", (None, None), NORM_DTYPES)
    rows, v = logits.shape
    _require(v > 0, "logits has no columns")
    _tensor(tokens, "tokens", (rows,), INTEGERS)
    _require(isinstance(temperature, (int, float)) and 2.0 ** -64 <= temperature <= 2.0 ** 64, f"temperature is {temperature!r}: 2^-64 to 2^64 are possible")
    for name, t in zip(("dlogp", "dentropy", "lse", "entropy"), others):
        if t is not None or name in ("lse", "entropy"):
            _tensor(t, name, (rows,), (torch.float32,))
    return _on_gpu(logits, tokens, *others), _rows(logits), _vector(tokens)


def token_logprobs(logits, tokens, temperature: float = 1.0, top: int = 0):
    """Log probabilities of one token of every row under softmax(logits / temperature), and what else is read off such rows.

    logits [rows, vocab] in bfloat16, float16 or float32, tokens [rows] in int32 or int64 -> (logp [rows], entropy [rows], lse [rows],
    top_ids [rows, top] int32, top_logp [rows, top]), in float32: the token's log probability, the entropy of the row's distribution, the logarithm of its
    sum of exponentials, and the `top` largest logits in descending order, equal ones by the lower word, with their log probabilities.

    A token outside [0, vocab) is none: its logp is zero.  Logits of -infinity are ruled out; where fewer than `top` are left, the rest are
    word -1 with -infinity, and a row of nothing has lse -infinity and entropy 0.  A NaN or +infinity makes its row's values NaN."""
    out = _native().token_logprobs(logits, tokens, temperature, top)
    if out is not None:
        return out
    device, logits, tokens = _logprob_inputs(logits, tokens, temperature)
    _integer(top, "top", 0, TOP_MOST)
    rows, v = logits.shape
    L = lib()
    with _current(device):
        logp, entropy, lse = (torch.empty(rows, dtype=torch.float32, device=device) for _ in range(3))
        top_ids = torch.empty(rows, top, dtype=torch.int32, device=device)
        top_logp = torch.empty(rows, top, dtype=torch.float32, device=device)
        a = _LogprobArgs(NORM_DTYPES[logits.dtype], 8 * tokens.element_size(), temperature, top, rows, v, logits.data_ptr(), tokens.data_ptr(), logp.data_ptr(),
                         entropy.data_ptr(), lse.data_ptr(), top_ids.data_ptr(), top_logp.data_ptr(), None, None, None, _ld(logits), v, 0, 0, None, 0)
        ws = _workspace(L.ccld_logprob_workspace, a, device)
        _call(L.ccld_token_logprobs, a, device)
    del ws
    return logp, entropy, lse, top_ids, top_logp


def token_logprobs_grad(dlogp, dentropy, logits, tokens, lse, entropy, temperature: float = 1.0):
    """Gradient of token_logprobs for those of logp and entropy (either may be None: zero) and the lse and entropy that it returned: dlogits [rows, vocab] in
    the type of logits.  A row of nothing has none, and the dlogp of a token that is none does not matter."""
    out = _native().token_logprobs_grad(dlogp, dentropy, logits, tokens, lse, entropy, temperature)
    if out is not None:
        return out
    device, logits, tokens = _logprob_inputs(logits, tokens, temperature, dlogp, dentropy, lse, entropy)
    dlogp, dentropy = (None if t is None else _plain(t) for t in (dlogp, dentropy))
    lse, entropy = _vector(lse), _vector(entropy)
    rows, v = logits.shape
    stride = lambda t: 0 if t is None else t.stride(0)
    with _current(device):
        dlogits = torch.empty(rows, v, dtype=logits.dtype, device=device)
        a = _LogprobArgs(NORM_DTYPES[logits.dtype], 8 * tokens.element_size(), temperature, 0, rows, v, logits.data_ptr(), tokens.data_ptr(), None, entropy.data_ptr(),
                         lse.data_ptr(), None, None, _ptr(dlogp), _ptr(dentropy), dlogits.data_ptr(), _ld(logits), v, stride(dlogp), stride(dentropy), None, 0)
        _call(lib().ccld_token_logprobs_grad, a, device)
    return dlogits


class TokenLogprobs(torch.autograd.Function):
    """token_logprobs with its gradient: TokenLogprobs.apply(logits, tokens, temperature) -> (logp [rows], entropy [rows])."""

    @staticmethod
    def forward(ctx, logits, tokens, temperature):
        logp, entropy, lse, _, _ = token_logprobs(logits, tokens, temperature)
        ctx.set_materialize_grads(False)
        ctx.temperature = temperature
        ctx.save_for_backward(logits, tokens, lse, entropy)
        return logp, entropy

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogp, dentropy):
        return token_logprobs_grad(dlogp, dentropy, *ctx.saved_tensors, ctx.temperature), None, None


# ---- the norms around a block, its gate and the residual scale -----------------------------------------------------------
def _norm_inputs(h, b, gate, w_post, w_pre, eps, dh_out=None, du=None, *rstd):
    _tensor(h, "h", (None, None), NORM_DTYPES)
    rows, d = h.shape
    own = (h.dtype,)
    _tensor(b, "b", (rows, d), own)
    _tensor(w_post, "w_post", (d,), own)
    _tensor(w_pre, "w_pre", (d,), own)
    _require(0 < d <= NORM_MAX, f"h has {d} columns: 1 to {NORM_MAX} are possible")
    if gate is not None:
        _tensor(gate, "gate", (None, d), own)
        groups = gate.shape[0]
        _require(groups > 0 and rows % groups == 0, f"{rows} rows cannot share {groups} rows of gate evenly")
        gate = _rows(gate)
    _require(eps >= 0, f"eps is {eps}")
    for name, t in (("dh_out", dh_out), ("du", du)):
        if t is not None:
            _tensor(t, name, (rows, d), own)
    for name, t in zip(("rstd_post", "rstd_pre"), rstd):
        _tensor(t, name, (rows,), (torch.float32,))
    device = _on_gpu(h, b, gate, w_post, w_pre, dh_out, du, *rstd)
    return device, _rows(h), _rows(b), gate, _vector(w_post), _vector(w_pre)


def norm_residual(h, b, gate, w_post, w_pre, scale: float = 1.0, eps: float = 1e-6):
    """A block's end and the next one's beginning: the norm of the block's output b, its gate, the residual stream h with its
    scale, and the norm that the next block reads.

        h' = scale h + gate (b / rms(b) w_post)          u = h' / rms(h') w_pre          rms(x) = sqrt(mean(x^2) + eps)

    h, b [rows, d] in bfloat16, float16 or float32, w_post and w_pre [d]; gate [g, d], each of whose rows serves rows / g
    consecutive rows, or None.  -> (h', u, 1 / rms(b), 1 / rms(h')), the last two [rows] in float32."""
    out = _native().norm_residual(h, b, gate, w_post, w_pre, scale, eps)
    if out is not None:
        return out
    device, h, b, gate, w_post, w_pre = _norm_inputs(h, b, gate, w_post, w_pre, eps)
    rows, d = h.shape
    with _current(device):
        h_out = torch.empty(rows, d, dtype=h.dtype, device=device)
        u = torch.empty(rows, d, dtype=h.dtype, device=device)
        rstd_post = torch.empty(rows, dtype=torch.float32, device=device)
        rstd_pre = torch.empty(rows, dtype=torch.float32, device=device)
        a = _NormArgs(NORM_DTYPES[h.dtype], scale, eps, 0, rows, d, 1 if gate is None else gate.shape[0], h.data_ptr(), b.data_ptr(),
                      _ptr(gate), w_post.data_ptr(), w_pre.data_ptr(), h_out.data_ptr(), u.data_ptr(), rstd_post.data_ptr(),
                      rstd_pre.data_ptr(), None, None, None, None, None, None, None,
                      _ld(h), _ld(b), d if gate is None else _ld(gate), d, d, d, d, d, d, None, 0)
        _call(lib().ccld_norm_residual, a, device)
    return h_out, u, rstd_post, rstd_pre


def norm_residual_grad(dh_out, du, h, b, gate, w_post, w_pre, rstd_post, rstd_pre, scale: float = 1.0):
    """Gradients of norm_residual for those of h' and u (either may be None: zero) and the two vectors that it returned:
    (dh, db, dgate, dw_post, dw_pre), all in the type of h; dgate is None without a gate."""
    out = _native().norm_residual_grad(dh_out, du, h, b, gate, w_post, w_pre, rstd_post, rstd_pre, scale)
    if out is not None:
        return out
    device, h, b, gate, w_post, w_pre = _norm_inputs(h, b, gate, w_post, w_pre, 0.0, dh_out, du, rstd_post, rstd_pre)
    rows, d = h.shape
    dh_out, du = (None if t is None else _rows(t) for t in (dh_out, du))
    rstd_post, rstd_pre = _vector(rstd_post), _vector(rstd_pre)
    L = lib()
    with _current(device):
        new = lambda *shape: torch.empty(shape, dtype=h.dtype, device=device)
        dh, db, dw_post, dw_pre = new(rows, d), new(rows, d), new(d), new(d)
        dgate = None if gate is None else new(*gate.shape)
        a = _NormArgs(NORM_DTYPES[h.dtype], scale, 0.0, 0, rows, d, 1 if gate is None else gate.shape[0], h.data_ptr(), b.data_ptr(),
                      _ptr(gate), w_post.data_ptr(), w_pre.data_ptr(), None, None, rstd_post.data_ptr(), rstd_pre.data_ptr(),
                      _ptr(dh_out), _ptr(du), dh.data_ptr(), db.data_ptr(), _ptr(dgate), dw_post.data_ptr(), dw_pre.data_ptr(),
                      _ld(h), _ld(b), d if gate is None else _ld(gate), d, d, d if dh_out is None else _ld(dh_out),
                      d if du is None else _ld(du), d, d, None, 0)
        ws = _workspace(L.ccld_norm_workspace, a, device)
        _call(L.ccld_norm_residual_grad, a, device)
    del ws
    return dh, db, dgate, dw_post, dw_pre


class NormResidual(torch.autograd.Function):
    """norm_residual with its gradients: NormResidual.apply(h, b, gate, w_post, w_pre, scale, eps) -> (h', u)."""

    @staticmethod
    def forward(ctx, h, b, gate, w_post, w_pre, scale, eps):
        h_out, u, rstd_post, rstd_pre = norm_residual(h, b, gate, w_post, w_pre, scale, eps)
        ctx.set_materialize_grads(False)
        ctx.scale = scale
        ctx.save_for_backward(h, b, gate, w_post, w_pre, rstd_post, rstd_pre)
        return h_out, u

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh_out, du):
        return (*norm_residual_grad(dh_out, du, *ctx.saved_tensors, scale=ctx.scale), None, None)


# ---- the optimizer --------------------------------------------------------------------------------------------------------
def _padded(n: int) -> int:
    return -(-n // ADAMW_BLOCK) * ADAMW_BLOCK


def _adamw_params(params):
    _require(isinstance(params, (list, tuple)), "params is no list")
    for i, p in enumerate(params):
        if not isinstance(p, torch.Tensor):
            raise ValueError(f"params[{i}] is no tensor")
        if p.dtype not in NORM_DTYPES or p.dtype != params[0].dtype:
            raise ValueError(f"params[{i}] has type {p.dtype}" + (f", params[0] {params[0].dtype}: one call takes one type" if i else ""))
        _require(p.is_contiguous(), f"params[{i}] is not contiguous")
        _require(not p.is_neg() and not p._is_zerotensor(), f"params[{i}] is a view that cannot be written to")
    ranges = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size(), i) for i, p in enumerate(params) if p.numel())
    for (_, end, i), (start, _, k) in zip(ranges, ranges[1:]):
        _require(start >= end, f"params[{min(i, k)}] and params[{max(i, k)}] share memory")


def adamw_state(params, bits: int = 32, masters: bool = False) -> dict:
    """The state of adamw for these parameters before the first step: `count` (steps taken, int64 on the GPU) and the moments `m` and `v` of all
    tensors in one buffer each, in float32, or (bits=8) as float8_e4m3fn and float8_e5m2 relative to `m_scale` and `v_scale`, one for each
    ADAMW_BLOCK elements.  A tensor's values start at a multiple of ADAMW_BLOCK and zeros follow them up to the next.  masters adds `master`,
    the parameters in float32, of which 16-bit ones are then a rounding."""
    _adamw_params(params)
    _require(len(params) > 0, "params is empty")
    _require(bits in (8, 32), f"bits is {bits!r}: 8 and 32 are possible")
    _require(not masters or params[0].dtype != torch.float32, "masters are for 16-bit parameters")
    device, total = _on_gpu(*params), sum(_padded(p.numel()) for p in params)
    zeros = lambda n, dtype: torch.zeros(n, dtype=dtype, device=device)
    state = {"count": zeros(1, torch.int64), "m": zeros(total, torch.float32 if bits == 32 else torch.float8_e4m3fn),
             "v": zeros(total, torch.float32 if bits == 32 else torch.float8_e5m2)}
    if bits == 8:
        state.update(m_scale=zeros(total // ADAMW_BLOCK, torch.float32), v_scale=zeros(total // ADAMW_BLOCK, torch.float32))
    if masters:
        state["master"], at = zeros(total, torch.float32), 0
        for p in params:
            state["master"][at:at + p.numel()] = p.detach().reshape(-1)
            at += _padded(p.numel())
    return state


def _adamw_inputs(params, grads, state, lr, betas, eps, weight_decay, scale, seed):
    """(device, gradients as they can be read, their type, bits, total)"""
    _adamw_params(params)
    _require(isinstance(grads, (list, tuple)) and len(grads) == len(params), f"grads is no list of {len(params)}")
    _require(isinstance(betas, (list, tuple)) and len(betas) == 2 and all(isinstance(b, (int, float)) and 0 <= b < 1 for b in betas),
             f"betas is {betas!r}: two numbers from 0 to less than 1 are possible")
    for name, v in (("lr", lr), ("eps", eps), ("weight_decay", weight_decay)) + (() if isinstance(scale, torch.Tensor) else (("scale", scale),)):
        _require(isinstance(v, (int, float)) and math.isfinite(v), f"{name} is {v!r}: finite numbers are possible")
    _require(eps >= 0, f"eps is {eps}")
    _require(isinstance(seed, int), f"seed is {seed!r}")
    _require(isinstance(state, dict), "state is no dict")
    total = sum(_padded(p.numel()) for p in params)
    _tensor(state.get("count"), "count", (1,), (torch.int64,))
    m = state.get("m")
    _tensor(m, "m", (total,), (torch.float32, torch.float8_e4m3fn))
    bits = 32 if m.dtype == torch.float32 else 8
    _tensor(state.get("v"), "v", (total,), (torch.float32 if bits == 32 else torch.float8_e5m2,))
    names = ["count", "m", "v"]
    if bits == 8:
        names += ["m_scale", "v_scale"]
    for name in names[3:]:
        _tensor(state.get(name), name, (total // ADAMW_BLOCK,), (torch.float32,))
    if state.get("master") is not None:
        names.append("master")
        _tensor(state["master"], "master", (total,), (torch.float32,))
        _require(not params or params[0].dtype != torch.float32, "masters are for 16-bit parameters")
    for name in names:
        _require(state[name].is_contiguous(), f"{name} is not contiguous")
    of = [g for g in grads if g is not None]
    dtype = of[0].dtype if of and isinstance(of[0], torch.Tensor) else torch.float32
    for i, (p, g) in enumerate(zip(params, grads)):
        if g is not None:
            _tensor(g, f"grads[{i}]", p.shape, (p.dtype, torch.float32))
            _require(g.dtype == dtype, f"grads[{i}] has type {g.dtype}, others {dtype}: one call takes one type")
    if isinstance(scale, torch.Tensor):
        _require(scale.numel() == 1, f"scale has shape {tuple(scale.shape)}")
        _require(scale.dtype == torch.float32, f"scale has type {scale.dtype}")
    device = _on_gpu(state["m"], *params, *of, *(state[n] for n in names), scale if isinstance(scale, torch.Tensor) else None)
    return device, [None if g is None else _vector(g) for g in grads], dtype, bits, total


def adamw(params, grads, state, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0, scale=1.0, seed: int = 0) -> None:
    """A step of AdamW over all tensors of params, in place, with their gradients and the state that adamw_state made for them:

        m = b1 m + (1 - b1) scale g      v = b2 v + (1 - b2) (scale g)^2
        p = p - lr weight_decay p - lr / (1 - b1^count) m / (sqrt(v) / sqrt(1 - b2^count) + eps)

    params are contiguous and of one type, bfloat16, float16 or float32; grads of that type or float32, all of one.  A tensor whose
    gradient is None is left as it is, with its state.  scale is a number, or a tensor of one float32 on the GPU (a clipping that was
    computed there).  The count is kept on the GPU: a captured step counts on when it is replayed (with
    the rates that it was captured with).  It is one for all tensors, those without a gradient too: one whose first gradient comes late is corrected
    with the count of the others, and its first step may be larger than lr.  With eps 0 a parameter that never had a gradient becomes NaN, as the formula has it.  8-bit states are rounded up or down
    at random, by `seed`, the count and the element.  A gradient that is not finite leaves NaN: in 8-bit states, in its whole block."""
    if _native().adamw(params, grads, state, lr, betas, eps, weight_decay, scale, seed) is not None:
        return
    # (their own copies: another thread may change the caller's while this one is between its checks and the call)
    params, grads = (list(x) if isinstance(x, (list, tuple)) else x for x in (params, grads))
    state = dict(state) if isinstance(state, dict) else state
    device, grads, grad_dtype, bits, total = _adamw_inputs(params, grads, state, lr, betas, eps, weight_decay, scale, seed)
    if not params:
        return
    at, listed = 0, []
    for p, g in zip(params, grads):
        if g is not None:
            listed.append(_AdamwTensor(p.data_ptr(), g.data_ptr(), p.numel(), at))
        at += _padded(p.numel())
    table = (_AdamwTensor * len(listed))(*listed)
    with _current(device):
        by = scale if isinstance(scale, torch.Tensor) else None
        by = None if by is None else _plain(by)
        ws = torch.empty(ADAMW_WORKSPACE, dtype=torch.uint8, device=device)
        a = _AdamwArgs(NORM_DTYPES[params[0].dtype], NORM_DTYPES[grad_dtype if listed else params[0].dtype], bits, 0, lr, betas[0], betas[1], eps, weight_decay,
                       1.0 if by is not None else scale, _ptr(by), seed & (1 << 64) - 1, C.addressof(table) if listed else None, len(listed), total,
                       state["count"].data_ptr(), state["m"].data_ptr(), state["v"].data_ptr(), _ptr(state.get("m_scale")), _ptr(state.get("v_scale")),
                       _ptr(state.get("master")), ws.data_ptr(), ADAMW_WORKSPACE)
        _call(lib().ccld_adamw, a, device)
    del ws
    torch.autograd.graph.increment_version([p for p, g in zip(params, grads) if g is not None and not p.is_inference()])


class AdamW:
    """adamw with the state that it keeps: AdamW(params, lr), then step() after every backward pass.  All of params have one weight decay: where some are to have another, there are
    two of these."""

    def __init__(self, params, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0, bits: int = 32, masters: bool = False,
                 seed: int = 0):
        self.params = list(params)
        self.lr, self.betas, self.eps, self.weight_decay, self.seed = lr, betas, eps, weight_decay, seed
        self.state = adamw_state(self.params, bits, masters)

    def step(self, grads=None, scale=1.0) -> None:
        """One step with the parameters' gradients, or with those that are given."""
        grads = [p.grad for p in self.params] if grads is None else grads
        adamw(self.params, grads, self.state, self.lr, self.betas, self.eps, self.weight_decay, scale, self.seed)

    def state_dict(self) -> dict:
        """Copies of the state's tensors."""
        return {name: t.clone() for name, t in self.state.items()}

    def load_state_dict(self, state: dict) -> None:
        """Takes over a state of the same parameters and kind."""
        _require(set(state) == set(self.state), f"the state has {sorted(state)}, expected {sorted(self.state)}")
        for name, t in self.state.items():
            _tensor(state[name], name, t.shape, (t.dtype,))
        for name, t in self.state.items():
            t.copy_(state[name])
