"""The computation of a training step between its collectives, on the GPU.

A rank that the analysis calls computation-slow (Section 2.2, S1) has a slow card, or was given more work than its peers.
These operators are the work to run on such a card, and the kinds of work that are uneven by design: the products of
a rank's experts, whose rows routing decides, and the loss over the vocabulary, which the last pipeline stage alone has; and the norms around a block, which only memory bounds.  The HIP library computes them; this module checks arguments and marshals them,
PyTorch supplies memory and the stream.  Every call goes to the current stream of its tensors' device and returns before it is
done; outputs and workspaces come from torch's allocator, so calls may be captured into a graph.

Matrices have unit stride within a row and any row stride.  The functions named `*_grad` are the gradients by themselves;
the classes at the end of each section give the same to automatic differentiation.
"""
from __future__ import annotations

import ctypes as C

import torch

from .ccld import CcldError, lib

DTYPES = {torch.bfloat16: 0, torch.float16: 1}
NORM_DTYPES = {**DTYPES, torch.float32: 2}
NORM_MAX = 16384


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


# ---- checks and marshalling -------------------------------------------------------------------------------------
def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _tensor(t, name: str, shape, dtype):
    """A tensor of this shape (None: any size) and type."""
    _require(torch.is_tensor(t), f"{name} is no tensor")
    _require(t.dim() == len(shape) and all(s is None or s == n for s, n in zip(shape, t.shape)),
             f"{name} has shape {tuple(t.shape)}, expected {tuple('any' if s is None else s for s in shape)}")
    _require(t.dtype in dtype if isinstance(dtype, (tuple, dict)) else t.dtype == dtype, f"{name} has type {t.dtype}")
    return t


def _on_gpu(**tensors):
    """All on one GPU."""
    first = None
    for name, t in tensors.items():
        if t is not None:
            _require(t.is_cuda, f"{name} is not on a GPU: there is no CPU path")
            first = t if first is None else first
            _require(t.device == first.device, f"{name} is on {t.device}, not on {first.device}")


def _rows(t):
    """The tensor itself where its last dimension has unit stride and its rows do not overlap, else a copy that does so
    (expanded and transposed tensors: gradients of broadcast outputs come as the former)."""
    if t.stride(-1) != 1 and t.shape[-1] > 1 or any(st < t.shape[-1] and n > 1 for st, n in zip(t.stride()[:-1], t.shape[:-1])):
        return t.contiguous()
    return t


def _ld(t) -> int:
    """Elements between rows; that of a single row may be anything."""
    return max(t.stride(-2), t.shape[-1]) if t.shape[-2] > 1 else t.shape[-1]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise CcldError(status, where)


def _workspace(query, args, device, *extra):
    """A buffer of the size that the query names, set in the arguments; torch's allocator starts buffers on 512 bytes."""
    need = C.c_uint64(0)
    _check(query(C.addressof(args), *extra, C.addressof(need)), query.__name__)
    ws = torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None
    args.workspace, args.workspace_bytes = _ptr(ws), need.value
    return ws


def _call(fn, args, device) -> None:
    _check(fn(C.addressof(args), torch.cuda.current_stream(device).cuda_stream), fn.__name__)


# ---- products grouped by expert ---------------------------------------------------------------------------------------
def _expert_args(x, w, offsets):
    _tensor(w, "w", (None, None, None), DTYPES)
    e, n, k = w.shape
    _tensor(x, "x", (None, k), w.dtype)
    _tensor(offsets, "offsets", (e + 1,), (torch.int32, torch.int64))
    _require(e > 0 and n > 0 and k > 0, f"w has shape {tuple(w.shape)}: no size may be zero")
    _on_gpu(w=w, x=x, offsets=offsets)
    x, w, offsets = _rows(x), _rows(w), offsets.contiguous()
    a = _ExpertArgs(dtype=DTYPES[w.dtype], offsets_bits=8 * offsets.element_size(), rows=x.shape[0], k=k, n=n, n_experts=e,
                    x=_ptr(x), w=_ptr(w), offsets=_ptr(offsets), ldx=_ld(x), ldw=_ld(w),
                    expert_stride=w.stride(0) if e > 1 else 0)
    return a, (x, w, offsets)


def expert_product(x, w, offsets):
    """y[r] = x[r] w[e]^T for the rows offsets[e] .. offsets[e + 1) - 1 of every expert e.

    x [rows, k] and w [experts, n, k] in bfloat16 or float16, offsets [experts + 1] in int32 or int64 -> y [rows, n].
    Rows that belong to no expert are zero.  The offsets stay on the device; they must not decrease."""
    a, keep = _expert_args(x, w, offsets)
    with torch.cuda.device(w.device):
        y = torch.empty(a.rows, a.n, dtype=w.dtype, device=w.device)
        a.y, a.ldy = _ptr(y), a.n
        ws = _workspace(lib().ccld_expert_workspace, a, w.device, 0)
        _call(lib().ccld_expert_product, a, w.device)
    del keep, ws
    return y


def expert_product_grad(dy, x, w, offsets, need_dx: bool = True, need_dw: bool = True):
    """Gradients of expert_product: (dx [rows, k], dw [experts, n, k]); None for one that is not needed."""
    a, keep = _expert_args(x, w, offsets)
    _tensor(dy, "dy", (a.rows, a.n), w.dtype)
    _on_gpu(w=w, dy=dy)
    dy = _rows(dy)
    with torch.cuda.device(w.device):
        dx = torch.empty(a.rows, a.k, dtype=w.dtype, device=w.device) if need_dx else None
        dw = torch.empty(a.n_experts, a.n, a.k, dtype=w.dtype, device=w.device) if need_dw else None
        a.dy, a.lddy, a.dx, a.lddx, a.dw = _ptr(dy), _ld(dy), _ptr(dx), a.k, _ptr(dw)
        ws = _workspace(lib().ccld_expert_workspace, a, w.device, 1)
        _call(lib().ccld_expert_product_grad, a, w.device)
    del keep, ws
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


# ---- softmax cross entropy over a vocabulary ----------------------------------------------------------------------------
def _vocab_args(h, w, labels):
    _tensor(w, "w", (None, None), DTYPES)
    v, d = w.shape
    _tensor(h, "h", (None, d), w.dtype)
    _tensor(labels, "labels", (h.shape[0],), (torch.int32, torch.int64))
    _require(v > 0 and d > 0, f"w has shape {tuple(w.shape)}: no size may be zero")
    _on_gpu(w=w, h=h, labels=labels)
    h, w, labels = _rows(h), _rows(w), labels.contiguous()
    a = _VocabArgs(dtype=DTYPES[w.dtype], label_bits=8 * labels.element_size(), rows=h.shape[0], d=d, vocab=v, h=_ptr(h),
                   w=_ptr(w), labels=_ptr(labels), ldh=_ld(h), ldw=_ld(w))
    return a, (h, w, labels)


def vocab_loss(h, w, labels):
    """Softmax cross entropy of every row of h [rows, d] over the vocabulary w [vocab, d], whose logits h w^T are never kept.

    h and w in bfloat16 or float16, labels [rows] in int32 or int64 -> (loss [rows], lse [rows]) in float32, lse being the
    logarithm of the sum of the logits' exponentials.  A row whose label is outside [0, vocab) has no target: both are zero."""
    a, keep = _vocab_args(h, w, labels)
    with torch.cuda.device(w.device):
        loss, lse = torch.empty(2, a.rows, dtype=torch.float32, device=w.device).unbind(0)
        a.loss, a.lse = _ptr(loss), _ptr(lse)
        ws = _workspace(lib().ccld_vocab_workspace, a, w.device, 0)
        _call(lib().ccld_vocab_loss, a, w.device)
    del keep, ws
    return loss, lse


def vocab_loss_grad(dloss, h, w, labels, lse, need_dh: bool = True, need_dw: bool = True):
    """Gradients of vocab_loss for dloss [rows], the gradient of each row's loss, and the lse that it returned:
    (dh [rows, d], dw [vocab, d]) in the type of h and w; None for one that is not needed.  The logits are taken again, in
    pieces of the vocabulary.  Rows without a target have no gradient, whatever they hold."""
    a, keep = _vocab_args(h, w, labels)
    _tensor(dloss, "dloss", (a.rows,), torch.float32)
    _tensor(lse, "lse", (a.rows,), torch.float32)
    _on_gpu(w=w, dloss=dloss, lse=lse)
    lse = lse.contiguous()
    with torch.cuda.device(w.device):
        dh = torch.empty(a.rows, a.d, dtype=w.dtype, device=w.device) if need_dh else None
        dw = torch.empty(a.vocab, a.d, dtype=w.dtype, device=w.device) if need_dw else None
        a.dloss, a.dloss_stride, a.lse = _ptr(dloss), dloss.stride(0), _ptr(lse)
        a.dh, a.lddh, a.dw, a.lddw = _ptr(dh), a.d, _ptr(dw), a.d
        ws = _workspace(lib().ccld_vocab_workspace, a, w.device, 1)
        _call(lib().ccld_vocab_loss_grad, a, w.device)
    del keep, ws
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


# ---- the norms around a block, its gate and the residual scale -----------------------------------------------------------
def _norm_args(h, b, gate, w_post, w_pre, scale, eps):
    _tensor(h, "h", (None, None), NORM_DTYPES)
    rows, d = h.shape
    _tensor(b, "b", (rows, d), h.dtype)
    _tensor(w_post, "w_post", (d,), h.dtype)
    _tensor(w_pre, "w_pre", (d,), h.dtype)
    _require(0 < d <= NORM_MAX, f"h has {d} columns: 1 to {NORM_MAX} are possible")
    groups = 1
    if gate is not None:
        _tensor(gate, "gate", (None, d), h.dtype)
        groups = gate.shape[0]
        _require(groups > 0 and rows % groups == 0, f"{rows} rows cannot share {groups} rows of gate evenly")
    _require(eps >= 0, f"eps is {eps}")
    _on_gpu(h=h, b=b, gate=gate, w_post=w_post, w_pre=w_pre)
    h, b, w_post, w_pre = _rows(h), _rows(b), w_post.contiguous(), w_pre.contiguous()
    gate = None if gate is None else _rows(gate)
    a = _NormArgs(dtype=NORM_DTYPES[h.dtype], scale=scale, eps=eps, rows=rows, d=d, groups=groups, h=_ptr(h), b=_ptr(b),
                  gate=_ptr(gate), w_post=_ptr(w_post), w_pre=_ptr(w_pre), ldh=_ld(h), ldb=_ld(b),
                  ldgate=d if gate is None else _ld(gate))
    return a, (h, b, gate, w_post, w_pre)


def norm_residual(h, b, gate, w_post, w_pre, scale: float = 1.0, eps: float = 1e-6):
    """A block's end and the next one's beginning: the norm of the block's output b, its gate, the residual stream h with its
    scale, and the norm that the next block reads.

        h' = scale h + gate (b / rms(b) w_post)          u = h' / rms(h') w_pre          rms(x) = sqrt(mean(x^2) + eps)

    h, b [rows, d] in bfloat16, float16 or float32, w_post and w_pre [d]; gate [g, d], each of whose rows serves rows / g
    consecutive rows, or None.  -> (h', u, 1 / rms(b), 1 / rms(h')), the last two [rows] in float32."""
    a, keep = _norm_args(h, b, gate, w_post, w_pre, scale, eps)
    with torch.cuda.device(h.device):
        h_out, u = (torch.empty(a.rows, a.d, dtype=h.dtype, device=h.device) for _ in range(2))
        rstd_post, rstd_pre = torch.empty(2, a.rows, dtype=torch.float32, device=h.device).unbind(0)
        a.h_out, a.u, a.ldh_out, a.ldu = _ptr(h_out), _ptr(u), a.d, a.d
        a.rstd_post, a.rstd_pre = _ptr(rstd_post), _ptr(rstd_pre)
        _call(lib().ccld_norm_residual, a, h.device)
    del keep
    return h_out, u, rstd_post, rstd_pre


def norm_residual_grad(dh_out, du, h, b, gate, w_post, w_pre, rstd_post, rstd_pre, scale: float = 1.0):
    """Gradients of norm_residual for those of h' and u (either may be None: zero) and the two vectors that it returned:
    (dh, db, dgate, dw_post, dw_pre), all in the type of h; dgate is None without a gate."""
    a, keep = _norm_args(h, b, gate, w_post, w_pre, scale, 0.0)
    for name, t in (("dh_out", dh_out), ("du", du)):
        if t is not None:
            _tensor(t, name, (a.rows, a.d), h.dtype)
    _tensor(rstd_post, "rstd_post", (a.rows,), torch.float32)
    _tensor(rstd_pre, "rstd_pre", (a.rows,), torch.float32)
    _on_gpu(h=h, dh_out=dh_out, du=du, rstd_post=rstd_post, rstd_pre=rstd_pre)
    dh_out, du = (None if t is None else _rows(t) for t in (dh_out, du))
    rstd_post, rstd_pre = rstd_post.contiguous(), rstd_pre.contiguous()
    with torch.cuda.device(h.device):
        dh, db = (torch.empty(a.rows, a.d, dtype=h.dtype, device=h.device) for _ in range(2))
        dgate = None if gate is None else torch.empty(a.groups, a.d, dtype=h.dtype, device=h.device)
        dw_post, dw_pre = (torch.empty(a.d, dtype=h.dtype, device=h.device) for _ in range(2))
        a.dh_out, a.du, a.dh, a.db, a.dgate, a.dw_post, a.dw_pre = map(_ptr, (dh_out, du, dh, db, dgate, dw_post, dw_pre))
        a.lddh_out, a.lddu = (a.d if t is None else _ld(t) for t in (dh_out, du))
        a.lddh, a.lddb = a.d, a.d
        a.rstd_post, a.rstd_pre = _ptr(rstd_post), _ptr(rstd_pre)
        ws = _workspace(lib().ccld_norm_workspace, a, h.device)
        _call(lib().ccld_norm_residual_grad, a, h.device)
    del keep, ws
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
