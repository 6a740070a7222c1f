"""The computation of a training step between its collectives, on the GPU.

A rank that the analysis calls computation-slow (Section 2.2, S1) has a slow card, or was given more work than its peers.
These operators are the work to run on such a card, and the kinds of work that are uneven by design: the products of
a rank's experts, whose rows routing decides, and the loss over the vocabulary, which the last pipeline stage alone has; and the norms around a block, which only memory bounds.  The HIP library computes them; this module checks arguments and marshals them
(for ordinary tensors in native code), PyTorch supplies memory and the stream.  Every call goes to the current stream of its tensors' device and returns before it is
done; outputs and workspaces come from torch's allocator, so calls may be captured into a graph.  (Who captures a backward pass of
the classes below captures its forward pass with it, while no eager result of the same leaves is alive: torch would have the
captured pass wait for a stream that is not captured.)

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
