// Calls of the training step's operators from Python, for tensors that are as they should be (module _step).
//
// A small operator is bound by the host: checks, outputs and arguments of a norm take 15 us in Python and 3 here, its kernel 3.  These
// functions have the arguments of their namesakes in step.py, which describes them.  They return what those return, or None where anything is out
// of the ordinary (a tensor of another shape, type, device or layout, a refusal of the library's): nothing has been enqueued then,
// and step.py, which knows how to lay tensors out and what to say of wrong ones, makes the call.  A failure of the device's raises what step.py
// raises: work may have been enqueued.
#include <algorithm>
#include <utility>
#include <vector>

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include "ccld.h"

namespace {

using at::Tensor;

struct Declined {};
void require(bool ok) { if (!ok) throw Declined(); }

struct Failed { ccld_status status; const char* call; };
// the library refuses before it enqueues anything, in every way but this one
void made(ccld_status s, const char* call) {
  if (s == CCLD_E_HIP) throw Failed{s, call};
  require(s == CCLD_OK);
}

// the arguments of a call; tensors are borrowed
const Tensor& tensor(PyObject* p) {
  require(THPVariable_CheckExact(p));
  return THPVariable_Unpack(p);
}
bool truth(PyObject* p) {
  require(PyBool_Check(p));
  return p == Py_True;
}
int64_t whole(PyObject* p) {
  require(PyLong_CheckExact(p));
  int over = 0;
  const int64_t v = PyLong_AsLongLongAndOverflow(p, &over);
  require(!over);
  return v;
}
double number(PyObject* p) {
  require(PyFloat_CheckExact(p) || PyLong_CheckExact(p));
  const double v = PyFloat_AsDouble(p);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Declined();
  }
  return v;
}

// The GPU of a call's tensors, which has to be the current one.
struct Device {
  c10::Device device;
  explicit Device(const Tensor& first) : device(first.device()) { require(device.is_cuda() && device.index() == c10::hip::current_device()); }
  // (a tensor whose memory holds its values: neither lazily negated nor zeros without memory)
  void has(const Tensor& t) const { require(t.device() == device && !t.is_neg() && !t._is_zerotensor()); }
  // rows of unit stride that do not overlap
  void matrix(const Tensor& t, int64_t rows, int64_t cols, at::ScalarType type) const {
    has(t);
    require(t.dim() == 2 && t.scalar_type() == type && t.size(0) == rows && t.size(1) == cols);
    require((t.stride(1) == 1 || cols == 1) && (t.stride(0) >= cols || rows <= 1));
  }
  void vector(const Tensor& t, int64_t n, at::ScalarType type) const {
    has(t);
    require(t.dim() == 1 && t.scalar_type() == type && t.size(0) == n && t.is_contiguous());
  }
  // (straight from the GPU's allocator: torch::empty takes 0.2 us longer to get there)
  Tensor empty(at::IntArrayRef shape, at::ScalarType type) const { return at::detail::empty_cuda(shape, type, device, std::nullopt); }
  void* stream() const { return c10::hip::getCurrentHIPStream(device.index()).stream(); }
};

int64_t ld(const Tensor& t) { return t.size(-2) > 1 ? std::max(t.stride(-2), t.size(-1)) : t.size(-1); }
void* out(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
const void* in(const Tensor& t) { return t.const_data_ptr(); }

int32_t type_of(const Tensor& t, bool fp32) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return CCLD_BF16;
    case at::kHalf: return CCLD_FP16;
    case at::kFloat: require(fp32); return CCLD_FP32;
    default: throw Declined();
  }
}
int32_t bits_of(const Tensor& t) {
  require(t.scalar_type() == at::kInt || t.scalar_type() == at::kLong);
  return t.scalar_type() == at::kInt ? 32 : 64;
}

// memory and calls need no interpreter
struct WithoutInterpreter {
  PyThreadState* state = PyEval_SaveThread();
  ~WithoutInterpreter() { PyEval_RestoreThread(state); }
};

// Makes the call with a workspace of the size that the query names; torch's allocator keeps its memory for the stream's later work.
template <class A, class Query, class Call>
void run(A& a, const Device& d, Query query, Call call, const char* name) {
  uint64_t need = 0;
  require(query(&a, &need) == CCLD_OK);
  Tensor ws;
  if (need) {
    ws = d.empty({(int64_t)need}, at::kByte);
    a.workspace = ws.data_ptr();
    a.workspace_bytes = need;
  }
  made(call(&a, d.stream()), name);
}

PyObject* wrap(const Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}
template <class... T>
PyObject* tuple(const T&... t) {
  PyObject* p = PyTuple_New(sizeof...(T));
  if (!p) throw python_error();
  Py_ssize_t i = 0;
  (PyTuple_SET_ITEM(p, i++, wrap(t)), ...);
  return p;
}

// ---- products grouped by expert ------------------------------------------------------------------------------------
ccld_expert_args expert_args(const Device& d, const Tensor& x, const Tensor& w, const Tensor& offsets) {
  require(w.dim() == 3 && x.dim() == 2);
  const int64_t e = w.size(0), n = w.size(1), k = w.size(2), rows = x.size(0);
  require(e > 0 && n > 0 && k > 0);
  ccld_expert_args a{};
  a.dtype = type_of(w, false);
  d.has(w);
  require((w.stride(2) == 1 || k == 1) && (w.stride(1) >= k || n == 1) && (w.stride(0) >= k || e == 1));
  d.matrix(x, rows, k, w.scalar_type());
  a.offsets_bits = bits_of(offsets);
  d.vector(offsets, e + 1, offsets.scalar_type());
  a.rows = rows; a.k = k; a.n = n; a.n_experts = e;
  a.x = in(x); a.w = in(w); a.offsets = in(offsets);
  a.ldx = ld(x); a.ldw = ld(w); a.expert_stride = e > 1 ? w.stride(0) : 0;
  a.lddy = a.ldy = n;
  a.lddx = k;
  return a;
}

PyObject* expert_product(PyObject* const* args) {
  const Tensor &x = tensor(args[0]), &w = tensor(args[1]), &offsets = tensor(args[2]);
  const Device d(w);
  ccld_expert_args a = expert_args(d, x, w, offsets);
  Tensor y;
  {
    WithoutInterpreter free;
    y = d.empty({a.rows, a.n}, w.scalar_type());
    a.y = out(y);
    run(a, d, [](auto* p, uint64_t* need) { return ccld_expert_workspace(p, 0, need); }, ccld_expert_product, "ccld_expert_product");
  }
  return wrap(y);
}

PyObject* expert_product_grad(PyObject* const* args) {
  const Tensor &dy = tensor(args[0]), &x = tensor(args[1]), &w = tensor(args[2]), &offsets = tensor(args[3]);
  const bool need_dx = truth(args[4]), need_dw = truth(args[5]);
  const Device d(w);
  ccld_expert_args a = expert_args(d, x, w, offsets);
  d.matrix(dy, a.rows, a.n, w.scalar_type());
  a.dy = in(dy);
  a.lddy = ld(dy);
  Tensor dx, dw;
  {
    WithoutInterpreter free;
    if (need_dx) dx = d.empty({a.rows, a.k}, w.scalar_type());
    if (need_dw) dw = d.empty(w.sizes(), w.scalar_type());
    a.dx = out(dx); a.dw = out(dw);
    run(a, d, [](auto* p, uint64_t* need) { return ccld_expert_workspace(p, 1, need); }, ccld_expert_product_grad, "ccld_expert_product_grad");
  }
  return tuple(dx, dw);
}

// ---- softmax cross entropy over a vocabulary -----------------------------------------------------------------------
ccld_vocab_args vocab_args(const Device& d, const Tensor& h, const Tensor& w, const Tensor& labels) {
  require(w.dim() == 2 && h.dim() == 2);
  const int64_t v = w.size(0), width = w.size(1), rows = h.size(0);
  require(v > 0 && width > 0);
  ccld_vocab_args a{};
  a.dtype = type_of(w, false);
  d.matrix(w, v, width, w.scalar_type());
  d.matrix(h, rows, width, w.scalar_type());
  a.label_bits = bits_of(labels);
  d.vector(labels, rows, labels.scalar_type());
  a.rows = rows; a.d = width; a.vocab = v;
  a.h = in(h); a.w = in(w); a.labels = in(labels);
  a.ldh = ld(h); a.ldw = ld(w);
  a.lddh = a.lddw = width;
  return a;
}

PyObject* vocab_loss(PyObject* const* args) {
  const Tensor &h = tensor(args[0]), &w = tensor(args[1]), &labels = tensor(args[2]);
  const Device d(w);
  ccld_vocab_args a = vocab_args(d, h, w, labels);
  Tensor loss, lse;
  {
    WithoutInterpreter free;
    loss = d.empty({a.rows}, at::kFloat);
    lse = d.empty({a.rows}, at::kFloat);
    a.loss = static_cast<float*>(out(loss));
    a.lse = static_cast<float*>(out(lse));
    run(a, d, [](auto* p, uint64_t* need) { return ccld_vocab_workspace(p, 0, need); }, ccld_vocab_loss, "ccld_vocab_loss");
  }
  return tuple(loss, lse);
}

PyObject* vocab_loss_grad(PyObject* const* args) {
  const Tensor &dloss = tensor(args[0]), &h = tensor(args[1]), &w = tensor(args[2]), &labels = tensor(args[3]), &lse = tensor(args[4]);
  const bool need_dh = truth(args[5]), need_dw = truth(args[6]);
  const Device d(w);
  ccld_vocab_args a = vocab_args(d, h, w, labels);
  d.has(dloss);
  require(dloss.dim() == 1 && dloss.size(0) == a.rows && dloss.scalar_type() == at::kFloat);
  d.vector(lse, a.rows, at::kFloat);
  a.dloss = static_cast<const float*>(in(dloss));
  a.dloss_stride = dloss.stride(0);
  a.lse = static_cast<float*>(const_cast<void*>(in(lse)));          // read only in this call
  Tensor dh, dw;
  {
    WithoutInterpreter free;
    if (need_dh) dh = d.empty({a.rows, a.d}, w.scalar_type());
    if (need_dw) dw = d.empty({a.vocab, a.d}, w.scalar_type());
    a.dh = out(dh); a.dw = out(dw);
    run(a, d, [](auto* p, uint64_t* need) { return ccld_vocab_workspace(p, 1, need); }, ccld_vocab_loss_grad, "ccld_vocab_loss_grad");
  }
  return tuple(dh, dw);
}

// ---- log probabilities of given tokens -------------------------------------------------------------------------------
ccld_logprob_args logprob_args(const Device& d, const Tensor& logits, const Tensor& tokens, double temperature) {
  require(logits.dim() == 2);
  ccld_logprob_args a{};
  a.dtype = type_of(logits, true);
  a.rows = logits.size(0); a.vocab = logits.size(1);
  require(a.vocab > 0);
  d.matrix(logits, a.rows, a.vocab, logits.scalar_type());
  a.token_bits = bits_of(tokens);
  d.vector(tokens, a.rows, tokens.scalar_type());
  a.temperature = (float)temperature;
  a.logits = in(logits); a.tokens = in(tokens);
  a.ldlogits = ld(logits);
  a.lddlogits = a.vocab;
  return a;
}

PyObject* token_logprobs(PyObject* const* args) {
  const Tensor &logits = tensor(args[0]), &tokens = tensor(args[1]);
  const Device d(logits);
  ccld_logprob_args a = logprob_args(d, logits, tokens, number(args[2]));
  const int64_t top = whole(args[3]);
  require(top >= 0 && top <= CCLD_TOP_MOST);
  a.top = (int32_t)top;
  Tensor logp, entropy, lse, top_ids, top_logp;
  {
    WithoutInterpreter free;
    logp = d.empty({a.rows}, at::kFloat);
    entropy = d.empty({a.rows}, at::kFloat);
    lse = d.empty({a.rows}, at::kFloat);
    top_ids = d.empty({a.rows, top}, at::kInt);
    top_logp = d.empty({a.rows, top}, at::kFloat);
    a.logp = static_cast<float*>(out(logp));
    a.entropy = static_cast<float*>(out(entropy));
    a.lse = static_cast<float*>(out(lse));
    a.top_ids = static_cast<int32_t*>(out(top_ids));
    a.top_logp = static_cast<float*>(out(top_logp));
    run(a, d, ccld_logprob_workspace, ccld_token_logprobs, "ccld_token_logprobs");
  }
  return tuple(logp, entropy, lse, top_ids, top_logp);
}

PyObject* token_logprobs_grad(PyObject* const* args) {
  const Tensor &logits = tensor(args[2]), &tokens = tensor(args[3]), &lse = tensor(args[4]), &entropy = tensor(args[5]);
  const Device d(logits);
  ccld_logprob_args a = logprob_args(d, logits, tokens, number(args[6]));
  auto gradient = [&](PyObject* p, const float*& at, int64_t& stride) {
    if (p == Py_None) return;
    const Tensor& t = tensor(p);
    d.has(t);
    require(t.dim() == 1 && t.size(0) == a.rows && t.scalar_type() == at::kFloat);
    at = static_cast<const float*>(in(t));
    stride = t.stride(0);
  };
  gradient(args[0], a.dlogp, a.dlogp_stride);
  gradient(args[1], a.dentropy, a.dentropy_stride);
  d.vector(lse, a.rows, at::kFloat);
  d.vector(entropy, a.rows, at::kFloat);
  a.lse = static_cast<float*>(const_cast<void*>(in(lse)));          // read only in this call
  a.entropy = static_cast<float*>(const_cast<void*>(in(entropy)));
  Tensor dlogits;
  {
    WithoutInterpreter free;
    dlogits = d.empty({a.rows, a.vocab}, logits.scalar_type());
    a.dlogits = out(dlogits);
    made(ccld_token_logprobs_grad(&a, d.stream()), "ccld_token_logprobs_grad");
  }
  return wrap(dlogits);
}

// ---- the norms around a block, its gate and the residual scale ---------------------------------------------------------
ccld_norm_args norm_args(const Device& d, const Tensor& h, const Tensor& b, PyObject* gate, const Tensor& w_post, const Tensor& w_pre) {
  require(h.dim() == 2);
  const int64_t rows = h.size(0), width = h.size(1);
  const at::ScalarType type = h.scalar_type();
  ccld_norm_args a{};
  a.dtype = type_of(h, true);
  d.matrix(h, rows, width, type);
  d.matrix(b, rows, width, type);
  d.vector(w_post, width, type);
  d.vector(w_pre, width, type);
  a.groups = 1;
  a.ldgate = width;
  if (gate != Py_None) {
    const Tensor& g = tensor(gate);
    require(g.dim() == 2);
    d.matrix(g, g.size(0), width, type);
    a.gate = in(g);
    a.groups = g.size(0);
    a.ldgate = ld(g);
    require(a.groups > 0 && rows % a.groups == 0);
  }
  a.rows = rows; a.d = width;
  a.h = in(h); a.b = in(b); a.w_post = in(w_post); a.w_pre = in(w_pre);
  a.ldh = ld(h); a.ldb = ld(b);
  a.ldh_out = a.ldu = a.lddh_out = a.lddu = a.lddh = a.lddb = width;
  return a;
}

PyObject* norm_residual(PyObject* const* args) {
  const Tensor &h = tensor(args[0]), &b = tensor(args[1]), &w_post = tensor(args[3]), &w_pre = tensor(args[4]);
  const Device d(h);
  ccld_norm_args a = norm_args(d, h, b, args[2], w_post, w_pre);
  a.scale = (float)number(args[5]);
  a.eps = (float)number(args[6]);
  Tensor h_out, u, rstd_post, rstd_pre;
  {
    WithoutInterpreter free;
    h_out = d.empty({a.rows, a.d}, h.scalar_type());
    u = d.empty({a.rows, a.d}, h.scalar_type());
    rstd_post = d.empty({a.rows}, at::kFloat);
    rstd_pre = d.empty({a.rows}, at::kFloat);
    a.h_out = out(h_out); a.u = out(u);
    a.rstd_post = static_cast<float*>(out(rstd_post));
    a.rstd_pre = static_cast<float*>(out(rstd_pre));
    made(ccld_norm_residual(&a, d.stream()), "ccld_norm_residual");
  }
  return tuple(h_out, u, rstd_post, rstd_pre);
}

PyObject* norm_residual_grad(PyObject* const* args) {
  const Tensor &h = tensor(args[2]), &b = tensor(args[3]), &w_post = tensor(args[5]), &w_pre = tensor(args[6]);
  const Tensor &rstd_post = tensor(args[7]), &rstd_pre = tensor(args[8]);
  const Device d(h);
  ccld_norm_args a = norm_args(d, h, b, args[4], w_post, w_pre);
  a.scale = (float)number(args[9]);
  const at::ScalarType type = h.scalar_type();
  auto gradient = [&](PyObject* p, const void*& at, int64_t& stride) {
    if (p == Py_None) return;
    const Tensor& t = tensor(p);
    d.matrix(t, a.rows, a.d, type);
    at = in(t);
    stride = ld(t);
  };
  gradient(args[0], a.dh_out, a.lddh_out);
  gradient(args[1], a.du, a.lddu);
  d.vector(rstd_post, a.rows, at::kFloat);
  d.vector(rstd_pre, a.rows, at::kFloat);
  a.rstd_post = static_cast<float*>(const_cast<void*>(in(rstd_post)));          // read only in this call
  a.rstd_pre = static_cast<float*>(const_cast<void*>(in(rstd_pre)));
  Tensor dh, db, dgate, dw_post, dw_pre;
  {
    WithoutInterpreter free;
    dh = d.empty({a.rows, a.d}, type);
    db = d.empty({a.rows, a.d}, type);
    if (a.gate) dgate = d.empty({a.groups, a.d}, type);
    dw_post = d.empty({a.d}, type);
    dw_pre = d.empty({a.d}, type);
    a.dh = out(dh); a.db = out(db); a.dgate = out(dgate); a.dw_post = out(dw_post); a.dw_pre = out(dw_pre);
    run(a, d, ccld_norm_workspace, ccld_norm_residual_grad, "ccld_norm_residual_grad");
  }
  return tuple(dh, db, dgate, dw_post, dw_pre);
}

// ---- the choice of experts, and tokens sorted by expert and back -----------------------------------------------------
ccld_route_args route_args(const Device& d, const Tensor& scores, int64_t k, bool over_all) {
  require(scores.dim() == 2);
  ccld_route_args a{};
  a.dtype = type_of(scores, true);
  a.over_all = over_all;
  a.tokens = scores.size(0); a.n_experts = scores.size(1); a.k = k;
  require(k >= 1 && k <= a.n_experts && k <= CCLD_ROUTE_MOST && a.n_experts <= CCLD_ROUTE_EXPERTS);
  d.matrix(scores, a.tokens, a.n_experts, scores.scalar_type());
  a.scores = in(scores);
  a.ldscores = ld(scores);
  a.lddscores = a.n_experts;
  return a;
}
void contiguous(const Device& d, const Tensor& t, int64_t rows, int64_t cols, at::ScalarType type) {
  d.matrix(t, rows, cols, type);
  require(t.is_contiguous());
}

PyObject* route(PyObject* const* args) {
  const Tensor& scores = tensor(args[0]);
  const Device d(scores);
  ccld_route_args a = route_args(d, scores, whole(args[1]), truth(args[2]));
  Tensor experts, weights;
  {
    WithoutInterpreter free;
    experts = d.empty({a.tokens, a.k}, at::kInt);
    weights = d.empty({a.tokens, a.k}, at::kFloat);
    a.experts = static_cast<int32_t*>(out(experts));
    a.weights = static_cast<float*>(out(weights));
    made(ccld_route(&a, d.stream()), "ccld_route");
  }
  return tuple(experts, weights);
}

PyObject* route_grad(PyObject* const* args) {
  const Tensor &dweights = tensor(args[0]), &scores = tensor(args[1]), &experts = tensor(args[2]), &weights = tensor(args[3]);
  const Device d(scores);
  require(experts.dim() == 2);
  ccld_route_args a = route_args(d, scores, experts.size(1), truth(args[4]));
  contiguous(d, experts, a.tokens, a.k, at::kInt);
  contiguous(d, weights, a.tokens, a.k, at::kFloat);
  contiguous(d, dweights, a.tokens, a.k, at::kFloat);
  a.experts = static_cast<int32_t*>(const_cast<void*>(in(experts)));          // read only in this call
  a.weights = static_cast<float*>(const_cast<void*>(in(weights)));
  a.dweights = static_cast<const float*>(in(dweights));
  Tensor dscores;
  {
    WithoutInterpreter free;
    dscores = d.empty({a.tokens, a.n_experts}, scores.scalar_type());
    a.dscores = out(dscores);
    made(ccld_route_grad(&a, d.stream()), "ccld_route_grad");
  }
  return wrap(dscores);
}

PyObject* expert_order(PyObject* const* args) {
  const Tensor& experts = tensor(args[0]);
  const Device d(experts);
  require(experts.dim() == 2 && experts.is_contiguous());
  d.has(experts);
  ccld_order_args a{};
  a.expert_bits = bits_of(experts);
  a.tokens = experts.size(0); a.k = experts.size(1); a.n_experts = whole(args[1]);
  require(a.k > 0 && a.n_experts >= 1 && a.n_experts <= CCLD_ROUTE_EXPERTS);
  a.experts = in(experts);
  Tensor places, offsets;
  {
    WithoutInterpreter free;
    places = d.empty({a.tokens, a.k}, at::kInt);
    offsets = d.empty({a.n_experts + 1}, at::kInt);
    a.places = static_cast<int32_t*>(out(places));
    a.offsets = static_cast<int32_t*>(out(offsets));
    run(a, d, ccld_order_workspace, ccld_expert_order, "ccld_expert_order");
  }
  return tuple(places, offsets);
}

// x [tokens][d] and y [tokens k][d], one of which may be missing
ccld_exchange_args exchange_args(const Device& d, const Tensor& places, const Tensor* x, const Tensor* y, const Tensor* weights, const Tensor* offsets) {
  require(places.dim() == 2);
  const Tensor& m = x ? *x : *y;
  require(m.dim() == 2);
  ccld_exchange_args a{};
  a.dtype = type_of(m, true);
  a.tokens = places.size(0); a.k = places.size(1); a.d = m.size(1);
  require(a.k > 0 && a.k <= CCLD_ROUTE_MOST && a.d > 0);
  contiguous(d, places, a.tokens, a.k, at::kInt);
  a.places = static_cast<const int32_t*>(in(places));
  a.ldx = a.ldy = a.ldx_out = a.ldy_out = a.d;
  if (x) {
    d.matrix(*x, a.tokens, a.d, m.scalar_type());
    a.x = in(*x);
    a.ldx = ld(*x);
  }
  if (y) {
    d.matrix(*y, a.tokens * a.k, a.d, m.scalar_type());
    a.y = in(*y);
    a.ldy = ld(*y);
  }
  if (weights) {
    contiguous(d, *weights, a.tokens, a.k, at::kFloat);
    a.weights = static_cast<const float*>(in(*weights));
  }
  if (offsets) {
    require(offsets->dim() == 1 && offsets->size(0) > 0);
    d.vector(*offsets, offsets->size(0), at::kInt);
    a.used = static_cast<const int32_t*>(in(*offsets)) + offsets->size(0) - 1;
  }
  return a;
}

PyObject* dispatch(PyObject* const* args) {
  const Tensor &x = tensor(args[0]), &places = tensor(args[1]), &offsets = tensor(args[2]);
  const Device d(x);
  ccld_exchange_args a = exchange_args(d, places, &x, nullptr, nullptr, &offsets);
  Tensor rows;
  {
    WithoutInterpreter free;
    rows = d.empty({a.tokens * a.k, a.d}, x.scalar_type());
    a.y_out = out(rows);
    made(ccld_dispatch(&a, d.stream()), "ccld_dispatch");
  }
  return wrap(rows);
}

PyObject* dispatch_grad(PyObject* const* args) {
  const Tensor &drows = tensor(args[0]), &places = tensor(args[1]);
  const Device d(drows);
  ccld_exchange_args a = exchange_args(d, places, nullptr, &drows, nullptr, nullptr);
  Tensor dx;
  {
    WithoutInterpreter free;
    dx = d.empty({a.tokens, a.d}, drows.scalar_type());
    a.x_out = out(dx);
    made(ccld_dispatch_grad(&a, d.stream()), "ccld_dispatch_grad");
  }
  return wrap(dx);
}

PyObject* combine(PyObject* const* args) {
  const Tensor &y = tensor(args[0]), &places = tensor(args[1]), &weights = tensor(args[2]);
  const Device d(y);
  ccld_exchange_args a = exchange_args(d, places, nullptr, &y, &weights, nullptr);
  Tensor res;
  {
    WithoutInterpreter free;
    res = d.empty({a.tokens, a.d}, y.scalar_type());
    a.x_out = out(res);
    made(ccld_combine(&a, d.stream()), "ccld_combine");
  }
  return wrap(res);
}

PyObject* combine_grad(PyObject* const* args) {
  const Tensor &dout = tensor(args[0]), &y = tensor(args[1]), &places = tensor(args[2]), &weights = tensor(args[3]), &offsets = tensor(args[4]);
  const bool need_dweights = truth(args[5]);
  const Device d(y);
  ccld_exchange_args a = exchange_args(d, places, &dout, &y, &weights, &offsets);
  Tensor dy, dweights;
  {
    WithoutInterpreter free;
    dy = d.empty({a.tokens * a.k, a.d}, y.scalar_type());
    if (need_dweights) dweights = d.empty({a.tokens, a.k}, at::kFloat);
    a.y_out = out(dy);
    a.dweights = static_cast<float*>(out(dweights));
    made(ccld_combine_grad(&a, d.stream()), "ccld_combine_grad");
  }
  return tuple(dy, dweights);
}

// ---- the optimizer -----------------------------------------------------------------------------------------------------
// a list or tuple
struct Sequence {
  PyObject* p;
  Py_ssize_t n;
  explicit Sequence(PyObject* o) : p(o), n(0) {
    require(PyList_CheckExact(o) || PyTuple_CheckExact(o));
    n = Py_SIZE(o);
  }
  PyObject* operator[](Py_ssize_t i) const { return PyList_CheckExact(p) ? PyList_GET_ITEM(p, i) : PyTuple_GET_ITEM(p, i); }
};

// (parameters may be of a subclass of tensors)
const Tensor& parameter(PyObject* p) {
  require(THPVariable_Check(p));
  return THPVariable_Unpack(p);
}

PyObject* adamw(PyObject* const* args) {
  const Sequence params(args[0]), grads(args[1]), betas(args[4]);
  PyObject* const state = args[2];
  require(PyDict_CheckExact(state) && params.n > 0 && grads.n == params.n && betas.n == 2);
  const Tensor& first = parameter(params[0]);
  const Device d(first);
  ccld_adamw_args a{};
  a.dtype = a.grad_dtype = type_of(first, true);
  std::vector<ccld_adamw_tensor> tensors;
  std::vector<Tensor> stepped, kept_grads, kept_states;  // (held while the interpreter is left: another thread may change the lists and the dict)
  std::vector<std::pair<uintptr_t, uintptr_t>> ranges;
  tensors.reserve(params.n);
  stepped.reserve(params.n);
  kept_grads.reserve(params.n);
  kept_states.reserve(6);
  ranges.reserve(params.n);
  at::ScalarType grad_type = at::ScalarType::Undefined;
  for (Py_ssize_t i = 0; i < params.n; ++i) {
    const Tensor& p = parameter(params[i]);
    d.has(p);
    require(p.scalar_type() == first.scalar_type() && p.is_contiguous());
    const int64_t n = p.numel();
    if (n) ranges.emplace_back((uintptr_t)p.data_ptr(), (uintptr_t)p.data_ptr() + n * p.element_size());
    if (grads[i] != Py_None) {
      const Tensor& g = tensor(grads[i]);
      d.has(g);
      require(g.is_contiguous() && g.sizes() == p.sizes() && (g.scalar_type() == p.scalar_type() || g.scalar_type() == at::kFloat));
      require(grad_type == at::ScalarType::Undefined || grad_type == g.scalar_type());
      grad_type = g.scalar_type();
      tensors.push_back({p.data_ptr(), in(g), n, a.total});
      stepped.push_back(p);
      kept_grads.push_back(g);
    }
    a.total += (n + CCLD_ADAMW_BLOCK - 1) / CCLD_ADAMW_BLOCK * CCLD_ADAMW_BLOCK;
  }
  std::sort(ranges.begin(), ranges.end());
  for (size_t i = 1; i < ranges.size(); ++i) require(ranges[i].first >= ranges[i - 1].second);
  if (grad_type == at::kFloat) a.grad_dtype = CCLD_FP32;
  auto kept = [&](const char* name, int64_t n, at::ScalarType type) -> void* {
    PyObject* const o = PyDict_GetItemString(state, name);
    require(o);
    const Tensor& t = tensor(o);
    d.vector(t, n, type);
    kept_states.push_back(t);
    return t.data_ptr();
  };
  PyObject* const m = PyDict_GetItemString(state, "m");
  require(m);
  a.bits = tensor(m).scalar_type() == at::kFloat ? 32 : 8;
  a.count = static_cast<int64_t*>(kept("count", 1, at::kLong));
  a.m = kept("m", a.total, a.bits == 32 ? at::kFloat : at::kFloat8_e4m3fn);
  a.v = kept("v", a.total, a.bits == 32 ? at::kFloat : at::kFloat8_e5m2);
  if (a.bits == 8) {
    a.m_scale = static_cast<float*>(kept("m_scale", a.total / CCLD_ADAMW_BLOCK, at::kFloat));
    a.v_scale = static_cast<float*>(kept("v_scale", a.total / CCLD_ADAMW_BLOCK, at::kFloat));
  }
  if (PyObject* const o = PyDict_GetItemString(state, "master"); o && o != Py_None) {
    require(first.scalar_type() != at::kFloat);
    a.master = static_cast<float*>(kept("master", a.total, at::kFloat));
  }
  a.lr = number(args[3]); a.beta1 = number(betas[0]); a.beta2 = number(betas[1]); a.eps = number(args[5]); a.weight_decay = number(args[6]);
  if (THPVariable_CheckExact(args[7])) {
    const Tensor& by = tensor(args[7]);
    d.has(by);
    require(by.numel() == 1 && by.scalar_type() == at::kFloat);
    a.scale = 1;
    a.scale_by = static_cast<const float*>(in(by));
  } else {
    a.scale = number(args[7]);
  }
  a.seed = (uint64_t)whole(args[8]);
  a.tensors = tensors.data();
  a.n_tensors = (int64_t)tensors.size();
  {
    WithoutInterpreter free;
    const Tensor ws = d.empty({CCLD_ADAMW_WORKSPACE}, at::kByte);
    a.workspace = ws.data_ptr();
    a.workspace_bytes = CCLD_ADAMW_WORKSPACE;
    made(ccld_adamw(&a, d.stream()), "ccld_adamw");
    // (who saved a parameter for a backward pass is told that it has changed)
    for (const Tensor& p : stepped)
      if (!p.is_inference()) p.unsafeGetTensorImpl()->bump_version();
  }
  Py_RETURN_TRUE;
}

// raises CcldError
PyObject* raise(const Failed& f) {
  PyObject* module = PyImport_ImportModule("paper_2605_04478_amd.ccld");
  PyObject* type = module ? PyObject_GetAttrString(module, "CcldError") : nullptr;
  PyObject* error = type ? PyObject_CallFunction(type, "is", (int)f.status, f.call) : nullptr;
  if (error) PyErr_SetObject(type, error);
  Py_XDECREF(error);
  Py_XDECREF(type);
  Py_XDECREF(module);
  return nullptr;
}

// ---- the module ------------------------------------------------------------------------------------------------------
template <PyObject* (*F)(PyObject* const*), Py_ssize_t ARGS>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != ARGS) Py_RETURN_NONE;
  try {
    return F(args);
  } catch (const Declined&) {
    Py_RETURN_NONE;
  } catch (const Failed& f) {
    return raise(f);
  }
  END_HANDLE_TH_ERRORS
}
template <PyObject* (*F)(PyObject* const*), Py_ssize_t ARGS>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<F, ARGS>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<expert_product, 3>("expert_product"), method<expert_product_grad, 6>("expert_product_grad"),
                         method<vocab_loss, 3>("vocab_loss"),         method<vocab_loss_grad, 7>("vocab_loss_grad"),
                         method<norm_residual, 7>("norm_residual"),   method<norm_residual_grad, 10>("norm_residual_grad"),
                         method<route, 3>("route"),                   method<route_grad, 5>("route_grad"),
                         method<expert_order, 2>("expert_order"),     method<dispatch, 3>("dispatch"),
                         method<dispatch_grad, 2>("dispatch_grad"),   method<combine, 3>("combine"),
                         method<combine_grad, 6>("combine_grad"),     method<adamw, 9>("adamw"),
                         method<token_logprobs, 4>("token_logprobs"), method<token_logprobs_grad, 7>("token_logprobs_grad"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef definition = {PyModuleDef_HEAD_INIT, "_step", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__step() { return PyModule_Create(&definition); }
