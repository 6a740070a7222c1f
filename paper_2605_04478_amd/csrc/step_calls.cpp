// Calls of the training step's operators from Python, for tensors that are as they should be (module _step).
//
// A small operator is bound by the host: checks, outputs and arguments of a norm take 15 us in Python and 3 here, its kernel 3.  These
// functions have the arguments of their namesakes in step.py, which describes them.  They return what those return, or None where anything is out
// of the ordinary (a tensor of another shape, type, device or layout, a refusal of the library's): nothing has been enqueued then,
// and step.py, which knows how to lay tensors out and what to say of wrong ones, makes the call.  A failure of the device's raises what step.py
// raises: work may have been enqueued.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ops/empty.h>
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
  Tensor empty(at::IntArrayRef shape, at::ScalarType type) const { return at::empty(shape, at::TensorOptions().dtype(type).device(device)); }
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
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef definition = {PyModuleDef_HEAD_INIT, "_step", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__step() { return PyModule_Create(&definition); }
