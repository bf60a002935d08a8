// The plain calls of dropout, layer norm and the token log probabilities without an
// interpreter's steps in between: a Python call of few rows is made of these (layer norm of one
// row of 2048: 13 us with them, of which the GPU works 2.4).
//
// Each function takes the arguments of its namesake in lmzipf.py, allocates the results and
// calls the C ABI. It returns None, and has done nothing, where a call is not plain: all
// tensors torch's own, contiguous, of the right types and sizes, on the current device,
// none that autograd would record or that has a forward-mode tangent, all results to be
// allocated. lmzipf.py then goes through its own checks, which name what is wrong or take the
// call.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>

#include "../../include/lmzipf.h"

namespace {

struct {
  decltype(&lm_dropout) dropout;
  decltype(&lm_layer_norm) norm;
  decltype(&lm_layer_norm_grad_workspace_bytes) norm_grad_bytes;
  decltype(&lm_layer_norm_grad) norm_grad;
  decltype(&lm_token_logprobs_workspace_bytes) logp_bytes;
  decltype(&lm_token_logprobs) logp;
  decltype(&lm_token_logprobs_grad) logp_grad;
  decltype(&lm_status_string) status;
} lib;
PyObject* error;  // lmzipf.LmError

// Reads a call's arguments; `ok` stays true while the call is plain.
class Plain {
 public:
  Plain(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : args_(args), ok(n == want) {
    if (!ok) return;
    device_ = PyLong_AsLong(args[0]);
    stream = PyLong_AsVoidPtr(args[1]);
    records_ = c10::GradMode::is_enabled();
    tangents_ = c10::AutogradState::get_tls_state().get_fw_grad_mode();
    ok = !PyErr_Occurred();
    PyErr_Clear();
  }
  // A contiguous tensor on the current device (None: undefined).
  at::Tensor tensor(int i, bool optional = false) {
    if (!ok || (optional && args_[i] == Py_None)) return {};
    if (!(ok = THPVariable_CheckExact(args_[i]))) return {};
    const at::Tensor& t = THPVariable_Unpack(args_[i]);
    ok = t.is_cuda() && t.device().index() == device_ && t.layout() == at::kStrided &&
         t.is_contiguous() && !(records_ && t.requires_grad()) && !t.is_conj() && !t.is_neg() &&
         !(tangents_ && t._fw_grad(0).defined());  // torch has the one level
    return t;
  }
  // The matrix that a call is about: its rows, columns and dtype.
  at::Tensor matrix(int i) {
    at::Tensor t = tensor(i);
    if (!ok || !(ok = t.dim() > 0 && t.numel() > 0)) return {};
    dtype = t.scalar_type() == at::kFloat ? LM_F32 : LM_BF16;
    ok = dtype == LM_F32 || t.scalar_type() == at::kBFloat16;
    D = t.size(-1);
    rows = t.numel() / D;
    return t;
  }
  at::Tensor like(int i, const at::Tensor& x) {
    at::Tensor t = tensor(i, true);
    if (ok && t.defined()) ok = t.scalar_type() == x.scalar_type() && t.sizes() == x.sizes();
    return t;
  }
  at::Tensor floats(int i, int64_t n, bool optional = true) {
    at::Tensor t = tensor(i, optional);
    if (ok && t.defined()) ok = t.scalar_type() == at::kFloat && t.numel() == n;
    return t;
  }
  // One element.
  at::Tensor one(int i, at::ScalarType type) {
    at::Tensor t = tensor(i, true);
    if (ok && t.defined()) ok = t.scalar_type() == type && t.numel() >= 1;
    return t;
  }
  // A row's integer each.
  at::Tensor ids(int i, const at::Tensor& x) {
    at::Tensor t = tensor(i, true);
    if (ok && t.defined())
      ok = (t.scalar_type() == at::kInt || t.scalar_type() == at::kLong) &&
           t.sizes() == x.sizes().slice(0, x.dim() - 1);
    return t;
  }
  // A number or a tensor of one on the device.
  struct Seed {
    uint64_t number;
    const int64_t* at;
  };
  Seed seed(int i) {
    if (!ok) return {};
    if (PyLong_CheckExact(args_[i])) return {PyLong_AsUnsignedLongLongMask(args_[i]), nullptr};
    at::Tensor t = one(i, at::kLong);
    ok = ok && t.defined();
    return {0, ok ? t.const_data_ptr<int64_t>() : nullptr};
  }
  float real(int i) {
    if (!ok || !(ok = PyFloat_CheckExact(args_[i]) || PyLong_CheckExact(args_[i]))) return 0;
    const double x = PyFloat_AsDouble(args_[i]);
    ok = !PyErr_Occurred();
    PyErr_Clear();
    return static_cast<float>(x);
  }
  int64_t whole(int i) {
    if (!ok || !(ok = PyLong_CheckExact(args_[i]) || PyBool_Check(args_[i]))) return 0;
    const long long x = PyLong_AsLongLong(args_[i]);
    ok = !PyErr_Occurred();
    PyErr_Clear();
    return x;
  }

 private:
  PyObject* const* args_;
  long device_ = -1;
  bool records_ = true, tangents_ = true;

 public:
  bool ok;
  void* stream = nullptr;
  int64_t rows = 0, D = 0;
  int32_t dtype = 0;
};

void* at_of(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

at::Tensor make(const at::Tensor& x, at::IntArrayRef sizes, at::ScalarType type) {
  return at::empty(sizes, x.options().dtype(type));
}

// Results of a call, or its error.
template <int N>
PyObject* results(int rc, const char* what, const at::Tensor (&t)[N]) {
  if (rc != LM_OK) {
    PyErr_Format(error, "%s: %s", what, lib.status(rc));
    return nullptr;
  }
  PyObject* out = PyTuple_New(N);
  if (!out) return nullptr;
  for (int i = 0; i < N; ++i) {
    PyObject* x = t[i].defined() ? THPVariable_Wrap(t[i]) : Py_NewRef(Py_None);
    if (!x) {
      Py_DECREF(out);
      return nullptr;
    }
    PyTuple_SET_ITEM(out, i, x);
  }
  return out;
}

#define NOT_PLAIN(p) \
  if (!(p).ok) Py_RETURN_NONE

// (device, stream, x, p, seed, add)
PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Plain c(args, n, 6);
  const at::Tensor x = c.matrix(2);
  const float p = c.real(3);
  const auto seed = c.seed(4);
  const at::Tensor add = c.like(5, x);
  NOT_PLAIN(c);
  const at::Tensor out = at::empty_like(x);
  const int rc = lib.dropout(x.data_ptr(), c.D, at_of(add), c.D, out.data_ptr(), c.D, c.rows, c.D,
                             c.dtype, p, seed.number, seed.at, c.stream);
  return results<1>(rc, "lm_dropout", {out});
  END_HANDLE_TH_ERRORS
}

// (device, stream, x, weight, bias, eps, add, p, seed): y, h, mean, rstd
PyObject* layer_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Plain c(args, n, 9);
  const at::Tensor x = c.matrix(2);
  const at::Tensor weight = c.floats(3, c.D), bias = c.floats(4, c.D);
  const float eps = c.real(5);
  const at::Tensor add = c.like(6, x);
  const float p = c.real(7);
  const auto seed = c.seed(8);
  NOT_PLAIN(c);
  const bool changed = add.defined() || p > 0;
  const at::Tensor y = at::empty_like(x), h = changed ? at::empty_like(x) : at::Tensor();
  const auto lead = x.sizes().slice(0, x.dim() - 1);
  const at::Tensor mean = make(x, lead, at::kFloat), rstd = make(x, lead, at::kFloat);
  const int rc = lib.norm(x.data_ptr(), c.D, at_of(add), c.D, c.rows, c.D, c.dtype,
                          static_cast<const float*>(at_of(weight)),
                          static_cast<const float*>(at_of(bias)), eps, p, seed.number, seed.at,
                          y.data_ptr(), c.D, at_of(h), c.D, mean.data_ptr<float>(),
                          rstd.data_ptr<float>(), c.stream);
  return results<4>(rc, "lm_layer_norm", {y, changed ? h : x, mean, rstd});
  END_HANDLE_TH_ERRORS
}

// (device, stream, dy, h, mean, rstd, weight, add, p, seed, bias): dh, dx, dweight, dbias
PyObject* layer_norm_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Plain c(args, n, 11);
  const at::Tensor dy = c.matrix(2), h = c.like(3, dy);
  const at::Tensor mean = c.floats(4, c.rows, false), rstd = c.floats(5, c.rows, false);
  const at::Tensor weight = c.floats(6, c.D), add = c.like(7, dy);
  const float p = c.real(8);
  const auto seed = c.seed(9);
  const bool bias = c.ok && args[10] == Py_None ? weight.defined() : c.whole(10) != 0;
  c.ok = c.ok && h.defined();
  NOT_PLAIN(c);
  const at::Tensor dh = at::empty_like(dy), dx = p > 0 ? at::empty_like(dy) : at::Tensor();
  at::Tensor dw, db, ws;
  if (weight.defined()) dw = make(dy, {c.D}, at::kFloat);
  if (bias) db = make(dy, {c.D}, at::kFloat);
  size_t need = 0;
  if (dw.defined() || db.defined()) {
    need = lib.norm_grad_bytes(c.rows, c.D, c.dtype);
    if (need) ws = make(dy, {static_cast<int64_t>(need)}, at::kByte);
  }
  const int rc = lib.norm_grad(
      dy.data_ptr(), c.D, h.data_ptr(), c.D, at_of(add), c.D, c.rows, c.D, c.dtype,
      mean.data_ptr<float>(), rstd.data_ptr<float>(), static_cast<const float*>(at_of(weight)), p,
      seed.number, seed.at, dh.data_ptr(), c.D, at_of(dx), c.D, static_cast<float*>(at_of(dw)),
      static_cast<float*>(at_of(db)), 0, at_of(ws), need, c.stream);
  return results<4>(rc, "lm_layer_norm_grad", {dh, dx.defined() ? dx : dh, dw, db});
  END_HANDLE_TH_ERRORS
}

// (device, stream, logits, targets, scale, top, ignore, dev_err):
// logp, entropy, peak, log_sum, top_logp, top_ids
PyObject* token_logprobs(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Plain c(args, n, 8);
  const at::Tensor x = c.matrix(2), targets = c.ids(3, x);
  const float scale = c.real(4);
  const int64_t top = c.whole(5), ignore = c.whole(6);
  const at::Tensor err = c.one(7, at::kInt);
  c.ok = c.ok && top >= 0 && top <= LM_TOP_MAX;
  NOT_PLAIN(c);
  const auto lead = x.sizes().slice(0, x.dim() - 1);
  at::Tensor logp, top_logp, top_ids, ws;
  if (targets.defined()) logp = make(x, lead, at::kFloat);
  const at::Tensor entropy = make(x, lead, at::kFloat), peak = make(x, lead, at::kFloat),
                   log_sum = make(x, lead, at::kFloat);
  if (top) {
    at::DimVector sizes(lead.begin(), lead.end());
    sizes.push_back(top);
    top_logp = make(x, sizes, at::kFloat);
    top_ids = make(x, sizes, at::kInt);
  }
  const size_t need = lib.logp_bytes(c.rows, c.D, c.dtype, static_cast<int32_t>(top));
  if (need) ws = make(x, {static_cast<int64_t>(need)}, at::kByte);
  const bool wide = targets.defined() && targets.scalar_type() == at::kLong;
  const int rc = lib.logp(x.data_ptr(), c.D, c.rows, c.D, c.dtype, at_of(targets),
                          wide ? LM_I64 : LM_I32, ignore, scale, static_cast<int32_t>(top),
                          static_cast<float*>(at_of(logp)), entropy.data_ptr<float>(),
                          peak.data_ptr<float>(), log_sum.data_ptr<float>(),
                          static_cast<float*>(at_of(top_logp)),
                          static_cast<int32_t*>(at_of(top_ids)), static_cast<int32_t*>(at_of(err)),
                          at_of(ws), need, c.stream);
  return results<6>(rc, "lm_token_logprobs", {logp, entropy, peak, log_sum, top_logp, top_ids});
  END_HANDLE_TH_ERRORS
}

// (device, stream, logits, targets, peak, log_sum, dlogp, entropy, dentropy, scale, ignore): out
PyObject* token_logprobs_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Plain c(args, n, 11);
  const at::Tensor x = c.matrix(2), targets = c.ids(3, x);
  const at::Tensor peak = c.floats(4, c.rows, false), log_sum = c.floats(5, c.rows, false);
  const at::Tensor dlogp = c.floats(6, c.rows), entropy = c.floats(7, c.rows);
  const at::Tensor dentropy = c.floats(8, c.rows);
  const float scale = c.real(9);
  const int64_t ignore = c.whole(10);
  c.ok = c.ok && (targets.defined() || !dlogp.defined()) &&
         (entropy.defined() || !dentropy.defined());
  NOT_PLAIN(c);
  const at::Tensor out = at::empty_like(x);
  const bool wide = targets.defined() && targets.scalar_type() == at::kLong;
  const int rc = lib.logp_grad(
      x.data_ptr(), c.D, c.rows, c.D, c.dtype, at_of(targets), wide ? LM_I64 : LM_I32, ignore,
      scale, peak.data_ptr<float>(), log_sum.data_ptr<float>(),
      static_cast<const float*>(at_of(dlogp)), static_cast<const float*>(at_of(entropy)),
      static_cast<const float*>(at_of(dentropy)), out.data_ptr(), c.D, c.stream);
  return results<1>(rc, "lm_token_logprobs_grad", {out});
  END_HANDLE_TH_ERRORS
}

// (LmError, the addresses of the library's functions in the order of `lib`)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr int kFunctions = sizeof(lib) / sizeof(void*);
  if (n != kFunctions + 1) {
    PyErr_SetString(PyExc_TypeError, "bind: an exception and every function's address");
    return nullptr;
  }
  void* at[kFunctions];
  for (int i = 0; i < kFunctions; ++i) {
    at[i] = PyLong_AsVoidPtr(args[i + 1]);
    if (!at[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: a function has no address");
      return nullptr;
    }
  }
  Py_INCREF(args[0]);
  Py_XDECREF(error);
  error = args[0];
  static_assert(sizeof(at) == sizeof(lib), "function pointers");
  memcpy(&lib, at, sizeof(at));
  Py_RETURN_NONE;
}

#define METHOD(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}

PyMethodDef methods[] = {METHOD(bind),
                         METHOD(dropout),
                         METHOD(layer_norm),
                         METHOD(layer_norm_grad),
                         METHOD(token_logprobs),
                         METHOD(token_logprobs_grad),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lmzipf_calls", nullptr, -1, methods,
                      nullptr,               nullptr,         nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lmzipf_calls() { return PyModule_Create(&module); }
