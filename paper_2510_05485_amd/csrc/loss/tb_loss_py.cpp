// Host side of a loss called from Python: checks the tensors, fills in the C ABI's structs, allocates
// outputs and workspace and calls the library, in one step.  Like tb_host.cpp: every function returns
// None for whatever is not the plain case, and the general way in losses.py then converts, or raises the
// error that says what is wrong.  A policy loss on 16 x 32 positions takes the GPU 20 us; marshalling it
// in Python took the host 33 us, here it takes 9 with its two launches.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>

#include "tensorloss.h"

namespace {

const at::Tensor* tensor(PyObject* o) {
  return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
}
bool type_of(at::ScalarType s, int32_t* type) {
  *type = s == at::kFloat ? TB_FLOAT32 : s == at::kBFloat16 ? TB_BFLOAT16 : TB_FLOAT16;
  return s == at::kFloat || s == at::kBFloat16 || s == at::kHalf;
}
bool id_type(at::ScalarType s) { return s == at::kInt || s == at::kLong; }
bool take_float(PyObject* o, float* to) {
  if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
  const double v = PyFloat_AsDouble(o);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *to = float(v);
  return true;
}
bool take_int(PyObject* o, int32_t* to) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  *to = int32_t(v);
  return !overflow && v == *to;
}

// Logits, tokens, lengths, mask, temperature and status of a call; tokens may be null (None).
struct Call {
  const at::Tensor* x = nullptr;
  tb_logits_t logits = {};
  tb_positions_t at = {};
  bool packed = false;
  int32_t* status = nullptr;
  void* stream = nullptr;

  bool here(const at::Tensor* t) const {
    return t && t->layout() == at::kStrided && t->is_cuda() && t->device() == x->device();
  }
  // a contiguous float32 tensor over the positions
  bool over_positions(PyObject* o, const float** to) const {
    const at::Tensor* t = tensor(o);
    if (!here(t) || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->dim() != x->dim() - 1) return false;
    for (int64_t i = 0; i < t->dim(); ++i)
      if (t->size(i) != x->size(i)) return false;
    *to = t->data_ptr<float>();
    return true;
  }
  bool take(PyObject* logits_, PyObject* tokens_, PyObject* lengths_, PyObject* mask_, PyObject* temperature_,
            PyObject* status_) {
    x = tensor(logits_);
    if (!x || !x->is_cuda() || x->layout() != at::kStrided || (x->dim() != 2 && x->dim() != 3)) return false;
    if (!type_of(x->scalar_type(), &logits.type) || !take_float(temperature_, &logits.temperature)) return false;
    const auto s = c10::hip::getCurrentHIPStream();
    if (s.device_index() != x->device().index()) return false;
    stream = static_cast<void*>(s.stream());
    packed = x->dim() == 2;
    const int64_t B = packed ? 1 : x->size(0), T = x->size(packed ? 0 : 1), V = x->size(-1);
    if (V < 1 || V > INT32_MAX || B > INT32_MAX || T > INT32_MAX || (V > 1 && x->stride(-1) != 1)) return false;
    logits.data = x->data_ptr();
    logits.seq_stride = packed ? 0 : x->stride(0);
    logits.pos_stride = x->stride(packed ? 0 : 1);
    logits.B = int32_t(B);
    logits.T = int32_t(T);
    logits.V = int32_t(V);
    if (tokens_) {
      const at::Tensor* t = tensor(tokens_);
      if (!here(t) || !id_type(t->scalar_type()) || t->dim() != x->dim() - 1 || t->size(-1) != T ||
          (!packed && t->size(0) != B) || (T > 1 && t->stride(-1) != 1))
        return false;
      at.tokens = t->data_ptr();
      at.token_stride = packed ? T : t->stride(0);
      at.token_bytes = t->scalar_type() == at::kLong ? 8 : 4;
    }
    if (lengths_ != Py_None) {
      const at::Tensor* t = tensor(lengths_);
      if (packed || !here(t) || t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != B || !t->is_contiguous())
        return false;
      at.lengths = t->data_ptr<int32_t>();
    }
    if (mask_ != Py_None) {
      const at::Tensor* t = tensor(mask_);
      if (!here(t) || (t->scalar_type() != at::kBool && t->scalar_type() != at::kByte) || t->dim() != x->dim() - 1 ||
          t->size(-1) != T || (!packed && t->size(0) != B) || !t->is_contiguous())
        return false;
      at.mask = static_cast<const uint8_t*>(t->data_ptr());
    }
    if (status_ != Py_None) {
      const at::Tensor* t = tensor(status_);
      if (!here(t) || t->scalar_type() != at::kInt || t->numel() != 1) return false;
      status = t->data_ptr<int32_t>();
    }
    return true;
  }
  at::Tensor values(at::IntArrayRef shape) const {
    return at::empty(shape, at::TensorOptions().dtype(at::kFloat).device(x->device()));
  }
  at::IntArrayRef positions() const { return x->sizes().slice(0, x->dim() - 1); }
  at::Tensor workspace(size_t* bytes) const {
    *bytes = tensorloss_workspace_bytes(logits.B, logits.T);
    return at::empty({int64_t(*bytes)}, at::TensorOptions().dtype(at::kByte).device(x->device()));
  }
  // the gradient's tensor: the caller's, or a new one
  bool gradient(PyObject* out, PyObject* scale, at::Tensor* to, tb_gradient_t* g) const {
    if (!take_float(scale, &g->scale)) return false;
    if (out == Py_None) {
      *to = at::empty(x->sizes(), x->options().requires_grad(false));
    } else {
      const at::Tensor* t = tensor(out);
      if (!here(t) || t->scalar_type() != x->scalar_type() || t->sizes() != x->sizes() || t->requires_grad() ||
          (logits.V > 1 && t->stride(-1) != 1))
        return false;
      *to = *t;
    }
    g->data = to->data_ptr();
    g->seq_stride = packed ? 0 : to->stride(0);
    g->pos_stride = to->stride(packed ? 0 : 1);
    return true;
  }
};

PyObject* results(std::initializer_list<at::Tensor> all, PyObject* out, int out_at) {
  PyObject* tuple = PyTuple_New(Py_ssize_t(all.size()));
  if (!tuple) return nullptr;
  int i = 0;
  for (const at::Tensor& t : all) {
    PyObject* o;
    if (i == out_at && out != Py_None) {
      Py_INCREF(out);
      o = out;
    } else {
      o = THPVariable_Wrap(t);
    }
    if (!o) {
      Py_DECREF(tuple);
      return nullptr;
    }
    PyTuple_SET_ITEM(tuple, i++, o);
  }
  return tuple;
}

// logprobs(logits, tokens, lengths, mask, temperature, status, want_entropy): tensor, (tensor, tensor) or None
PyObject* logprobs(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Call c;
  if (n != 7 || !c.take(args[0], args[1], args[2], args[3], args[4], args[5])) Py_RETURN_NONE;
  const bool entropy = args[6] == Py_True;
  at::Tensor lp = c.values(c.positions()), h;
  if (entropy) h = c.values(c.positions());
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorloss_token_logprobs(&c.logits, &c.at, lp.data_ptr<float>(), entropy ? h.data_ptr<float>() : nullptr, nullptr,
                                 c.status, c.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  if (!entropy) return THPVariable_Wrap(std::move(lp));
  return results({lp, h}, Py_None, -1);
}

// policy(logits, tokens, lengths, mask, temperature, status, out, grad_scale, old_logprobs, advantages,
// ref_logprobs, clip_low, clip_high, kl_coef, entropy_coef, average): (terms, gradient, logprobs) or None
PyObject* policy(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Call c;
  if (n != 16 || !c.take(args[0], args[1], args[2], args[3], args[4], args[5])) Py_RETURN_NONE;
  tb_policy_t p = {};
  if (!c.over_positions(args[8], &p.old_logprobs) || !take_float(args[11], &p.clip_low) ||
      !take_float(args[12], &p.clip_high) || !take_float(args[13], &p.kl_coef) ||
      !take_float(args[14], &p.entropy_coef) || !take_int(args[15], &p.average))
    Py_RETURN_NONE;
  if (args[10] != Py_None && !c.over_positions(args[10], &p.ref_logprobs)) Py_RETURN_NONE;
  const at::Tensor* a = tensor(args[9]);
  if (!c.here(a)) Py_RETURN_NONE;
  p.each = c.packed || a->dim() == 2;
  if (p.each) {
    if (!c.over_positions(args[9], &p.advantages)) Py_RETURN_NONE;
  } else {
    if (a->dim() != 1 || a->size(0) != c.logits.B || a->scalar_type() != at::kFloat || !a->is_contiguous()) Py_RETURN_NONE;
    p.advantages = a->data_ptr<float>();
  }
  at::Tensor out;
  tb_gradient_t g = {};
  if (!c.gradient(args[6], args[7], &out, &g)) Py_RETURN_NONE;
  at::Tensor terms = c.values({4}), lp = c.values(c.positions());
  size_t bytes;
  at::Tensor workspace = c.workspace(&bytes);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorloss_policy(&c.logits, &c.at, &p, &g, terms.data_ptr<float>(), lp.data_ptr<float>(), nullptr, nullptr,
                         nullptr, c.status, workspace.data_ptr(), bytes, c.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  return results({terms, out, lp}, args[6], 1);
}

// preference(logits, tokens, lengths, mask, temperature, status, out, grad_scale, ref_logprobs, beta, kind,
// label_smoothing): (terms, gradient, sequence log-probabilities, margins) or None
PyObject* preference(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Call c;
  if (n != 12 || !c.take(args[0], args[1], args[2], args[3], args[4], args[5]) || c.packed) Py_RETURN_NONE;
  tb_preference_t p = {};
  if (!c.over_positions(args[8], &p.ref_logprobs) || !take_float(args[9], &p.beta) || !take_int(args[10], &p.kind) ||
      !take_float(args[11], &p.label_smoothing))
    Py_RETURN_NONE;
  at::Tensor out;
  tb_gradient_t g = {};
  if (!c.gradient(args[6], args[7], &out, &g)) Py_RETURN_NONE;
  at::Tensor terms = c.values({3}), sums = c.values({c.logits.B}), margins = c.values({c.logits.B / 2});
  size_t bytes;
  at::Tensor workspace = c.workspace(&bytes);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorloss_preference(&c.logits, &c.at, &p, &g, terms.data_ptr<float>(), sums.data_ptr<float>(),
                             margins.data_ptr<float>(), nullptr, nullptr, c.status, workspace.data_ptr(), bytes, c.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  return results({terms, out, sums, margins}, args[6], 1);
}

// distill(logits, lengths, mask, temperature, status, out, grad_scale, teacher_ids, teacher_logits, average):
// (terms, gradient, row losses) or None
PyObject* distill(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Call c;
  if (n != 10 || !c.take(args[0], nullptr, args[1], args[2], args[3], args[4])) Py_RETURN_NONE;
  const at::Tensor *ids = tensor(args[7]), *t = tensor(args[8]);
  tb_teacher_t q = {};
  if (!c.here(ids) || !c.here(t) || !id_type(ids->scalar_type()) || !type_of(t->scalar_type(), &q.type) ||
      ids->dim() != c.x->dim() || ids->sizes() != t->sizes() || !ids->is_contiguous() || !t->is_contiguous() ||
      ids->sizes().slice(0, ids->dim() - 1) != c.positions() || ids->size(-1) > TB_TEACHER_MOST ||
      !take_int(args[9], &q.average))
    Py_RETURN_NONE;
  q.ids = ids->data_ptr();
  q.logits = t->data_ptr();
  q.id_bytes = ids->scalar_type() == at::kLong ? 8 : 4;
  q.K = int32_t(ids->size(-1));
  at::Tensor out;
  tb_gradient_t g = {};
  if (!c.gradient(args[5], args[6], &out, &g)) Py_RETURN_NONE;
  at::Tensor terms = c.values({1}), rows = c.values(c.positions());
  size_t bytes;
  at::Tensor workspace = c.workspace(&bytes);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorloss_distill(&c.logits, &c.at, &q, &g, terms.data_ptr<float>(), rows.data_ptr<float>(), nullptr, nullptr,
                          c.status, workspace.data_ptr(), bytes, c.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  return results({terms, out, rows}, args[5], 1);
}

// at:: functions throw (out of memory): to Python as the exceptions that torch itself raises
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return F(self, args, n);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"logprobs", reinterpret_cast<PyCFunction>(guarded<logprobs>), METH_FASTCALL, nullptr},
    {"policy", reinterpret_cast<PyCFunction>(guarded<policy>), METH_FASTCALL, nullptr},
    {"preference", reinterpret_cast<PyCFunction>(guarded<preference>), METH_FASTCALL, nullptr},
    {"distill", reinterpret_cast<PyCFunction>(guarded<distill>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_loss_host", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__loss_host(void) { return PyModule_Create(&module); }
