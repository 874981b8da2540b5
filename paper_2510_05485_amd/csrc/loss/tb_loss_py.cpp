// Host side of a loss called from Python: checks the tensors, fills in the C ABI's structs, allocates
// outputs and workspace and calls the library, in one step.  Like tb_host.cpp: every function returns
// None for whatever is not the plain case, and the general way in losses.py then converts, or raises the
// error that says what is wrong.  A policy loss on 16 x 32 positions, 18 us of work for the GPU, took 40 us
// a call with the marshalling in Python; one token's log-probability 14.9, and 5.2 so.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>
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
  const at::Tensor *tokens = nullptr, *lengths = nullptr, *mask = nullptr;
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
  bool take_rows(const at::Tensor* t) {
    x = t;
    if (!x || !x->is_cuda() || x->layout() != at::kStrided || (x->dim() != 2 && x->dim() != 3)) return false;
    if (!type_of(x->scalar_type(), &logits.type) || x->_fw_grad(0).defined()) return false;
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
    return true;
  }
  bool take_tokens(const at::Tensor* t) {
    if (!here(t) || !id_type(t->scalar_type()) || t->dim() != x->dim() - 1 || t->size(-1) != logits.T ||
        (!packed && t->size(0) != logits.B) || (logits.T > 1 && t->stride(-1) != 1))
      return false;
    tokens = t;
    at.tokens = t->data_ptr();
    at.token_stride = packed ? logits.T : t->stride(0);
    at.token_bytes = t->scalar_type() == at::kLong ? 8 : 4;
    return true;
  }
  bool take_lengths(const at::Tensor* t) {
    if (packed || !here(t) || t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != logits.B ||
        !t->is_contiguous())
      return false;
    lengths = t;
    at.lengths = t->data_ptr<int32_t>();
    return true;
  }
  bool take_mask(const at::Tensor* t) {
    if (!here(t) || (t->scalar_type() != at::kBool && t->scalar_type() != at::kByte) || t->dim() != x->dim() - 1 ||
        t->size(-1) != logits.T || (!packed && t->size(0) != logits.B) || !t->is_contiguous())
      return false;
    mask = t;
    at.mask = static_cast<const uint8_t*>(t->data_ptr());
    return true;
  }
  // a teacher's entries of all positions
  bool take_teacher(const at::Tensor* ids, const at::Tensor* t, tb_teacher_t* q) const {
    if (!here(ids) || !here(t) || !id_type(ids->scalar_type()) || !type_of(t->scalar_type(), &q->type) ||
        ids->dim() != x->dim() || ids->sizes() != t->sizes() || !ids->is_contiguous() || !t->is_contiguous() ||
        ids->sizes().slice(0, ids->dim() - 1) != positions() || ids->size(-1) > TB_TEACHER_MOST)
      return false;
    q->ids = ids->data_ptr();
    q->logits = t->data_ptr();
    q->id_bytes = ids->scalar_type() == at::kLong ? 8 : 4;
    q->K = int32_t(ids->size(-1));
    return true;
  }
  bool take(PyObject* logits_, PyObject* tokens_, PyObject* lengths_, PyObject* mask_, PyObject* temperature_,
            PyObject* status_) {
    if (!take_float(temperature_, &logits.temperature) || !take_rows(tensor(logits_))) return false;
    if (tokens_ && !take_tokens(tensor(tokens_))) return false;
    if (lengths_ != Py_None && !take_lengths(tensor(lengths_))) return false;
    if (mask_ != Py_None && !take_mask(tensor(mask_))) return false;
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
  at::Tensor row_state() const { return values({logits.B, logits.T, TB_ROW_STATE}); }
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

// The backward pass of all operators: the gradient of rows whose statistics and cotangents the forward
// pass has left.  Incoming gradients are of the log-probabilities and entropies themselves (kValues), or
// of a scalar loss that `d_lp`, `d_entropy` are the cotangents of.  Everything that the kernels read comes from
// the saved tensors as they are unpacked: where hooks are active (checkpointing, offloading), these are other
// tensors than the forward pass's, whose memory may be gone, and their strides may be others.
struct RowsBackward : public torch::autograd::Node {
  using Saved = torch::autograd::SavedVariable;
  enum Kind { kValues, kLoss, kSequences, kDistill } kind;
  tb_logits_t logits_of;  // (shape, type and temperature)
  int32_t average = 0;    // of a distillation
  int64_t dims;
  Saved logits, tokens, lengths, mask, state, d_lp, d_entropy, ids, teacher_logits;

  static Saved kept(const at::Tensor* t) { return t && t->defined() ? Saved(*t, false) : Saved(); }
  RowsBackward(Kind k, const Call& c, const at::Tensor& row_state) : kind(k), logits_of(c.logits), dims(c.x->dim()) {
    logits = kept(c.x);
    tokens = kept(c.tokens);
    lengths = kept(c.lengths);
    mask = kept(c.mask);
    state = kept(&row_state);
    set_next_edges(torch::autograd::collect_next_edges(*c.x));
  }
  static constexpr const char* kHooks =
      "a tensor saved for the losses' backward pass has come back from its hooks with another shape, type or device";
  std::string name() const override { return "TensorLossBackward"; }
  void release_variables() override {
    std::lock_guard<std::mutex> lock(mutex_);
    for (Saved* s : {&logits, &tokens, &lengths, &mask, &state, &d_lp, &d_entropy, &ids, &teacher_logits}) s->reset_data();
  }
  torch::autograd::variable_list apply(torch::autograd::variable_list&& in) override {
    std::lock_guard<std::mutex> lock(mutex_);
    TORCH_CHECK(!at::GradMode::is_enabled(), "the losses over logits cannot be differentiated twice");
    if (!in[0].defined() && (in.size() < 2 || !in[1].defined())) return {at::Tensor()};
    // (unpacking checks that nothing has been written over since)
    auto rows = [](const at::Tensor& t) {
      return t.defined() && t.dim() > 0 && t.stride(-1) != 1 && t.size(-1) > 1 ? t.contiguous() : t;
    };
    auto whole = [](const at::Tensor& t) { return t.defined() ? t.contiguous() : t; };
    const at::Tensor x = rows(logits.unpack()), ids_of_rows = rows(tokens.unpack()), n = whole(lengths.unpack()),
                     m = whole(mask.unpack()), s = whole(state.unpack());
    at::Tensor d = whole(d_lp.unpack()), dh = whole(d_entropy.unpack()), up;
    const c10::OptionalDeviceGuard guard(x.device());
    Call c;
    c.logits.temperature = logits_of.temperature;
    bool alike = x.dim() == dims && c.take_rows(&x) && c.logits.B == logits_of.B && c.logits.T == logits_of.T &&
                 c.logits.V == logits_of.V && c.logits.type == logits_of.type;
    auto values = [&](const at::Tensor& t, int64_t count) {
      return c.here(&t) && t.scalar_type() == at::kFloat && t.numel() == count;
    };
    const int64_t count = int64_t(logits_of.B) * logits_of.T;
    alike = alike && (!ids_of_rows.defined() || c.take_tokens(&ids_of_rows)) && (!n.defined() || c.take_lengths(&n)) &&
            (!m.defined() || c.take_mask(&m)) && values(s, TB_ROW_STATE * count) &&
            (!d.defined() || values(d, kind == kSequences ? logits_of.B : count)) && (!dh.defined() || values(dh, count));
    TORCH_CHECK(alike, kHooks);
    if (kind == kValues) {
      if (in[0].defined()) d = in[0].to(at::kFloat).contiguous();
      if (in.size() > 1 && in[1].defined()) dh = in[1].to(at::kFloat).contiguous();
      if (!d.defined()) d = at::zeros_like(dh);
    } else {
      up = in[0].to(at::kFloat).contiguous();
    }
    at::Tensor out = at::empty(x.sizes(), x.options().requires_grad(false));
    tb_gradient_t g = {out.data_ptr(), x.dim() == 2 ? 0 : out.stride(0), out.stride(x.dim() - 2), 1.f};
    const float* upstream = up.defined() ? up.data_ptr<float>() : nullptr;
    int rc;
    if (kind == kDistill) {
      const at::Tensor i = whole(ids.unpack()), q = whole(teacher_logits.unpack());
      tb_teacher_t teacher = {};
      TORCH_CHECK(c.take_teacher(&i, &q, &teacher), kHooks);
      teacher.average = average;
      rc = tensorloss_distill_grad(&c.logits, &c.at, &teacher, s.data_ptr<float>(), d.data_ptr<float>(), upstream, &g,
                                   c.stream);
    } else {
      const bool each = kind != kSequences;
      rc = tensorloss_token_logprobs_grad(&c.logits, &c.at, s.data_ptr<float>(), d.data_ptr<float>(),
                                          dh.defined() ? dh.data_ptr<float>() : nullptr, each ? logits_of.T : 1, each,
                                          upstream, &g, c.stream);
    }
    TORCH_CHECK(rc == TB_OK, "tensorloss gradient: ", tensorbleu_status_string(rc));
    return {out};
  }
};
std::shared_ptr<RowsBackward> backward_of(RowsBackward::Kind kind, const Call& c, const at::Tensor& state) {
  return std::shared_ptr<RowsBackward>(new RowsBackward(kind, c, state), torch::autograd::deleteNode);
}
bool differentiated(const at::Tensor& x) { return at::GradMode::is_enabled() && x.requires_grad(); }
// A caller's tensor has been written over: torch notices it where the tensor, or one that shares its memory, is
// saved for a backward pass.  (Tensors of inference mode count no versions and are not saved.)
void written(PyObject* out, const at::Tensor& t) {
  if (out != Py_None && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// the loss, terms[0], as a tensor of its own that shares its memory
at::Tensor first_of(const at::Tensor& terms) {
  at::AutoDispatchBelowADInplaceOrView guard;
  return terms.select(0, 0);
}

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
  const int wanted = PyObject_IsTrue(args[6]);
  if (wanted < 0) return nullptr;
  const bool entropy = wanted;
  at::Tensor lp = c.values(c.positions()), h, state;
  if (entropy) h = c.values(c.positions());
  const bool backward = differentiated(*c.x);
  if (backward) state = c.row_state();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorloss_token_logprobs(&c.logits, &c.at, lp.data_ptr<float>(), entropy ? h.data_ptr<float>() : nullptr,
                                 backward ? state.data_ptr<float>() : nullptr, c.status, c.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  if (backward) {
    auto node = backward_of(RowsBackward::kValues, c, state);
    torch::autograd::set_history(lp, node);
    if (entropy) torch::autograd::set_history(h, node);
  }
  if (!entropy) return THPVariable_Wrap(std::move(lp));
  return results({lp, h}, Py_None, -1);
}

// policy(logits, tokens, lengths, mask, temperature, status, out, grad_scale, old_logprobs, advantages,
// ref_logprobs, clip_low, clip_high, kl_coef, entropy_coef, average): (terms, gradient, logprobs) or None;
// grad_scale None: the loss, for torch to differentiate, and out is not used
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
  const bool scalar = args[7] == Py_None, backward = scalar && differentiated(*c.x), bonus = p.entropy_coef != 0.f;
  at::Tensor out, state, d_lp, d_entropy;
  tb_gradient_t g = {};
  if (!scalar && !c.gradient(args[6], args[7], &out, &g)) Py_RETURN_NONE;
  if (backward) {
    state = c.row_state();
    d_lp = c.values(c.positions());
    if (bonus) d_entropy = c.values(c.positions());
  }
  at::Tensor terms = c.values({4}), lp = c.values(c.positions());
  size_t bytes;
  at::Tensor workspace = c.workspace(&bytes);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorloss_policy(&c.logits, &c.at, &p, scalar ? nullptr : &g, terms.data_ptr<float>(), lp.data_ptr<float>(),
                         backward ? state.data_ptr<float>() : nullptr, backward ? d_lp.data_ptr<float>() : nullptr,
                         backward && bonus ? d_entropy.data_ptr<float>() : nullptr, c.status, workspace.data_ptr(), bytes,
                         c.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  if (scalar) {
    at::Tensor loss = first_of(terms);
    if (backward) {
      auto node = backward_of(RowsBackward::kLoss, c, state);
      node->d_lp = RowsBackward::kept(&d_lp);
      node->d_entropy = RowsBackward::kept(&d_entropy);
      torch::autograd::set_history(loss, node);
    }
    return THPVariable_Wrap(std::move(loss));
  }
  written(args[6], out);
  return results({terms, out, lp}, args[6], 1);
}

// preference(logits, tokens, lengths, mask, temperature, status, out, grad_scale, ref_logprobs, beta, kind,
// label_smoothing): (terms, gradient, sequence log-probabilities, margins) or None; grad_scale None: the loss
PyObject* preference(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Call c;
  if (n != 12 || !c.take(args[0], args[1], args[2], args[3], args[4], args[5]) || c.packed) Py_RETURN_NONE;
  tb_preference_t p = {};
  if (!c.over_positions(args[8], &p.ref_logprobs) || !take_float(args[9], &p.beta) || !take_int(args[10], &p.kind) ||
      !take_float(args[11], &p.label_smoothing))
    Py_RETURN_NONE;
  const bool scalar = args[7] == Py_None, backward = scalar && differentiated(*c.x);
  at::Tensor out, state, d_sequence;
  tb_gradient_t g = {};
  if (!scalar && !c.gradient(args[6], args[7], &out, &g)) Py_RETURN_NONE;
  if (backward) {
    state = c.row_state();
    d_sequence = c.values({c.logits.B});
  }
  at::Tensor terms = c.values({3}), sums = c.values({c.logits.B}), margins = c.values({c.logits.B / 2});
  size_t bytes;
  at::Tensor workspace = c.workspace(&bytes);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorloss_preference(&c.logits, &c.at, &p, scalar ? nullptr : &g, terms.data_ptr<float>(), sums.data_ptr<float>(),
                             margins.data_ptr<float>(), backward ? state.data_ptr<float>() : nullptr,
                             backward ? d_sequence.data_ptr<float>() : nullptr, c.status, workspace.data_ptr(), bytes,
                             c.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  if (scalar) {
    at::Tensor loss = first_of(terms);
    if (backward) {
      auto node = backward_of(RowsBackward::kSequences, c, state);
      node->d_lp = RowsBackward::kept(&d_sequence);
      torch::autograd::set_history(loss, node);
    }
    return THPVariable_Wrap(std::move(loss));
  }
  written(args[6], out);
  return results({terms, out, sums, margins}, args[6], 1);
}

// distill(logits, lengths, mask, temperature, status, out, grad_scale, teacher_ids, teacher_logits, average):
// (terms, gradient, row losses) or None; grad_scale None: the loss
PyObject* distill(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Call c;
  if (n != 10 || !c.take(args[0], nullptr, args[1], args[2], args[3], args[4])) Py_RETURN_NONE;
  const at::Tensor *ids = tensor(args[7]), *t = tensor(args[8]);
  tb_teacher_t q = {};
  if (!c.take_teacher(ids, t, &q) || !take_int(args[9], &q.average)) Py_RETURN_NONE;
  const bool scalar = args[6] == Py_None, backward = scalar && differentiated(*c.x);
  at::Tensor out, state, d_row;
  tb_gradient_t g = {};
  if (!scalar && !c.gradient(args[5], args[6], &out, &g)) Py_RETURN_NONE;
  if (backward) {
    state = c.row_state();
    d_row = c.values(c.positions());
  }
  at::Tensor terms = c.values({1}), rows = c.values(c.positions());
  size_t bytes;
  at::Tensor workspace = c.workspace(&bytes);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorloss_distill(&c.logits, &c.at, &q, scalar ? nullptr : &g, terms.data_ptr<float>(), rows.data_ptr<float>(),
                          backward ? state.data_ptr<float>() : nullptr, backward ? d_row.data_ptr<float>() : nullptr,
                          c.status, workspace.data_ptr(), bytes, c.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  if (scalar) {
    at::Tensor loss = first_of(terms);
    if (backward) {
      auto node = backward_of(RowsBackward::kDistill, c, state);
      node->d_lp = RowsBackward::kept(&d_row);
      node->ids = RowsBackward::kept(ids);
      node->teacher_logits = RowsBackward::kept(t);
      node->average = q.average;
      torch::autograd::set_history(loss, node);
    }
    return THPVariable_Wrap(std::move(loss));
  }
  written(args[5], out);
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
