// Host side of an embedding called from Python, like ../loss/tb_loss_py.cpp: checks the tensors, fills in the C ABI's
// structs, allocates and calls the library in one step.  Every function returns None for whatever is not the plain
// case, and the general way in embeddings.py then converts, or raises the error that says what is wrong.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <ATen/ATen.h>

#include "../loss/tb_py_capture.h"
#include "tensorembed.h"

namespace {

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
bool type_of(at::ScalarType s, int32_t* type) {
  *type = s == at::kFloat ? TB_FLOAT32 : s == at::kBFloat16 ? TB_BFLOAT16 : TB_FLOAT16;
  return s == at::kFloat || s == at::kBFloat16 || s == at::kHalf;
}
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

// The positions of a call, [B, T] or [N], on the GPU of `home`.
struct Positions {
  tb_positions_t at = {};
  int32_t B = 0, T = 0;
  bool packed = false;
  int32_t* status = nullptr;
  void* stream = nullptr;
  c10::Device device = c10::Device(c10::kCPU);
  const at::Tensor *tokens = nullptr, *lengths = nullptr, *mask = nullptr;

  bool here(const at::Tensor* t) const { return t && t->layout() == at::kStrided && t->is_cuda() && t->device() == device; }
  bool take_home(const at::Tensor* t) {
    if (!t || !t->is_cuda() || t->layout() != at::kStrided) return false;
    device = t->device();
    const auto s = c10::hip::getCurrentHIPStream();
    stream = static_cast<void*>(s.stream());
    return s.device_index() == device.index();
  }
  bool take(const at::Tensor* tokens_, const at::Tensor* lengths_, const at::Tensor* mask_) {
    const at::Tensor* t = tokens_;
    if (!here(t) || (t->scalar_type() != at::kInt && t->scalar_type() != at::kLong) || (t->dim() != 1 && t->dim() != 2))
      return false;
    packed = t->dim() == 1;
    const int64_t b = packed ? 1 : t->size(0), n = t->size(-1);
    if (b > INT32_MAX || n > INT32_MAX || (t->numel() > 0 && n > 1 && t->stride(-1) != 1)) return false;
    tokens = t;
    B = int32_t(b);
    T = int32_t(n);
    at.tokens = t->data_ptr();
    at.token_stride = packed ? n : t->stride(0);
    at.token_bytes = t->scalar_type() == at::kLong ? 8 : 4;
    if (lengths_) {
      t = lengths_;
      if (packed || !here(t) || t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != B || !t->is_contiguous()) return false;
      lengths = t;
      at.lengths = t->data_ptr<int32_t>();
    }
    if (mask_) {
      t = mask_;
      if (!here(t) || (t->scalar_type() != at::kBool && t->scalar_type() != at::kByte) || t->sizes() != tokens->sizes() ||
          !t->is_contiguous())
        return false;
      mask = t;
      at.mask = static_cast<const uint8_t*>(t->data_ptr());
    }
    return true;
  }
  bool take(PyObject* tokens_, PyObject* lengths_, PyObject* mask_, PyObject* status_) {
    const at::Tensor *n = tensor(lengths_), *m = tensor(mask_);
    if ((!n && lengths_ != Py_None) || (!m && mask_ != Py_None) || !take(tensor(tokens_), n, m)) return false;
    if (status_ == Py_None) return true;
    const at::Tensor* t = tensor(status_);
    if (!here(t) || t->scalar_type() != at::kInt || t->numel() != 1) return false;
    status = t->data_ptr<int32_t>();
    return true;
  }
  // rows [B, T, D] or [N, D] over these positions
  bool take_rows(const at::Tensor* t, tb_embedding_rows_t* rows) const {
    if (!here(t) || !type_of(t->scalar_type(), &rows->type) || t->dim() != tokens->dim() + 1 || t->size(-1) < 1 ||
        t->size(-1) > TB_WIDTH_MOST || t->sizes().slice(0, t->dim() - 1) != tokens->sizes() ||
        (t->numel() > 0 && t->size(-1) > 1 && t->stride(-1) != 1))
      return false;
    *rows = {t->data_ptr(), packed ? 0 : t->stride(0), t->stride(packed ? 0 : 1), B, T, int32_t(t->size(-1)), rows->type};
    return true;
  }
};

// The gradient of `rows` in a table of V rows, into `out`.
int gradient_into(const Positions& p, const tb_embedding_rows_t& rows, const at::Tensor& out, float scale, bool accumulate) {
  tb_table_gradient_t g = {out.data_ptr(), out.stride(0), int32_t(out.size(0)), 0, scale, accumulate};
  type_of(out.scalar_type(), &g.type);
  const size_t bytes = tensorembed_workspace_bytes(p.B, p.T, g.V, rows.D);
  const at::Tensor workspace = at::empty({int64_t(bytes)}, at::TensorOptions().dtype(at::kByte).device(p.device));
  return tensorembed_gradient(&rows, &p.at, &g, p.status, workspace.data_ptr(), bytes, p.stream);
}

// Everything that the kernels read comes from the saved tensors as they are unpacked: where hooks are active
// (checkpointing, offloading), these are other tensors than the forward pass's, and their strides may be others.
struct EmbeddingBackward : public torch::autograd::Node {
  using Saved = torch::autograd::SavedVariable;
  Saved tokens, lengths, mask;
  std::vector<int64_t> sizes;  // of the tokens
  int64_t V, D;
  at::ScalarType type;
  c10::Device device;
  float scale;

  static Saved kept(const at::Tensor* t) { return t ? Saved(*t, false) : Saved(); }
  EmbeddingBackward(const Positions& p, const at::Tensor& table, float by)
      : sizes(p.tokens->sizes().vec()), V(table.size(0)), D(table.size(1)), type(table.scalar_type()), device(table.device()),
        scale(by) {
    tokens = kept(p.tokens);
    lengths = kept(p.lengths);
    mask = kept(p.mask);
    set_next_edges(torch::autograd::collect_next_edges(table));
  }
  std::string name() const override { return "TensorEmbeddingBackward"; }
  void release_variables() override {
    std::lock_guard<std::mutex> lock(mutex_);
    for (Saved* s : {&tokens, &lengths, &mask}) s->reset_data();
  }
  torch::autograd::variable_list apply(torch::autograd::variable_list&& in) override {
    std::lock_guard<std::mutex> lock(mutex_);
    TORCH_CHECK(!at::GradMode::is_enabled(), "the embedding cannot be differentiated twice");
    TORCH_CHECK(!tb::leaves_capture(this), tb::kLeavesCapture);
    if (!in[0].defined()) return {at::Tensor()};
    at::Tensor ids = tokens.unpack(), n = lengths.unpack(), m = mask.unpack(), rows = in[0];
    if (ids.defined() && ids.dim() > 0 && ids.size(-1) > 1 && ids.stride(-1) != 1) ids = ids.contiguous();
    if (n.defined()) n = n.contiguous();
    if (m.defined()) m = m.contiguous();
    const c10::OptionalDeviceGuard guard(device);
    rows = rows.to(type);
    if (rows.size(-1) > 1 && rows.stride(-1) != 1) rows = rows.contiguous();
    Positions p;
    tb_embedding_rows_t given = {};
    TORCH_CHECK(p.take_home(&rows) && rows.device() == device && p.take(&ids, n.defined() ? &n : nullptr, m.defined() ? &m : nullptr) &&
                    ids.sizes() == at::IntArrayRef(sizes) && p.take_rows(&rows, &given) && given.D == D,
                "a tensor of the embedding's backward pass has come with another shape, type or device");
    at::Tensor out = at::empty({V, D}, rows.options().requires_grad(false));
    const int rc = gradient_into(p, given, out, scale, false);
    TORCH_CHECK(rc == TB_OK, "tensorembed gradient: ", tensorbleu_status_string(rc));
    return {out};
  }
};

// lookup(table, tokens, lengths, mask, scale, status): a tensor, or None
PyObject* lookup(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Positions p;
  const at::Tensor* table = n == 6 ? tensor(args[0]) : nullptr;
  float scale;
  if (!p.take_home(table) || !p.take(args[1], args[2], args[3], args[5]) || !take_float(args[4], &scale)) Py_RETURN_NONE;
  tb_table_t t = {};
  if (!type_of(table->scalar_type(), &t.type) || table->dim() != 2 || table->_fw_grad(0).defined() || table->size(0) < 1 ||
      table->size(0) > INT32_MAX || table->size(1) < 1 || table->size(1) > TB_WIDTH_MOST ||
      (table->size(1) > 1 && table->stride(1) != 1))
    Py_RETURN_NONE;
  t.data = table->data_ptr();
  t.row_stride = table->stride(0);
  t.V = int32_t(table->size(0));
  t.D = int32_t(table->size(1));
  at::DimVector shape(p.tokens->sizes().begin(), p.tokens->sizes().end());
  shape.push_back(t.D);
  at::Tensor out = at::empty(shape, table->options().requires_grad(false));
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = tensorembed_lookup(&t, &p.at, p.B, p.T, scale, out.data_ptr(), p.status, p.stream);
  Py_END_ALLOW_THREADS
  if (rc != TB_OK) Py_RETURN_NONE;
  if (at::GradMode::is_enabled() && table->requires_grad())
    torch::autograd::set_history(
        out, std::shared_ptr<EmbeddingBackward>(new EmbeddingBackward(p, *table, scale), torch::autograd::deleteNode));
  return THPVariable_Wrap(std::move(out));
}

// gradient(rows, tokens, V, lengths, mask, scale, dtype, out, accumulate, status): a tensor, or None.  dtype: 0 that of the rows,
// 1 float32
PyObject* gradient(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Positions p;
  const at::Tensor* rows = n == 10 ? tensor(args[0]) : nullptr;
  tb_embedding_rows_t given = {};
  float scale;
  if (!p.take_home(rows) || !p.take(args[1], args[3], args[4], args[9]) || !p.take_rows(rows, &given) ||
      !take_float(args[5], &scale) || rows->_fw_grad(0).defined() || !PyLong_CheckExact(args[2]) || !PyLong_CheckExact(args[6]) ||
      !PyBool_Check(args[8]))
    Py_RETURN_NONE;
  int overflow = 0;
  const long V = PyLong_AsLongAndOverflow(args[2], &overflow), wide = PyLong_AsLong(args[6]);
  if (overflow || V < 1 || V > INT32_MAX || (wide != 0 && wide != 1)) Py_RETURN_NONE;
  const bool accumulate = args[8] == Py_True;
  at::Tensor out;
  if (args[7] == Py_None) {
    if (accumulate) Py_RETURN_NONE;
    out = at::empty({V, given.D}, rows->options().dtype(wide ? at::kFloat : rows->scalar_type()).requires_grad(false));
  } else {
    const at::Tensor* t = tensor(args[7]);
    if (!p.here(t) || t->dim() != 2 || t->size(0) != V || t->size(1) != given.D || (given.D > 1 && t->stride(1) != 1) ||
        t->requires_grad() || t->scalar_type() != (wide ? at::kFloat : rows->scalar_type()))
      Py_RETURN_NONE;
    out = *t;
  }
  const int rc = gradient_into(p, given, out, scale, accumulate);
  if (rc != TB_OK) Py_RETURN_NONE;
  if (args[7] == Py_None) return THPVariable_Wrap(std::move(out));
  if (!out.is_inference()) out.unsafeGetTensorImpl()->bump_version();
  Py_INCREF(args[7]);
  return args[7];
}

// at:: functions throw (out of memory): to Python as the exceptions that torch itself raises
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return F(self, args, n);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"lookup", reinterpret_cast<PyCFunction>(guarded<lookup>), METH_FASTCALL, nullptr},
                         {"gradient", reinterpret_cast<PyCFunction>(guarded<gradient>), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_embed_host", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__embed_host(void) { return PyModule_Create(&module); }
