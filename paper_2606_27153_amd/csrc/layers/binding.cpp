// The operators of a token's way to its experts and back and of its row of a table,
// called without a Python call for each property of each tensor.  For few tokens
// a kernel takes 3 to 4 us; the checks, outputs and the call take 7 to 9 us in
// Python and 4 to 6 here (the sort, with three outputs, 8.7 and 5.8).
//
// Each function checks what its counterpart in layers.py does, and returns None
// where anything does not fit or there is nothing to do: that one says what it is.
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "muon_layers.h"

namespace {

PyObject *g_get_device, *g_get_stream;   // torch's own, which say them without a lookup by name

struct Failed {};   // thrown and caught here: the arguments do not fit

void need(bool ok) {
  if (!ok) throw Failed{};
}

const at::Tensor& tensor(PyObject* o) {
  need(THPVariable_Check(o));
  const at::Tensor& t = THPVariable_Unpack(o);
  need(t.defined() && t.layout() == at::kStrided && t.is_cuda());
  return t;
}

int dtype_code(const at::Tensor& t) {
  return t.scalar_type() == at::kFloat ? MUON_F32 : t.scalar_type() == at::kBFloat16 ? MUON_BF16 : -1;
}

// A matrix of contiguous rows, of the dtype and on the device that the first one has.
struct Matrix {
  const void* p;
  int64_t rows, cols, ld;
  int dtype;
  int64_t device;
  explicit Matrix(PyObject* o) {
    const at::Tensor& t = tensor(o);
    dtype = dtype_code(t);
    need(dtype >= 0 && t.dim() == 2 && t.size(1) > 0 && t.stride(1) == 1 && t.stride(0) >= t.size(1));
    p = t.const_data_ptr();
    rows = t.size(0);
    cols = t.size(1);
    ld = t.stride(0);
    device = t.get_device();
  }
  void like(const Matrix& a, int64_t r) const {
    need(dtype == a.dtype && device == a.device && rows == r && cols == a.cols);
  }
};

// Contiguous numbers of 4 or 8 bytes.
struct Numbers {
  const at::Tensor& t;
  const void* p;
  int32_t bytes;
  explicit Numbers(PyObject* o) : t(tensor(o)) {
    bytes = t.scalar_type() == at::kInt ? 4 : t.scalar_type() == at::kLong ? 8 : 0;
    need(bytes && t.is_contiguous());
    p = t.const_data_ptr();
  }
};

struct Routing {
  const int32_t *position, *source;
  int64_t tokens;
  int32_t top;
  Routing(PyObject* o, int64_t device) {
    need(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 3);
    const at::Tensor &at = tensor(PyTuple_GET_ITEM(o, 1)), &from = tensor(PyTuple_GET_ITEM(o, 2));
    for (const at::Tensor* t : {&at, &from})
      need(t->scalar_type() == at::kInt && t->is_contiguous() && t->get_device() == device);
    need(at.dim() == 2 && from.dim() == 1 && from.size(0) == at.numel());
    need(at.numel() > 0 && at.size(1) <= MUON_GROUPED_MAX_EXPERTS);
    position = static_cast<const int32_t*>(at.const_data_ptr());
    source = static_cast<const int32_t*>(from.const_data_ptr());
    tokens = at.size(0);
    top = int32_t(at.size(1));
  }
};

struct Weights {
  const void* p;
  int32_t dtype;
  Weights(PyObject* o, const Matrix& x, const Routing& r) {
    const at::Tensor& t = tensor(o);
    dtype = dtype_code(t);
    need((dtype == MUON_F32 || dtype == x.dtype) && t.dim() == 2 && t.size(0) == r.tokens && t.size(1) == r.top &&
         t.is_contiguous() && t.get_device() == x.device);
    p = t.const_data_ptr();
  }
};

// torch's current stream on a device, which has to be the current one.
void* stream_of(int64_t device) {
  PyObject* index = PyObject_CallNoArgs(g_get_device);
  need(index != nullptr);
  const int64_t current = PyLong_AsLongLong(index);
  PyObject* stream = current == device ? PyObject_CallOneArg(g_get_stream, index) : nullptr;
  Py_DECREF(index);
  need(stream != nullptr);
  void* s = PyLong_AsVoidPtr(stream);
  Py_DECREF(stream);
  need(!PyErr_Occurred());
  return s;
}

at::Tensor empty(at::IntArrayRef sizes, int64_t device, at::ScalarType type) {
  return at::empty(sizes, at::TensorOptions().device(at::Device(at::kCUDA, c10::DeviceIndex(device))).dtype(type));
}
at::Tensor empty_like(const Matrix& x, at::IntArrayRef sizes) {
  return empty(sizes, x.device, x.dtype == MUON_F32 ? at::kFloat : at::kBFloat16);
}

void called(muon_status s) { need(s == MUON_OK); }

// Other threads run Python meanwhile: an allocation or a launch may wait.
class NoGil {
 public:
  NoGil() : state_(PyEval_SaveThread()) {}
  ~NoGil() { PyEval_RestoreThread(state_); }
  NoGil(const NoGil&) = delete;
  NoGil& operator=(const NoGil&) = delete;

 private:
  PyThreadState* state_;
};

// sort_by_expert(experts, count) -> (offsets, position, source)
PyObject* sort_by_expert(PyObject* const* args, Py_ssize_t n) {
  need(n == 2);
  const Numbers e(args[0]);
  need(PyLong_Check(args[1]));
  const int64_t count = PyLong_AsLongLong(args[1]), device = e.t.get_device();
  need(e.t.dim() == 2 && e.t.numel() > 0 && count >= 1 && count <= MUON_GROUPED_MAX_EXPERTS &&
       e.t.size(1) <= MUON_GROUPED_MAX_EXPERTS);
  const int64_t tokens = e.t.size(0);
  const int32_t top = int32_t(e.t.size(1));
  void* const stream = stream_of(device);
  at::Tensor offsets, position, source, ws;
  {
    const NoGil run;
    size_t bytes = 0;
    called(muon_sort_by_expert_workspace_bytes(tokens, top, &bytes));
    offsets = empty({count + 1}, device, at::kInt);
    position = empty({tokens, top}, device, at::kInt);
    source = empty({tokens * top}, device, at::kInt);
    if (bytes) ws = empty({int64_t(bytes)}, device, at::kByte);
    called(muon_sort_by_expert(e.p, e.bytes, tokens, top, int32_t(count), static_cast<int32_t*>(offsets.data_ptr()),
                               static_cast<int32_t*>(position.data_ptr()), static_cast<int32_t*>(source.data_ptr()),
                               bytes ? ws.data_ptr() : nullptr, bytes, stream));
  }
  return Py_BuildValue("NNN", THPVariable_Wrap(offsets), THPVariable_Wrap(position), THPVariable_Wrap(source));
}

// dispatch_forward(x, routing) -> rows
PyObject* dispatch_forward(PyObject* const* args, Py_ssize_t n) {
  need(n == 2);
  const Matrix x(args[0]);
  const Routing r(args[1], x.device);
  need(x.rows == r.tokens);
  void* const stream = stream_of(x.device);
  at::Tensor rows;
  {
    const NoGil run;
    rows = empty_like(x, {r.tokens * r.top, x.cols});
    called(muon_dispatch_forward(x.p, x.ld, r.position, r.source, rows.data_ptr(), x.cols, r.tokens, r.top, x.cols,
                                 x.dtype, stream));
  }
  return THPVariable_Wrap(rows);
}

// dispatch_backward(drows, routing) -> dx
PyObject* dispatch_backward(PyObject* const* args, Py_ssize_t n) {
  need(n == 2);
  const Matrix g(args[0]);
  const Routing r(args[1], g.device);
  need(g.rows == r.tokens * r.top);
  void* const stream = stream_of(g.device);
  at::Tensor dx;
  {
    const NoGil run;
    dx = empty_like(g, {r.tokens, g.cols});
    called(muon_dispatch_backward(g.p, g.ld, r.position, dx.data_ptr(), g.cols, r.tokens, r.top, g.cols, g.dtype,
                                  stream));
  }
  return THPVariable_Wrap(dx);
}

// combine_forward(rows, weights, routing, residual) -> y
PyObject* combine_forward(PyObject* const* args, Py_ssize_t n) {
  need(n == 4);
  const Matrix h(args[0]);
  const Routing r(args[2], h.device);
  const Weights w(args[1], h, r);
  need(h.rows == r.tokens * r.top);
  const void* res = nullptr;
  int64_t ldres = 0;
  if (args[3] != Py_None) {
    const Matrix m(args[3]);
    m.like(h, r.tokens);
    res = m.p;
    ldres = m.ld;
  }
  void* const stream = stream_of(h.device);
  at::Tensor y;
  {
    const NoGil run;
    y = empty_like(h, {r.tokens, h.cols});
    called(muon_combine_forward(h.p, h.ld, w.p, w.dtype, r.position, res, ldres, y.data_ptr(), h.cols, r.tokens, r.top,
                                h.cols, h.dtype, stream));
  }
  return THPVariable_Wrap(y);
}

// combine_backward(dy, rows, weights, routing, rows_grad, weights_grad) -> (drows, dweights)
PyObject* combine_backward(PyObject* const* args, Py_ssize_t n) {
  need(n == 6);
  const Matrix g(args[0]), h(args[1]);
  const Routing r(args[3], g.device);
  const Weights w(args[2], g, r);
  need(g.rows == r.tokens && (args[4] == Py_True || args[4] == Py_False) &&
       (args[5] == Py_True || args[5] == Py_False));
  h.like(g, r.tokens * r.top);
  void* const stream = stream_of(g.device);
  at::Tensor dh, dw;
  const bool rows_grad = args[4] == Py_True, weights_grad = args[5] == Py_True;
  {
    const NoGil run;
    if (rows_grad) dh = empty_like(g, {h.rows, g.cols});
    if (weights_grad) dw = empty({r.tokens, r.top}, g.device, w.dtype == MUON_F32 ? at::kFloat : at::kBFloat16);
    called(muon_combine_backward(g.p, g.ld, h.p, h.ld, w.p, w.dtype, r.source, dh.defined() ? dh.data_ptr() : nullptr,
                                 g.cols, dw.defined() ? dw.data_ptr() : nullptr, r.tokens, r.top, g.cols, g.dtype,
                                 stream));
  }
  return Py_BuildValue("NN", THPVariable_Wrap(dh), THPVariable_Wrap(dw));   // (None for one that is not there)
}

// embedding_forward(ids, weight, scale) -> y
PyObject* embedding_forward(PyObject* const* args, Py_ssize_t n) {
  need(n == 3);
  const Numbers ids(args[0]);
  const Matrix w(args[1]);
  need(PyFloat_Check(args[2]) && ids.t.get_device() == w.device && ids.t.numel() > 0 && w.rows > 0);
  void* const stream = stream_of(w.device);
  c10::SmallVector<int64_t, 5> sizes(ids.t.sizes().begin(), ids.t.sizes().end());
  sizes.push_back(w.cols);
  const float scale = float(PyFloat_AS_DOUBLE(args[2]));
  at::Tensor y;
  {
    const NoGil run;
    y = empty_like(w, sizes);
    called(muon_embedding_forward(ids.p, ids.bytes, w.p, w.ld, y.data_ptr(), w.cols, ids.t.numel(), w.rows, w.cols,
                                  scale, w.dtype, stream));
  }
  return THPVariable_Wrap(y);
}

// embedding_backward(dy, ids, vocab, scale) -> dw, for dy without gaps
PyObject* embedding_backward(PyObject* const* args, Py_ssize_t n) {
  need(n == 4);
  const at::Tensor& dy = tensor(args[0]);
  const Numbers ids(args[1]);
  const int dtype = dtype_code(dy);
  need(dtype >= 0 && dy.is_contiguous() && dy.dim() == ids.t.dim() + 1 && PyLong_Check(args[2]) &&
       PyFloat_Check(args[3]));
  const int64_t rows = ids.t.numel(), cols = dy.size(-1), device = dy.get_device(), vocab = PyLong_AsLongLong(args[2]);
  need(dy.sizes().slice(0, ids.t.dim()).equals(ids.t.sizes()) && ids.t.get_device() == device && rows > 0 &&
       cols > 0 && vocab > 0);
  void* const stream = stream_of(device);
  const float scale = float(PyFloat_AS_DOUBLE(args[3]));
  at::Tensor dw;
  {
    const NoGil run;
    size_t bytes = 0;
    called(muon_embedding_workspace_bytes(rows, vocab, cols, &bytes));
    dw = empty({vocab, cols}, device, dy.scalar_type());
    const at::Tensor ws = empty({int64_t(bytes)}, device, at::kByte);
    called(muon_embedding_backward(dy.const_data_ptr(), cols, ids.p, ids.bytes, dw.data_ptr(), cols, rows, vocab, cols,
                                   scale, dtype, ws.data_ptr(), bytes, stream));
  }
  return THPVariable_Wrap(dw);
}

template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    return F(args, n);
  } catch (...) {   // (also a tensor without memory of its own, or no memory left)
  }
  PyErr_Clear();
  Py_RETURN_NONE;
}
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
constexpr PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<F>)), METH_FASTCALL,
          "As the function of this name in layers.py, or None where the arguments do not fit."};
}

PyMethodDef methods[] = {method<sort_by_expert>("sort_by_expert"),
                         method<dispatch_forward>("dispatch_forward"),
                         method<dispatch_backward>("dispatch_backward"),
                         method<combine_forward>("combine_forward"),
                         method<combine_backward>("combine_backward"),
                         method<embedding_forward>("embedding_forward"),
                         method<embedding_backward>("embedding_backward"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layers_binding", nullptr, -1, methods, nullptr, nullptr, nullptr,
                      nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__layers_binding() {
  PyObject* c = PyImport_ImportModule("torch._C");
  if (!c) return nullptr;
  g_get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
  g_get_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
  Py_DECREF(c);
  return g_get_device && g_get_stream ? PyModule_Create(&module) : nullptr;
}
