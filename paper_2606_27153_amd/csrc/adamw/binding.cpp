// The tensors of an AdamW step as the library takes them, checked and written down
// without a Python call for each of their properties: about 20 properties a
// tensor, which in Python take 1 us and here less than 0.1, so that a step over hundreds of
// small tensors is not bound by the host.
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <vector>

#include "muon_adamw.h"

namespace {

// Borrowed items of a list or tuple.
struct Items {
  PyObject* fast;
  explicit Items(PyObject* o) : fast(PySequence_Fast(o, "a sequence")) {}
  ~Items() { Py_XDECREF(fast); }
  Items(const Items&) = delete;
  Items& operator=(const Items&) = delete;
  bool ok() const { return fast != nullptr; }
  Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(fast); }
  PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast, i); }
};

const at::Tensor* tensor(PyObject* o) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.layout() == at::kStrided && t.is_contiguous() ? &t : nullptr;
}

int dtype_code(const at::Tensor& t) {
  return t.scalar_type() == at::kFloat ? MUON_F32 : t.scalar_type() == at::kBFloat16 ? MUON_BF16 : -1;
}

// The addresses that a step writes to: a table with a quarter of its places taken at most.
class Written {
 public:
  explicit Written(size_t count) {
    size_t places = 16;
    while (places < 4 * count) places *= 2;
    at_.resize(places);
  }
  // Whether p is new.
  bool add(const void* p) {
    size_t i = size_t(reinterpret_cast<uintptr_t>(p) * 0x9E3779B97F4A7C15u >> 20) & (at_.size() - 1);
    for (; at_[i]; i = (i + 1) & (at_.size() - 1))
      if (at_[i] == p) return false;
    at_[i] = p;
    return true;
  }

 private:
  std::vector<const void*> at_;
};

// Whether every tensor fits; fills `out`, the device and the states' bits.
bool collect(const Items& params, const Items& grads, const Items& states, const Items& steps,
             std::vector<muon_adamw_tensor>& out, int64_t& device, int& bits) {
  const Py_ssize_t n = params.size();
  if (grads.size() != n || states.size() != n || steps.size() != n) return false;
  out.resize(size_t(n));
  Written written(4 * size_t(n));
  device = -1;
  bits = 0;
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor *p = tensor(params[i]), *g = tensor(grads[i]);
    if (!p || !g || !p->is_cuda() || !g->is_cuda()) return false;
    if (device < 0) device = p->get_device();
    if (!PyTuple_Check(states[i]) && !PyList_Check(states[i])) return false;
    const Items s(states[i]);
    if (!s.ok() || (s.size() != 2 && s.size() != 3)) return false;
    const int b = s.size() == 3 ? 8 : 32;
    if (bits && b != bits) return false;
    bits = b;
    const at::Tensor *m = tensor(s[0]), *v = tensor(s[1]), *bases = b == 8 ? tensor(s[2]) : nullptr;
    if (!m || !v || (b == 8 && !bases)) return false;
    for (const at::Tensor* t : {p, g, m, v})
      if (!t->is_cuda() || t->get_device() != device) return false;
    const int64_t elements = p->numel();
    const auto kind = b == 8 ? at::kByte : at::kFloat;
    muon_adamw_tensor& t = out[size_t(i)];
    t.param_dtype = dtype_code(*p);
    t.grad_dtype = dtype_code(*g);
    if (t.param_dtype < 0 || t.grad_dtype < 0 || !g->sizes().equals(p->sizes()) || m->scalar_type() != kind ||
        v->scalar_type() != kind || m->numel() != elements || v->numel() != elements)
      return false;
    t.bases = nullptr;
    if (b == 8) {
      if (!bases->is_cuda() || bases->get_device() != device || bases->scalar_type() != at::kShort ||
          bases->dim() != 2 || bases->size(0) != (elements + MUON_ADAMW_BLOCK - 1) / MUON_ADAMW_BLOCK ||
          bases->size(1) != 2)
        return false;
      t.bases = static_cast<int16_t*>(bases->data_ptr());
    }
    t.param = p->data_ptr();
    t.grad = g->const_data_ptr();
    t.exp_avg = m->data_ptr();
    t.exp_avg_sq = v->data_ptr();
    t.n = elements;
    t.step = PyLong_AsLongLong(steps[i]);
    if (t.step == -1 && PyErr_Occurred()) return false;
    if (elements && !(written.add(t.param) && written.add(t.exp_avg) && written.add(t.exp_avg_sq) &&
                      (!t.bases || written.add(t.bases))))
      return false;
  }
  return true;
}

// adamw_tensors(params, grads, states, steps) -> (bytes, device index, bits), the bytes an
// array of muon_adamw_tensor; None where a tensor does not fit.
PyObject* adamw_tensors(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (count != 4) {
    PyErr_SetString(PyExc_TypeError, "adamw_tensors takes params, grads, states and steps");
    return nullptr;
  }
  try {
    const Items params(args[0]), grads(args[1]), states(args[2]), steps(args[3]);
    std::vector<muon_adamw_tensor> out;
    int64_t device;
    int bits;
    if (params.ok() && grads.ok() && states.ok() && steps.ok() &&
        collect(params, grads, states, steps, out, device, bits))
      return Py_BuildValue("NLi",
                           PyBytes_FromStringAndSize(reinterpret_cast<const char*>(out.data()),
                                                     Py_ssize_t(out.size() * sizeof(muon_adamw_tensor))),
                           static_cast<long long>(device), bits);
  } catch (...) {   // (a tensor without memory of its own)
  }
  PyErr_Clear();
  Py_RETURN_NONE;
}

// adamw_written(params, grads, states): raises the versions of the tensors that a step
// with these gradients wrote to (through their addresses, unseen by torch), so that
// autograd refuses a backward pass that would read one saved before.
PyObject* adamw_written(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (count != 3) {
    PyErr_SetString(PyExc_TypeError, "adamw_written takes params, grads and states");
    return nullptr;
  }
  const auto written = [](PyObject* o) {
    if (!THPVariable_Check(o)) return;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();   // (an inference tensor has none)
  };
  const Items params(args[0]), grads(args[1]), states(args[2]);
  if (!params.ok() || !grads.ok() || !states.ok()) return nullptr;
  for (Py_ssize_t i = 0; i < params.size() && i < grads.size() && i < states.size(); ++i) {
    if (grads[i] == Py_None) continue;
    written(params[i]);
    const Items state(states[i]);
    if (!state.ok()) return nullptr;
    for (Py_ssize_t k = 0; k < state.size(); ++k) written(state[k]);
  }
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"adamw_tensors", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(adamw_tensors)), METH_FASTCALL,
     "The tensors of an AdamW step as the library takes them, or None."},
    {"adamw_written", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(adamw_written)), METH_FASTCALL,
     "Raises the versions of the tensors that an AdamW step wrote to."},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_adamw_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__adamw_binding() { return PyModule_Create(&module); }
