// Descriptors and addresses of a list of gradients for fira_grad_norm and fira_clip_grads, read from torch's tensors
// directly: 0.05 us per tensor instead of 0.4 to 0.8 through Python's attributes, which bounds lists of small tensors.
// Part of the Python binding, not of the library.
//
// grad_list(Gs, out or None) -> (device index, descriptors, addresses, addresses of the outputs or None), each a bytes
// object as the C ABI takes it; None where the list is anything but contiguous float32 and bfloat16 tensors of one CUDA device with
// outputs of the same shapes: binding.py handles the other layouts, and says what is wrong.
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "../../include/fira.h"

namespace {

int type_code(const at::Tensor& t) {
  return t.scalar_type() == at::kFloat ? FIRA_F32 : t.scalar_type() == at::kBFloat16 ? FIRA_BF16 : -1;
}

PyObject* bytes_of(const void* p, size_t n) { return PyBytes_FromStringAndSize(static_cast<const char*>(p), (Py_ssize_t)n); }

PyObject* grad_list(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 2) { PyErr_SetString(PyExc_TypeError, "grad_list(gradients, outputs or None)"); return nullptr; }
  const bool in_place = args[1] == Py_None;
  for (int k = 0; k < (in_place ? 1 : 2); ++k)
    if (!PyList_Check(args[k]) && !PyTuple_Check(args[k])) Py_RETURN_NONE;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(args[0]);
  if (n == 0 || n > 0x7fffffff || (!in_place && PySequence_Fast_GET_SIZE(args[1]) != n)) Py_RETURN_NONE;
  try {
    std::vector<fira_grad_desc> descs((size_t)n);
    std::vector<void*> at((size_t)n), out_at(in_place ? 0 : (size_t)n);
    int device = -1;
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* obj = PySequence_Fast_GET_ITEM(args[0], i);
      PyObject* out_obj = in_place ? obj : PySequence_Fast_GET_ITEM(args[1], i);
      if (!THPVariable_Check(obj) || !THPVariable_Check(out_obj)) Py_RETURN_NONE;
      const at::Tensor& g = THPVariable_Unpack(obj);
      const at::Tensor& o = THPVariable_Unpack(out_obj);
      if (!g.defined() || !o.defined() || g.layout() != at::kStrided || o.layout() != at::kStrided || !g.is_cuda() || !o.is_cuda() ||
          !g.is_contiguous() || !o.is_contiguous() || g.sizes() != o.sizes())
        Py_RETURN_NONE;
      const int code = type_code(g), out_code = type_code(o);
      if (code < 0 || out_code < 0) Py_RETURN_NONE;
      if (i == 0) device = g.get_device();
      if (g.get_device() != device || o.get_device() != device) Py_RETURN_NONE;
      descs[(size_t)i] = fira_grad_desc{1, g.numel(), 0, 0, code, out_code};
      at[(size_t)i] = g.data_ptr();
      if (!in_place) out_at[(size_t)i] = o.data_ptr();
    }
    PyObject* d = bytes_of(descs.data(), descs.size() * sizeof(fira_grad_desc));
    PyObject* a = bytes_of(at.data(), at.size() * sizeof(void*));
    PyObject* b = in_place ? Py_NewRef(Py_None) : bytes_of(out_at.data(), out_at.size() * sizeof(void*));
    PyObject* index = PyLong_FromLong(device);
    PyObject* r = d && a && b && index ? PyTuple_Pack(4, index, d, a, b) : nullptr;
    Py_XDECREF(index); Py_XDECREF(d); Py_XDECREF(a); Py_XDECREF(b);
    return r;
  } catch (...) {                           // a tensor without storage, say: binding.py meets it again, and reports it
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

PyMethodDef methods[] = {{"grad_list", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(grad_list)), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native_lists", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// With what binding.py holds against its own before it uses the module: torch's version and the size of a descriptor.
extern "C" __attribute__((visibility("default"))) PyObject* PyInit__native_lists() {
  PyObject* m = PyModule_Create(&module);
  if (m && (PyModule_AddStringConstant(m, "torch_version", FIRA_LISTS_TORCH) < 0 || PyModule_AddIntConstant(m, "desc_bytes", sizeof(fira_grad_desc)) < 0)) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
