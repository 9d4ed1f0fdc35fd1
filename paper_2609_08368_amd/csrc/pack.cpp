// Python module _pack: the bytes of the rl_tensor that describes a torch tensor
// (include/rl_attn.h), for the ctypes calls of the binding. In C++ since a call
// has up to twelve tensors, and reading one through its Python attributes takes
// 0.56 us where the small calls' kernels take 4.
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>

#include "rl_attn.h"

namespace {

int dtype_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return RL_BF16;
    case at::kFloat: return RL_F32;
    case at::kInt: return RL_I32;
    case at::kLong: return RL_I64;
    case at::kFloat8_e4m3fn: return RL_FP8_E4M3;
    default: return 0;                              // (refused by the library, by name)
  }
}

// The library dereferences the pointers on the current HIP device, so every tensor
// must live there (a host pointer would reach a kernel).
PyObject* arg(PyObject*, PyObject* o) {
  if (o == Py_None) Py_RETURN_NONE;
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a tensor or None, got %s", Py_TYPE(o)->tp_name);
    return nullptr;
  }
  try {
    const at::Tensor& t = THPVariable_Unpack(o);
    const c10::Device device = t.device();
    if (!device.is_cuda() || device != c10::impl::VirtualGuardImpl(device.type()).getDevice()) {
      PyErr_Format(PyExc_ValueError, "tensor on %s: the library reads and writes tensors on the current device",
                   device.str().c_str());
      return nullptr;
    }
    const int64_t n = t.dim();
    if (n > 4) {
      PyErr_SetString(PyExc_ValueError, "rl_tensor holds at most 4 dimensions");
      return nullptr;
    }
    rl_tensor r;
    std::memset(&r, 0, sizeof r);
    r.data = t.data_ptr();
    r.dtype = dtype_of(t);
    r.ndim = (int32_t)n;
    for (int64_t i = 0; i < n; ++i) {
      r.shape[i] = t.size(i);
      r.strides[i] = t.stride(i);
    }
    return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&r), sizeof r);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef methods[] = {
    {"arg", arg, METH_O, "The bytes of an rl_tensor describing a tensor on the current device; None -> None."},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pack", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pack() { return PyModule_Create(&module); }
