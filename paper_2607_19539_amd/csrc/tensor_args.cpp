// tensor_args.cpp -- the binding's check of a tensor argument, as a Python extension.
//
// want(name, tensor, shape, kind) is the tensor's device pointer, if it is a contiguous device tensor of exactly
// this shape and one of the kind's types; opt is the same and passes None on.  A call of an operator makes up to
// nine such checks: in Python each takes 0.37 us, here less than 0.1, of a call that takes 3 us to enqueue.
#include <ATen/core/Tensor.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

PyObject* g_refuse = nullptr;  // refuse(name, tensor, shape, kind) raises what is wrong

// The kinds of the binding's constants, in their order.
bool of_kind(at::ScalarType t, long kind) {
  switch (kind) {
    case 0: return t == at::kBFloat16 || t == at::kShort;  // bf16 or its bit patterns
    case 1: return t == at::kChar;
    case 2: return t == at::kInt;
    case 3: return t == at::kFloat;
    case 4: return t == at::kBFloat16;
    case 5: return t == at::kFloat || t == at::kBFloat16;
    case 6: return t == at::kDouble;
    default: return false;
  }
}

// Kinds from here on: the tensor is on the current device, too.
constexpr long kHere = 16;

c10::DeviceIndex current_device() { return c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index(); }

bool fits(const at::Tensor& t, PyObject* shape, long kind) {
  if (kind >= kHere) {
    if (!t.is_cuda() || t.device().index() != current_device()) return false;
    kind -= kHere;
  }
  if (!of_kind(t.scalar_type(), kind) || !PyTuple_Check(shape)) return false;
  const auto sizes = t.sizes();
  if (PyTuple_GET_SIZE(shape) != (Py_ssize_t)sizes.size()) return false;
  for (size_t i = 0; i < sizes.size(); ++i)
    if (PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i)) != sizes[i]) return false;
  return t.is_cuda() && t.is_contiguous();
}

PyObject* want(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "want(name, tensor, shape, kind)");
    return nullptr;
  }
  try {
    const long kind = PyLong_AsLong(args[3]);
    if (THPVariable_Check(args[1])) {
      const at::Tensor& t = THPVariable_Unpack(args[1]);
      if (fits(t, args[2], kind) && !PyErr_Occurred()) return PyLong_FromVoidPtr(t.data_ptr());
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
  if (PyErr_Occurred()) return nullptr;
  if (!g_refuse) {
    PyErr_SetString(PyExc_ValueError, "not the tensor wanted");
    return nullptr;
  }
  return PyObject_Vectorcall(g_refuse, args, 4, nullptr);
}

PyObject* opt(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  if (n == 4 && args[1] == Py_None) Py_RETURN_NONE;
  return want(self, args, n);
}

// A tensor of a list as the C entry points take it (moe_tensor_t).
struct Entry {
  const void* data;
  void* out;
  int64_t count;
  int32_t type, reserved;
};

// table(tensors, outs or None): a bytes object of an Entry each, or None if a tensor is not a contiguous fp32 or bf16
// tensor on the current device or an out is not one of the same type and size.
PyObject* table(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "table(tensors, outs)");
    return nullptr;
  }
  PyObject* tensors = PySequence_Fast(args[0], "a sequence of tensors expected");
  if (!tensors) return nullptr;
  PyObject* outs = args[1] == Py_None ? nullptr : PySequence_Fast(args[1], "a sequence of tensors expected");
  if (args[1] != Py_None && !outs) {
    Py_DECREF(tensors);
    return nullptr;
  }
  const Py_ssize_t m = PySequence_Fast_GET_SIZE(tensors);
  PyObject* bytes = nullptr;
  bool good = !outs || PySequence_Fast_GET_SIZE(outs) == m;
  c10::DeviceIndex device = -1;  // asked for at the first tensor that is on a device
  try {
    bytes = PyBytes_FromStringAndSize(nullptr, m * (Py_ssize_t)sizeof(Entry));
    Entry* e = bytes ? (Entry*)PyBytes_AS_STRING(bytes) : nullptr;
    for (Py_ssize_t i = 0; e && good && i < m; ++i) {
      PyObject* p = PySequence_Fast_GET_ITEM(tensors, i);
      PyObject* q = outs ? PySequence_Fast_GET_ITEM(outs, i) : p;
      good = THPVariable_Check(p) && THPVariable_Check(q);
      if (!good) break;
      const at::Tensor &t = THPVariable_Unpack(p), &o = THPVariable_Unpack(q);
      good = of_kind(t.scalar_type(), 5) && o.scalar_type() == t.scalar_type() && o.numel() == t.numel() && t.is_cuda() &&
             o.is_cuda() && t.is_contiguous() && o.is_contiguous();
      if (good && device < 0) device = current_device();
      good = good && t.device().index() == device && o.device().index() == device;
      if (good) e[i] = Entry{t.data_ptr(), o.data_ptr(), t.numel(), t.scalar_type() == at::kBFloat16, 0};
    }
  } catch (const std::exception& x) {
    PyErr_SetString(PyExc_RuntimeError, x.what());
    good = false;
  }
  Py_DECREF(tensors);
  Py_XDECREF(outs);
  if (PyErr_Occurred()) {
    Py_XDECREF(bytes);
    return nullptr;
  }
  if (good) return bytes;
  Py_XDECREF(bytes);
  Py_RETURN_NONE;
}

PyObject* set_refuse(PyObject*, PyObject* fn) {
  Py_XINCREF(fn);
  Py_XDECREF(g_refuse);
  g_refuse = fn;
  Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {{"want", (PyCFunction)(void*)want, METH_FASTCALL, nullptr},
                           {"opt", (PyCFunction)(void*)opt, METH_FASTCALL, nullptr},
                           {"table", (PyCFunction)(void*)table, METH_FASTCALL, nullptr},
                           {"set_refuse", set_refuse, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_moe_args", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__moe_args() { return PyModule_Create(&g_module); }
