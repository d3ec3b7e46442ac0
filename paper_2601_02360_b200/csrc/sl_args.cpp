// Argument checks of the Python binding: device pointers of torch tensors, taken only when the tensor is what the
// call is about to read or write.  In Python a check costs 0.36 us, and a call has up to fifteen; here 0.05 us.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// bits of a type mask
int type_bit(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return 1;
    case at::kBFloat16: return 2;
    case at::kInt: return 4;
    case at::kChar: return 8;
    case at::kByte: return 16;
    default: return 0;
  }
}

const char* type_names(int mask) {
  switch (mask) {
    case 1: return "float32";
    case 2: return "bfloat16";
    case 3: return "float32 or bfloat16";
    case 4: return "int32";
    case 8: return "int8";
    case 16: return "uint8";
    default: return "a known type";
  }
}

// Accessors of a tensor may throw (data_ptr() and stride() of tensors without storage or strides): a Python error, since
// no C++ exception may leave a C function.
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_ValueError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_ValueError, "unknown C++ exception");
  }
  return nullptr;
}

PyObject* refuse(PyObject* name, PyObject* t, const char* what, long long a, long long b, int mask) {
  PyErr_Format(PyExc_ValueError, what, name, type_names(mask), a, b, t == nullptr ? Py_None : (PyObject*)Py_TYPE(t));
  return nullptr;
}

// A tensor of which nothing will be read may have no memory; any other without memory (a fake tensor, a wrapper around other
// tensors) is refused: its null pointer would say that an optional argument is absent.
bool backed(const void* p, long long numel) { return p != nullptr || numel <= 0; }

// what is in memory is the tensor: not so for a view that is negated when it is read (the imaginary part of a conjugate)
bool plain(const at::Tensor& t) { return !t.is_neg(); }

// The launch goes to the current device, to a stream of its own: the kernels cannot have another one's memory.  A tensor without
// memory is on no device; the current one is asked for once a call (0.04 us), not once a tensor.
bool here(const at::Tensor& t, const void* p, long device) { return p == nullptr || device < 0 || t.get_device() == device; }

// device() -> index of the current CUDA device, -1 without one
PyObject* device(PyObject*, PyObject*) {
  try {
    return PyLong_FromLong(c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index());
  } catch (...) {
    return PyLong_FromLong(-1);
  }
}

// ptr(tensor or None, name, numel, type mask, device = any) -> device pointer (0 for None)
PyObject* ptr(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4 && n != 5) {
    PyErr_SetString(PyExc_TypeError, "ptr(tensor, name, numel, types, device)");
    return nullptr;
  }
  PyObject* o = args[0];
  if (o == Py_None) return PyLong_FromLong(0);
  const long long numel = PyLong_AsLongLong(args[2]);
  const long mask = PyLong_AsLong(args[3]), device = n > 4 ? PyLong_AsLong(args[4]) : -1;
  if (PyErr_Occurred()) return nullptr;
  return guarded([&]() -> PyObject* {
    if (THPVariable_Check(o)) {
      const at::Tensor& t = THPVariable_Unpack(o);
      if ((type_bit(t.scalar_type()) & mask) && t.is_cuda() && plain(t) && t.numel() >= numel && t.is_contiguous()) {
        const void* p = t.data_ptr();
        if (backed(p, numel) && here(t, p, device)) return PyLong_FromUnsignedLongLong((unsigned long long)(uintptr_t)p);
      }
    }
    return refuse(args[1], o, "%U: expected a contiguous tensor of %s on the current CUDA device with at least %lld elements (got %lld, %R)", numel,
                  THPVariable_Check(o) ? (long long)THPVariable_Unpack(o).numel() : -1, (int)mask);
  });
}

// rows(matrix or None, name, n, d, type mask, device = any) -> (device pointer, elements between rows); (0, d) for None
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t k) {
  if (k != 5 && k != 6) {
    PyErr_SetString(PyExc_TypeError, "rows(matrix, name, n, d, types, device)");
    return nullptr;
  }
  PyObject* o = args[0];
  const long long n = PyLong_AsLongLong(args[2]), d = PyLong_AsLongLong(args[3]);
  const long mask = PyLong_AsLong(args[4]), device = k > 5 ? PyLong_AsLong(args[5]) : -1;
  if (PyErr_Occurred()) return nullptr;
  if (o == Py_None) return Py_BuildValue("(iL)", 0, d);
  return guarded([&]() -> PyObject* {
    if (THPVariable_Check(o)) {
      const at::Tensor& t = THPVariable_Unpack(o);
      if ((type_bit(t.scalar_type()) & mask) && t.is_cuda() && plain(t) && t.dim() == 2 && t.size(0) >= n && t.size(1) == d &&
          (d == 1 || t.stride(1) == 1) && (n <= 1 || t.stride(0) >= d)) {
        const void* p = t.data_ptr();
        if (backed(p, n * d) && here(t, p, device)) return Py_BuildValue("(KL)", (unsigned long long)(uintptr_t)p, n > 1 ? (long long)t.stride(0) : d);
      }
    }
    return refuse(args[1], o, "%U: expected a matrix of %s on the current CUDA device with dense, evenly spaced rows, %lld x %lld (got %R)", n, d, (int)mask);
  });
}

// type(tensor) -> bit of its type mask, 0 if unknown
PyObject* type(PyObject*, PyObject* o) {
  return guarded([&]() -> PyObject* { return PyLong_FromLong(THPVariable_Check(o) ? type_bit(THPVariable_Unpack(o).scalar_type()) : 0); });
}

PyMethodDef methods[] = {
    {"ptr", (PyCFunction)(void (*)(void))ptr, METH_FASTCALL, "ptr(tensor or None, name, numel, types, device): its device pointer"},
    {"rows", (PyCFunction)(void (*)(void))rows, METH_FASTCALL, "rows(matrix or None, name, n, d, types, device): its pointer and row distance"},
    {"device", device, METH_NOARGS, "device(): index of the current CUDA device, -1 without one"},
    {"type", type, METH_O, "type(tensor): the bit of its element type"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "sl_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_sl_args() { return PyModule_Create(&module); }
