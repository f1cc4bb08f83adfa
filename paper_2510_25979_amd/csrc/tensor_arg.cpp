// What the ctypes binding asks of every tensor argument, in one native call: is it a plain GPU tensor,
// contiguous, of the expected type and shape, and where does it start?  In Python these are six attribute look-ups and
// two tuples, 0.5 us a tensor (0.1 here).  attention_exact with five tensors takes 5.2 us of the host's time a call, 7.0 to
// 8.1 in Python; that is what small calls cost, and nothing where the kernel takes longer (64 x 12 heads of 64 x 64: 7.6 either way).
//
// Only the answer "yes" is given here.  Anything else -- a subclass, a tensor without storage, a wrong shape -- is None,
// and the Python code behind it decides and says what is wrong.
//
// Beside it calls of entry points with many arguments: their C types come from the header, so that a call is a conversion a number and no
// look-up (attncache_rotate's 28 arguments 0.6 us, by ctypes 2.4).
#include "../../include/attncache.h"

#include <limits>
#include <tuple>
#include <type_traits>
#include <utility>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

bool has_shape(const at::Tensor& t, PyObject* shape) {
  if (!PyTuple_CheckExact(shape)) return false;
  const c10::IntArrayRef sizes = t.sizes();
  if (PyTuple_GET_SIZE(shape) != (Py_ssize_t)sizes.size()) return false;
  for (size_t i = 0; i < sizes.size(); ++i) {
    PyObject* n = PyTuple_GET_ITEM(shape, (Py_ssize_t)i);
    if (!PyLong_CheckExact(n)) return false;
    int overflow = 0;
    if (PyLong_AsLongLongAndOverflow(n, &overflow) != sizes[i] || overflow) return false;
  }
  return true;
}

// address(tensor, dtype or None, shape or None) -> int or None
PyObject* address(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "address(tensor, dtype, shape)");
    return nullptr;
  }
  try {
    if (THPVariable_CheckExact(args[0])) {
      const at::Tensor& t = THPVariable_Unpack(args[0]);
      if (t.is_cuda() && t.is_contiguous() &&
          (args[1] == Py_None || (THPDtype_Check(args[1]) &&
                                  reinterpret_cast<THPDtype*>(args[1])->scalar_type == t.scalar_type())) &&
          (args[2] == Py_None || has_shape(t, args[2])))
        return PyLong_FromVoidPtr(t.data_ptr());
    }
  } catch (...) {   // (what Python raises for the same question, it raises itself)
  }
  Py_RETURN_NONE;
}

template <typename T>
bool take(PyObject* from, T* to) {
  if constexpr (std::is_pointer_v<T>) {
    *to = from == Py_None ? nullptr : static_cast<T>(PyLong_AsVoidPtr(from));
  } else if constexpr (std::is_floating_point_v<T>) {
    *to = static_cast<T>(PyFloat_AsDouble(from));
  } else if constexpr (std::is_same_v<T, size_t>) {
    *to = PyLong_AsSize_t(from);
  } else {
    const long long v = PyLong_AsLongLong(from);
    *to = static_cast<T>(v);
    if (v != *to) PyErr_Format(PyExc_OverflowError, "%lld is out of range", v);
  }
  return !PyErr_Occurred();
}
// entry(address, arguments ...) -> status
template <typename F>
struct Entry;
template <typename... A>
struct Entry<int32_t(A...)> {
  static PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 1 + (Py_ssize_t)sizeof...(A)) {
      PyErr_Format(PyExc_TypeError, "an address and %zd arguments, %zd given", (Py_ssize_t)sizeof...(A), n - 1);
      return nullptr;
    }
    return with(args, std::index_sequence_for<A...>{});
  }
  template <size_t... I>
  static PyObject* with(PyObject* const* args, std::index_sequence<I...>) {
    void* entry = nullptr;
    std::tuple<A...> a;
    if (!take(args[0], &entry) || !(take(args[I + 1], &std::get<I>(a)) && ...)) return nullptr;
    if (!entry) {
      PyErr_SetString(PyExc_ValueError, "no address");
      return nullptr;
    }
    int32_t status;
    Py_BEGIN_ALLOW_THREADS
    status = reinterpret_cast<int32_t (*)(A...)>(entry)(std::get<I>(a)...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
  }
};
#define AC_ENTRY(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(Entry<decltype(name)>::call)), METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    AC_ENTRY(attncache_rotate), AC_ENTRY(attncache_page_fork), AC_ENTRY(attention_paged_shared), AC_ENTRY(attention_window),
    AC_ENTRY(attention_paged_window),
    {"address", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(address)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_arg", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_arg() { return PyModule_Create(&module); }
