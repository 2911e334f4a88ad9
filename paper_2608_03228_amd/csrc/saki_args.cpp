// Argument marshalling of the Python binding's serving calls, as a CPython
// module (_saki_args): what a decode step calls takes 4 to 10 us on the GPU, and
// checking a call's tensors and converting its arguments took 6 us in Python
// and ctypes (1 here, where the tensors are read through torch's C++ types).
//
//   array(t, dtype, shape, dev, name)  data pointer of a dense tensor of this
//                                type and shape on this device
//   rows(t, dtype, shape, dev, name)   (data pointer, elements between tokens) of
//                                token rows [T, H, d] with dense heads
//   refusal(f)                   what array and rows call, with their arguments,
//                                for a tensor that is not so; it raises
//   saki_...(...)                the C entry points: None or an int for a pointer,
//                                ints and floats for numbers; the status or size

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstdint>
#include <exception>
#include <tuple>
#include <type_traits>
#include <utility>

#include "saki.h"

namespace {

PyObject* g_refusal = nullptr;

PyObject* refuse(PyObject* const* a) {
  if (g_refusal) {
    PyObject* r = PyObject_Vectorcall(g_refusal, a, 5, nullptr);
    Py_XDECREF(r);
  }
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an argument is not the tensor that is wanted");
  return nullptr;
}

// The tensor if it has this dtype and shape and lies on this device.
const at::Tensor* matching(PyObject* const* a) {
  if (!THPVariable_Check(a[0]) || !THPDtype_Check(a[1]) || !PyTuple_Check(a[2])) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(a[0]);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.is_neg() || t.is_conj() ||
      t.scalar_type() != reinterpret_cast<THPDtype*>(a[1])->scalar_type)
    return nullptr;
  const long dev = PyLong_AsLong(a[3]);
  const Py_ssize_t n = PyTuple_GET_SIZE(a[2]);
  if (t.get_device() != dev || t.dim() != n) return nullptr;
  for (Py_ssize_t i = 0; i < n; ++i)
    if (t.size(i) != PyLong_AsLongLong(PyTuple_GET_ITEM(a[2], i))) return nullptr;
  return &t;
}

// torch's accessors throw for tensors without memory of their own.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(a, n);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_ValueError, "an argument has no memory to point to");
  }
  return nullptr;
}

PyObject* array(PyObject* const* a, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "array takes 5 arguments");
    return nullptr;
  }
  const at::Tensor* t = matching(a);
  if (PyErr_Occurred()) return nullptr;
  return t && t->is_contiguous() ? PyLong_FromVoidPtr(t->data_ptr()) : refuse(a);
}

PyObject* rows(PyObject* const* a, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "rows takes 5 arguments");
    return nullptr;
  }
  const at::Tensor* t = matching(a);
  if (PyErr_Occurred()) return nullptr;
  if (!t || t->dim() != 3) return refuse(a);
  const int64_t T = t->size(0), H = t->size(1), d = t->size(2);
  int64_t ld = H * d;
  if (!t->is_contiguous()) {
    if ((t->stride(2) != 1 && d != 1) || (t->stride(1) != d && H != 1) || (t->stride(0) < ld && T != 1))
      return refuse(a);
    if (T > 1) ld = t->stride(0);
  }
  PyObject *p = PyLong_FromVoidPtr(t->data_ptr()), *l = PyLong_FromLongLong(ld);
  PyObject* r = p && l ? PyTuple_Pack(2, p, l) : nullptr;
  Py_XDECREF(p);
  Py_XDECREF(l);
  return r;
}

PyObject* refusal(PyObject*, PyObject* f) {
  Py_INCREF(f);
  Py_XSETREF(g_refusal, f);
  Py_RETURN_NONE;
}

template <typename T>
bool convert(PyObject* o, T* to) {
  if constexpr (std::is_pointer_v<T>) {
    *to = o == Py_None ? nullptr : (T)PyLong_AsVoidPtr(o);
    return *to || !PyErr_Occurred();
  } else if constexpr (std::is_floating_point_v<T>) {
    const double v = PyFloat_AsDouble(o);
    *to = (T)v;
    return v != -1.0 || !PyErr_Occurred();
  } else if constexpr (sizeof(T) == 8) {
    *to = PyLong_AsSize_t(o);
    return *to != (T)-1 || !PyErr_Occurred();
  } else {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v < INT_MIN || v > INT_MAX) {
      PyErr_SetString(PyExc_OverflowError, "an argument does not fit an int");
      return false;
    }
    *to = (T)v;
    return true;
  }
}

template <auto Fn>
struct Entry;
template <typename R, typename... A, R (*Fn)(A...)>
struct Entry<Fn> {
  template <size_t... I>
  static PyObject* run(PyObject* const* a, std::index_sequence<I...>) {
    std::tuple<A...> v;
    if (!(convert(a[I], &std::get<I>(v)) && ...)) return nullptr;
    R result;
    Py_BEGIN_ALLOW_THREADS;
    result = Fn(std::get<I>(v)...);
    Py_END_ALLOW_THREADS;
    if constexpr (std::is_same_v<R, size_t>)
      return PyLong_FromSize_t(result);
    else
      return PyLong_FromLong(result);
  }
  static PyObject* call(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != (Py_ssize_t)sizeof...(A)) {
      PyErr_Format(PyExc_TypeError, "%d arguments are wanted, got %zd", (int)sizeof...(A), n);
      return nullptr;
    }
    return run(a, std::index_sequence_for<A...>());
  }
};

#define SAKI_ENTRY(f) {#f, (PyCFunction)(void (*)(void))Entry<&f>::call, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"array", (PyCFunction)(void (*)(void))guarded<array>, METH_FASTCALL, nullptr},
    {"rows", (PyCFunction)(void (*)(void))guarded<rows>, METH_FASTCALL, nullptr},
    {"refusal", refusal, METH_O, nullptr},
    SAKI_ENTRY(saki_rope),
    SAKI_ENTRY(saki_block_tables),
    SAKI_ENTRY(saki_cache_write),
    SAKI_ENTRY(saki_cache_attend),
    SAKI_ENTRY(saki_cache_attend_workspace_bytes),
    SAKI_ENTRY(saki_attend_prompt),
    SAKI_ENTRY(saki_attend_prompt_workspace_bytes),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_saki_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__saki_args() { return PyModule_Create(&module); }
