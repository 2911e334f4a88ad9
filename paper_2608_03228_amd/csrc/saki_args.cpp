// Argument marshalling of the Python binding's serving calls, as a CPython
// module (_saki_args): what a decode step calls takes 4 to 10 us on the GPU, and
// checking a call's tensors and converting its arguments took 6 us in Python
// and ctypes (1.5 here).
//
//   array(t, dtype, shape, dev)  data pointer of a dense tensor of this type and
//                                shape on this device, None if it is not one
//   rows(t, dtype, shape, dev)   (data pointer, elements between tokens) of token
//                                rows [T, H, d] with dense heads, None likewise
//   saki_...(...)                the C entry points: None or an int for a pointer,
//                                ints and floats for numbers; the status or size

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <cstdint>
#include <tuple>
#include <type_traits>
#include <utility>

#include "saki.h"

namespace {

PyObject *s_dtype, *s_shape, *s_get_device, *s_is_contiguous, *s_data_ptr, *s_stride;

struct Ref {  // an owned reference
  PyObject* p;
  explicit Ref(PyObject* o) : p(o) {}
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
  ~Ref() { Py_XDECREF(p); }
};

// Whether t has this dtype and shape and lies on this device; -1 on an error.
int matches(PyObject* t, PyObject* dtype, PyObject* shape, PyObject* dev) {
  Ref d(PyObject_GetAttr(t, s_dtype));
  if (!d.p) return -1;
  if (d.p != dtype) return 0;
  Ref g(PyObject_CallMethodNoArgs(t, s_get_device));
  if (!g.p) return -1;
  int same = PyObject_RichCompareBool(g.p, dev, Py_EQ);
  if (same != 1) return same;
  Ref s(PyObject_GetAttr(t, s_shape));
  if (!s.p) return -1;
  return PyObject_RichCompareBool(s.p, shape, Py_EQ);
}

int contiguous(PyObject* t) {
  Ref c(PyObject_CallMethodNoArgs(t, s_is_contiguous));
  return c.p ? PyObject_IsTrue(c.p) : -1;
}

// The caller looks again, and says what is wrong, where this is None.
PyObject* none() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

PyObject* array(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "array takes 4 arguments");
    return nullptr;
  }
  if (matches(a[0], a[1], a[2], a[3]) != 1 || contiguous(a[0]) != 1) return none();
  return PyObject_CallMethodNoArgs(a[0], s_data_ptr);
}

PyObject* rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4 || !PyTuple_Check(a[2]) || PyTuple_GET_SIZE(a[2]) != 3) {
    PyErr_SetString(PyExc_TypeError, "rows takes 4 arguments, the third of 3 sizes");
    return nullptr;
  }
  if (matches(a[0], a[1], a[2], a[3]) != 1) return none();
  long long size[3], st[3];
  for (int i = 0; i < 3; ++i) {
    size[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(a[2], i));
    if (size[i] < 0 || size[i] > INT_MAX) return none();
  }
  long long ld = size[1] * size[2];
  const int dense = contiguous(a[0]);
  if (dense < 0) return none();
  if (!dense) {
    Ref s(PyObject_CallMethodNoArgs(a[0], s_stride));
    if (!s.p || !PyTuple_Check(s.p) || PyTuple_GET_SIZE(s.p) != 3) return none();
    for (int i = 0; i < 3; ++i) st[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s.p, i));
    if (PyErr_Occurred()) return none();
    if ((st[2] != 1 && size[2] != 1) || (st[1] != size[2] && size[1] != 1) || (st[0] < ld && size[0] != 1))
      return none();
    if (size[0] > 1) ld = st[0];
  }
  Ref p(PyObject_CallMethodNoArgs(a[0], s_data_ptr));
  return p.p ? Py_BuildValue("(OL)", p.p, ld) : nullptr;
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
    {"array", (PyCFunction)(void (*)(void))array, METH_FASTCALL, nullptr},
    {"rows", (PyCFunction)(void (*)(void))rows, METH_FASTCALL, nullptr},
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

PyMODINIT_FUNC PyInit__saki_args() {
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_stride = PyUnicode_InternFromString("stride");
  if (!s_dtype || !s_shape || !s_get_device || !s_is_contiguous || !s_data_ptr || !s_stride) return nullptr;
  return PyModule_Create(&module);
}
