// The binding's calls of the C ABI for work that takes the GPU a few microseconds,
// as CPython functions: arguments are read where they lie on the interpreter's stack,
// without ctypes' conversion objects (an rbq_quantize_kv call with its checks: 4.3 us
// of the host through ctypes, 2.5 here, and 0.2 since rows are judged by what their views span;
// its kernel for one token takes 3). The
// entry points are those that the ctypes library has loaded: bind() takes their addresses.
//
// An argument of a pointer type is None, an address, or an object with data_ptr().
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <tuple>
#include <utility>

#include "../../include/rbq.h"

namespace {

PyObject *str_data_ptr, *str_numel, *str_shape, *str_stride, *str_contiguous;

bool take(PyObject* o, int64_t& v) {
  v = PyLong_AsLong(o);
  return v != -1 || !PyErr_Occurred();
}
bool take(PyObject* o, int32_t& v) {
  int64_t x;
  if (!take(o, x)) return false;
  v = int32_t(x);
  if (v == x) return true;
  PyErr_Format(PyExc_OverflowError, "%lld does not fit into 32 bits", (long long)x);
  return false;
}
bool take(PyObject* o, size_t& v) {
  v = PyLong_AsSize_t(o);
  return v != size_t(-1) || !PyErr_Occurred();
}
bool take(PyObject* o, float& v) {
  const double x = PyFloat_AsDouble(o);
  v = float(x);
  return x != -1.0 || !PyErr_Occurred();
}
template <class T>
bool take(PyObject* o, T*& v) {
  if (o == Py_None) {
    v = nullptr;
    return true;
  }
  if (PyLong_Check(o)) {
    v = static_cast<T*>(PyLong_AsVoidPtr(o));
  } else {
    PyObject* p = PyObject_CallMethodNoArgs(o, str_data_ptr);
    if (p == nullptr) return false;
    v = static_cast<T*>(PyLong_AsVoidPtr(p));
    Py_DECREF(p);
  }
  return v != nullptr || !PyErr_Occurred();
}

enum {
  kQuantize, kDequantize, kDense, kSparse, kStep, kPrefill,
  kQuantize4, kDequantize4, kDense4, kSparse4, kStep4, kPrefill4,
  kEntries
};
void* entry[kEntries];

template <class F>
struct Entry;
template <class... A>
struct Entry<rbq_status (*)(A...)> {
  template <int E, size_t... I>
  static PyObject* call(PyObject* const* args, std::index_sequence<I...>) {
    std::tuple<A...> v;
    if (!(take(args[I], std::get<I>(v)) && ...)) return nullptr;
    const auto fn = reinterpret_cast<rbq_status (*)(A...)>(entry[E]);
    rbq_status st;
    Py_BEGIN_ALLOW_THREADS
    st = fn(std::get<I>(v)...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
  }
  template <int E>
  static PyObject* run(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != Py_ssize_t(sizeof...(A)) || entry[E] == nullptr)
      return PyErr_Format(PyExc_TypeError, "%zd arguments, the call takes %zu", n, sizeof...(A));
    return call<E>(args, std::index_sequence_for<A...>{});
  }
};

// elements of a buffer
bool elements_of(PyObject* o, int64_t& have) {
  PyObject* r = PyObject_CallMethodNoArgs(o, str_numel);
  if (r == nullptr) return false;
  const bool ok = take(r, have);
  Py_DECREF(r);
  return ok;
}

// elements from a view's first to its last, gaps included: 1 + sum (size - 1) stride
bool span_of(PyObject* o, int64_t& have) {
  PyObject* shape = PyObject_GetAttr(o, str_shape);
  PyObject* stride = shape != nullptr ? PyObject_CallMethodNoArgs(o, str_stride) : nullptr;
  bool ok = stride != nullptr && PyTuple_Check(shape) && PyTuple_Check(stride) &&
            PyTuple_GET_SIZE(shape) == PyTuple_GET_SIZE(stride);
  int64_t last = 0;
  for (Py_ssize_t d = 0; ok && d < PyTuple_GET_SIZE(shape); ++d) {
    int64_t size, step;
    ok = take(PyTuple_GET_ITEM(shape, d), size) && take(PyTuple_GET_ITEM(stride, d), step);
    if (ok) last += (size - 1) * step;
  }
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  if (ok) have = 1 + last;
  else if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "a buffer without sizes and strides");
  return ok;
}

// fits(rows, buffer, elements, buffer, elements, ...): whether every buffer that knows its size
// reaches as far as the call needs (None and addresses know nothing). The first `rows` buffers
// are judged by what they span, more than their elements where a view has gaps between its
// rows, less where it repeats them; the others by their elements.
PyObject* fits(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n % 2 == 0) return PyErr_Format(PyExc_TypeError, "a number, and pairs of a buffer and its elements");
  int64_t rows;
  if (!take(args[0], rows)) return nullptr;
  for (Py_ssize_t i = 1; i < n; i += 2) {
    int64_t need, have;
    if (!take(args[i + 1], need)) return nullptr;
    if (args[i] == Py_None || PyLong_Check(args[i])) continue;
    if (!elements_of(args[i], have)) return nullptr;
    if (i < 2 * rows && have > 0) {
      PyObject* c = PyObject_CallMethodNoArgs(args[i], str_contiguous);
      if (c == nullptr) return nullptr;
      Py_DECREF(c);
      if (c != Py_True && !span_of(args[i], have)) return nullptr;
    }
    if (have < need) Py_RETURN_FALSE;
  }
  Py_RETURN_TRUE;
}

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != kEntries) return PyErr_Format(PyExc_TypeError, "%d addresses", int(kEntries));
  for (int e = 0; e < kEntries; ++e)
    if (!take(args[e], entry[e])) return nullptr;
  Py_RETURN_NONE;
}

#define RBQ_ENTRY(NAME, E) \
  {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&Entry<decltype(&NAME)>::run<E>)), METH_FASTCALL, nullptr}
#define RBQ_HELPER(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RBQ_ENTRY(rbq_quantize_kv, kQuantize),
                         RBQ_ENTRY(rbq_dequantize_kv, kDequantize),
                         RBQ_ENTRY(rbq_dense_decode_kv8, kDense),
                         RBQ_ENTRY(rbq_sparse_decode_kv8, kSparse),
                         RBQ_ENTRY(rbq_decode_step_kv8, kStep),
                         RBQ_ENTRY(rbq_prefill_attention, kPrefill),
                         RBQ_ENTRY(rbq_quantize_kv4, kQuantize4),
                         RBQ_ENTRY(rbq_dequantize_kv4, kDequantize4),
                         RBQ_ENTRY(rbq_dense_decode_kv4, kDense4),
                         RBQ_ENTRY(rbq_sparse_decode_kv4, kSparse4),
                         RBQ_ENTRY(rbq_decode_step_kv4, kStep4),
                         RBQ_ENTRY(rbq_prefill_attention_kv4, kPrefill4),
                         RBQ_HELPER(fits),
                         RBQ_HELPER(bind),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_rbqcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rbqcall(void) {
  str_data_ptr = PyUnicode_InternFromString("data_ptr");
  str_numel = PyUnicode_InternFromString("numel");
  str_shape = PyUnicode_InternFromString("shape");
  str_stride = PyUnicode_InternFromString("stride");
  str_contiguous = PyUnicode_InternFromString("is_contiguous");
  return str_data_ptr && str_numel && str_shape && str_stride && str_contiguous ? PyModule_Create(&module_def) : nullptr;
}
