// Native part of the ctypes binding: conversion of Python lists (called with PyDLL: the GIL is held), and the calls that
// a program makes in every layer, as functions of a module "libmarshal".
#include <Python.h>

#include <cstdint>
#include <cstring>
#include <tuple>
#include <type_traits>
#include <utility>

#include "../../include/oxy.h"

// The n ints of `list` to `out`.  1, or 0 with no exception set where an element is not exactly an int, is
// out of range, or the list has another length: the caller then converts by Python's own means.
extern "C" int32_t oxy_ints_of_list(PyObject* list, int64_t* out, int64_t n) {
  if (!PyList_CheckExact(list) || PyList_GET_SIZE(list) != n) return 0;
  for (int64_t i = 0; i < n; ++i) {
    PyObject* o = PyList_GET_ITEM(list, i);
    if (!PyLong_CheckExact(o)) return 0;
    int overflow = 0;
    out[i] = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) return 0;
  }
  return 1;
}

namespace {

PyObject* g_value;      // the attribute's name
PyObject* g_void_p;     // ctypes.c_void_p

// An address: an int, None, or a ctypes.c_void_p.  False, with no exception set, for anything else (ctypes refuses other
// objects that have a value, numbers of its own kinds among them).
bool address_of(PyObject* o, uint64_t* out) {
  if (o == Py_None) return *out = 0, true;
  if (PyLong_CheckExact(o)) {
    *out = PyLong_AsUnsignedLongLong(o);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
  }
  if ((PyObject*)Py_TYPE(o) != g_void_p) return false;
  PyObject* v = PyObject_GetAttr(o, g_value);
  if (!v) return PyErr_Clear(), false;
  const bool ok = (v == Py_None || PyLong_CheckExact(v)) && address_of(v, out);
  Py_DECREF(v);
  return ok;
}
template <class T>
bool convert(PyObject* o, T* out) {
  if constexpr (std::is_pointer_v<T>) {
    uint64_t a = 0;
    if (!address_of(o, &a)) return false;
    *out = (T)a;
    return true;
  } else if constexpr (std::is_floating_point_v<T>) {
    if (!PyFloat_CheckExact(o)) return false;
    *out = (T)PyFloat_AS_DOUBLE(o);
    return true;
  } else {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
    *out = (T)x;
    return !overflow && (std::is_signed_v<T> ? (long long)*out == x : x >= 0);
  }
}

// Calls the library function whose address is `self`: its status, or None, and nothing called, where an argument is not
// exactly of the kinds above.  The GIL is released meanwhile, as ctypes does.
template <class... A, size_t... I>
PyObject* call_as(int32_t (*fn)(A...), PyObject* const* args, std::index_sequence<I...>) {
  std::tuple<A...> a;
  if (!(convert(args[I], &std::get<I>(a)) && ...)) Py_RETURN_NONE;
  int32_t status;
  Py_BEGIN_ALLOW_THREADS
  status = fn(std::get<I>(a)...);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}
template <class... A>
PyObject* call_with(int32_t (*fn)(A...), PyObject* const* args, Py_ssize_t n) {
  if (n != (Py_ssize_t)sizeof...(A)) Py_RETURN_NONE;
  return call_as(fn, args, std::index_sequence_for<A...>());
}
template <class Fn>
PyObject* call(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  return call_with((Fn)PyLong_AsVoidPtr(self), args, n);
}

// oxy_batch_info(batch): the four numbers as a tuple, or None where there is no such answer.
PyObject* call_info(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  const oxy_batch* batch = nullptr;
  int32_t v[4];
  if (n != 1 || !convert(args[0], &batch) ||
      ((decltype(&oxy_batch_info))PyLong_AsVoidPtr(self))(batch, v, v + 1, v + 2, v + 3) != OXY_OK)
    Py_RETURN_NONE;
  return Py_BuildValue("(iiii)", v[0], v[1], v[2], v[3]);
}
// oxy_batch_slots(batch, n): the slots as a list, or None.
PyObject* call_slots(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
  const oxy_batch* batch = nullptr;
  int32_t n = 0;
  if (n_args != 2 || !convert(args[0], &batch) || !convert(args[1], &n) || n < 1) Py_RETURN_NONE;
  int64_t* out = (int64_t*)PyMem_Malloc((size_t)n * sizeof(int64_t));
  if (!out) Py_RETURN_NONE;
  PyObject* list = nullptr;
  if (((decltype(&oxy_batch_slots))PyLong_AsVoidPtr(self))(batch, out, n) == OXY_OK && (list = PyList_New(n))) {
    for (int32_t i = 0; i < n; ++i) {
      PyObject* x = PyLong_FromLongLong(out[i]);
      if (!x) {
        Py_CLEAR(list);
        break;
      }
      PyList_SET_ITEM(list, i, x);
    }
  }
  PyMem_Free(out);
  if (list) return list;
  PyErr_Clear();
  Py_RETURN_NONE;
}
// A list of slots for the length of one call.
struct Slots {
  int64_t* v = nullptr;
  int32_t n = 0;
  explicit Slots(PyObject* list) {
    if (!PyList_CheckExact(list) || PyList_GET_SIZE(list) > INT32_MAX) return;
    n = (int32_t)PyList_GET_SIZE(list);
    v = (int64_t*)PyMem_Malloc((size_t)n * sizeof(int64_t));
    if (v && !oxy_ints_of_list(list, v, n)) release();
  }
  ~Slots() { release(); }
  void release() {
    PyMem_Free(v);
    v = nullptr;
  }
};
// Read-backs take their slots as a list of ints.
PyObject* call_gather(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  oxy_pool* pool;
  int32_t layer, status;
  void *k, *v, *stream;
  if (n != 6 || !convert(args[0], &pool) || !convert(args[1], &layer) || !convert(args[3], &k) || !convert(args[4], &v) ||
      !convert(args[5], &stream))
    Py_RETURN_NONE;
  const Slots slots(args[2]);
  if (!slots.v) Py_RETURN_NONE;
  Py_BEGIN_ALLOW_THREADS
  status = ((decltype(&oxy_gather_kv))PyLong_AsVoidPtr(self))(pool, layer, slots.v, slots.n, k, v, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}
PyObject* call_gather_layers(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  oxy_pool* pool;
  int32_t begin, end, status;
  void *k, *v, *stream;
  size_t stride;
  if (n != 8 || !convert(args[0], &pool) || !convert(args[1], &begin) || !convert(args[2], &end) || !convert(args[4], &k) ||
      !convert(args[5], &v) || !convert(args[6], &stride) || !convert(args[7], &stream))
    Py_RETURN_NONE;
  const Slots slots(args[3]);
  if (!slots.v) Py_RETURN_NONE;
  Py_BEGIN_ALLOW_THREADS
  status = ((decltype(&oxy_gather_kv_layers))PyLong_AsVoidPtr(self))(pool, begin, end, slots.v, slots.n, k, v, stride, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

#define OXY_CALL(name, function) {#name, (PyCFunction)(void (*)())function, METH_FASTCALL, nullptr}
#define OXY_METHOD(name) OXY_CALL(name, call<decltype(&name)>)
PyMethodDef g_calls[] = {OXY_METHOD(oxy_mixed_attention), OXY_METHOD(oxy_mixed_attention_static), OXY_METHOD(oxy_stream_append),
                         OXY_METHOD(oxy_append_attention), OXY_METHOD(oxy_rotary_append), OXY_METHOD(oxy_rotary),
                         OXY_METHOD(oxy_rotary_axes), OXY_METHOD(oxy_rotary_axes_append), OXY_METHOD(oxy_prefix_attention), OXY_METHOD(oxy_prompt_attention),
                         OXY_CALL(oxy_batch_info, call_info), OXY_CALL(oxy_batch_slots, call_slots),
                         OXY_CALL(oxy_gather_kv, call_gather), OXY_CALL(oxy_gather_kv_layers, call_gather_layers),
                         {nullptr, nullptr, 0, nullptr}};

// bound(name, address): the call of that name, or None
PyObject* bound(PyObject*, PyObject* args) {
  const char* name;
  PyObject* address;
  if (!PyArg_ParseTuple(args, "sO!", &name, &PyLong_Type, &address)) return nullptr;
  for (PyMethodDef* m = g_calls; m->ml_name; ++m)
    if (!strcmp(m->ml_name, name)) return PyCFunction_NewEx(m, address, nullptr);
  Py_RETURN_NONE;
}
PyMethodDef g_methods[] = {{"bound", bound, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "libmarshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_libmarshal(void) {
  PyObject* ctypes = PyImport_ImportModule("ctypes");
  if (!ctypes) return nullptr;
  g_void_p = PyObject_GetAttrString(ctypes, "c_void_p");
  Py_DECREF(ctypes);
  g_value = PyUnicode_InternFromString("value");
  return g_void_p && g_value ? PyModule_Create(&g_module) : nullptr;
}
