// Native part of the ctypes binding: conversion of Python lists (called with PyDLL: the GIL is held), and the calls that
// a program makes in every layer, as functions of a module "libmarshal".
#include <Python.h>

#include <cstdint>
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

PyObject* g_value;   // the attribute's name

// An address: an int, None, or an object with an int or None as its `value` (ctypes.c_void_p).  False, with no exception
// set, for anything else.
bool address_of(PyObject* o, uint64_t* out) {
  if (o == Py_None) return *out = 0, true;
  if (PyLong_CheckExact(o)) {
    *out = PyLong_AsUnsignedLongLong(o);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
  }
  if (PyFloat_Check(o) || PyLong_Check(o)) return false;
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

#define OXY_METHOD(name) {#name, (PyCFunction)(void (*)())call<decltype(&name)>, METH_FASTCALL, nullptr}
PyMethodDef g_calls[] = {OXY_METHOD(oxy_mixed_attention), OXY_METHOD(oxy_mixed_attention_static), OXY_METHOD(oxy_stream_append),
                         OXY_METHOD(oxy_append_attention), OXY_METHOD(oxy_rotary_append), OXY_METHOD(oxy_rotary),
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
  g_value = PyUnicode_InternFromString("value");
  return g_value ? PyModule_Create(&g_module) : nullptr;
}
