// What the binding's two marshalling sources share (attn_marshal.cpp, attn_paged_marshal.cpp): Python errors as C++ exceptions, arguments out of Python objects.
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "../../include/attn.h"

namespace marshal {

extern PyObject* attn_error;   // binding.AttnError

struct Raised {};   // a Python error is set

[[noreturn]] inline void raise(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw Raised();
}

inline void check_status(int status, const char* where) {
  if (status == ATTN_OK) return;
  PyObject* e = PyObject_CallFunction(attn_error, "is", status, where);
  if (e != nullptr) {
    PyErr_SetObject(attn_error, e);
    Py_DECREF(e);
  }
  throw Raised();
}

inline const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a torch.Tensor");
  return THPVariable_Unpack(o);
}
inline void* data(PyObject* o) {   // of a buffer the library checks for: None is its NULL
  return o == Py_None ? nullptr : tensor(o).data_ptr();
}
inline PyObject* wrap(const at::Tensor& t) {
  PyObject* o = THPVariable_Wrap(t);
  if (o == nullptr) throw Raised();
  return o;
}
inline double number(PyObject* o) {   // float(o)
  PyObject* f = PyNumber_Float(o);
  if (f == nullptr) throw Raised();
  const double v = PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  return v;
}
inline bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised();
  return v != 0;
}
inline uint64_t low64(PyObject* o) {   // int(o) & (2^64 - 1)
  PyObject* i = PyNumber_Long(o);
  if (i == nullptr) throw Raised();
  const uint64_t v = PyLong_AsUnsignedLongLongMask(i);
  Py_DECREF(i);
  if (v == (uint64_t)-1 && PyErr_Occurred()) throw Raised();
  return v;
}

inline int32_t clamped32(PyObject* o) {   // an integer, kept within 32 bits
  PyObject* i = PyNumber_Index(o);
  if (i == nullptr) throw Raised();
  int beyond = 0;
  const long long v = PyLong_AsLongLongAndOverflow(i, &beyond);
  Py_DECREF(i);
  if (beyond != 0) return beyond > 0 ? INT32_MAX : INT32_MIN;
  return v > INT32_MAX ? INT32_MAX : (v < INT32_MIN ? INT32_MIN : (int32_t)v);
}

// The library call itself runs without the interpreter lock.
template <typename F> int without_gil(F&& f) {
  PyThreadState* s = PyEval_SaveThread();
  const int status = f();
  PyEval_RestoreThread(s);
  return status;
}

template <typename F> PyObject* guarded(F&& f) {
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

inline PyObject* tuple(std::initializer_list<PyObject*> items) {   // takes the references over
  PyObject* t = PyTuple_New((Py_ssize_t)items.size());
  if (t == nullptr) throw Raised();
  Py_ssize_t i = 0;
  for (PyObject* o : items) PyTuple_SET_ITEM(t, i++, o);
  return t;
}

// An error on the engine's thread, which runs without the interpreter lock: `set` raises it, and it is carried to the caller of backward().
template <typename F> [[noreturn]] void refused_in_backward(F&& set) {
  const PyGILState_STATE gil = PyGILState_Ensure();
  python_error e;
  try {
    set();
  } catch (const Raised&) {
    e.persist();
  }
  PyGILState_Release(gil);
  throw e;
}

// Of a forward pass under capture (attn_paged_marshal.cpp).
void refuse_eager_graphs(std::initializer_list<const at::Tensor*> tensors);

// Where the gradients of a node are themselves recorded (create_graph): to differentiate them again is an error, whichever of the node's inputs is asked for.
void mark_once_differentiable(const torch::autograd::Node& node, torch::autograd::variable_list& grads, const char* text);

// The functions of attn_paged_marshal.cpp, ended by an empty entry.
extern PyMethodDef paged_methods[];

}  // namespace marshal
