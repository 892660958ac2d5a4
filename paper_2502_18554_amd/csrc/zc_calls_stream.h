// The stream of a native call: as given, or torch's current one.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>

namespace zc_calls {

struct Streams {
  PyObject *device, *raw;            // torch's own: the current device, and the current stream's handle on a device
  PyObject* cuda_stream;             // a name

  void set(PyObject* new_device, PyObject* new_raw) {
    PyObject* const old_device = device;
    PyObject* const old_raw = raw;
    device = Py_NewRef(new_device);
    raw = Py_NewRef(new_raw);
    Py_XDECREF(old_device);
    Py_XDECREF(old_raw);
  }
  // False where the object is not of a plain form (nothing raised), or with an exception set.
  bool of(PyObject* given, void*& stream) const {
    if (!device) return false;
    if (given != Py_None) return handle(PyObject_GetAttr(given, cuda_stream), stream);
    PyObject* const now = PyObject_CallNoArgs(device);
    if (!now) return false;
    PyObject* const r = PyObject_CallOneArg(raw, now);
    Py_DECREF(now);
    return handle(r, stream);
  }
  static bool handle(PyObject* r, void*& stream) {
    if (!r) return false;
    uint64_t v = 0;
    bool ok = PyLong_CheckExact(r);
    if (ok) {
      v = PyLong_AsUnsignedLongLong(r);
      if (v == ~uint64_t(0) && PyErr_Occurred()) {
        PyErr_Clear();
        ok = false;
      }
    }
    Py_DECREF(r);
    stream = reinterpret_cast<void*>(v);
    return ok;
  }
};

}  // namespace zc_calls
