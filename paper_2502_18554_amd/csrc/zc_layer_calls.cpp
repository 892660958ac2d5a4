// The calls around the collective (zc_adamw, zc_mx_*) in native code: from torch's tensors to the C ABI of libzc.so.
//
// A step over a list of tensors asks each of them for address, size, type and layout.  From Python, or through Python's attributes, that is 0.4 to 0.8 us a
// tensor, more than the step itself takes on small ones; here the tensors are read as what they are, 20 ns each.  That needs the headers
// of torch and its libraries: this is a module of its own, which is only used with the torch that it was built for; without it these calls go through ctypes, and the
// codec's native calls (zc_calls.cpp) are as they were.
// Nothing is decided here: what is not of a plain form, or does not fit together, is answered with NotImplemented, and binding.py takes the call its own way.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstdint>
#include <vector>

#include "../../include/zc.h"
#include "zc_calls_stream.h"

namespace {

zc_calls::Streams g_streams;
bool stream_of(PyObject* given, void*& stream) { return g_streams.of(given, stream); }

struct Calls {
  decltype(&zc_adamw) adamw;
  decltype(&zc_mx_quantize) quantize;
  decltype(&zc_mx_dequantize) dequantize;
  decltype(&zc_mx_product) product;
  decltype(&zc_mx_linear) linear;
} g_calls;

PyObject* not_this_way() {
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NOTIMPLEMENTED;
}

const at::Tensor* tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}
int type_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return ZC_F32;
    case at::kBFloat16: return ZC_BF16;
    case at::kHalf: return ZC_F16;
    default: return -1;
  }
}

struct Matrix {
  void* at;
  int type;
  size_t rows, cols, stride;
};
bool matrix(PyObject* o, Matrix& m) {
  const at::Tensor* const t = tensor(o);
  if (!t || t->dim() != 2) return false;
  m.type = type_of(*t);
  m.rows = size_t(t->size(0)), m.cols = size_t(t->size(1));
  m.at = t->data_ptr();
  m.stride = m.rows > 1 || size_t(t->stride(0)) > m.cols ? size_t(t->stride(0)) : m.cols;
  return m.type >= 0 && (m.cols <= 1 || t->stride(1) == 1);
}

struct Held {
  void *codes, *scales;
  size_t codes_stride, scales_stride;
};
bool bytes_of_rows(PyObject* o, size_t rows, size_t least, void*& at, size_t& stride) {
  const at::Tensor* const t = tensor(o);
  if (!t || t->dim() != 2 || t->scalar_type() != at::kByte || size_t(t->size(0)) != rows || size_t(t->size(1)) < least || (t->size(1) > 1 && t->stride(1) != 1)) return false;
  if (rows > 1 && t->stride(0) < t->size(1)) return false;
  at = t->data_ptr();
  stride = size_t(rows > 1 ? t->stride(0) : t->size(1));
  return true;
}
bool held(PyObject* codes, PyObject* scales, size_t rows, size_t cols, Held& h) {
  const size_t blocks = (cols + 31) / 32;
  return bytes_of_rows(codes, rows, 16 * blocks, h.codes, h.codes_stride) && bytes_of_rows(scales, rows, blocks, h.scales, h.scales_stride);
}
bool bias_of(PyObject* o, size_t n, const float*& p) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* const t = tensor(o);
  if (!t || t->scalar_type() != at::kFloat || size_t(t->numel()) != n || !t->is_contiguous()) return false;
  p = static_cast<const float*>(t->data_ptr());
  return true;
}
// A state or a workspace.
bool workspace_of(PyObject* o, void*& p, size_t& bytes) {
  const at::Tensor* const t = tensor(o);
  if (!t || !t->is_contiguous()) return false;           // (its bytes are not all its own, or not all there, otherwise)
  p = t->data_ptr();
  bytes = t->nbytes();
  return true;
}

PyObject* answer(int st) { return PyLong_FromLong(st); }

// (d_in, d_codes, d_scales, d_codes_t, d_scales_t, stream)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Matrix x;
  Held h{}, ht{};
  void* stream;
  if (n_args != 6 || !matrix(a[0], x)) return not_this_way();
  if ((a[1] != Py_None || a[2] != Py_None) && !held(a[1], a[2], x.rows, x.cols, h)) return not_this_way();
  if ((a[3] != Py_None || a[4] != Py_None) && !held(a[3], a[4], x.cols, x.rows, ht)) return not_this_way();
  if (!stream_of(a[5], stream)) return not_this_way();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = g_calls.quantize(x.at, x.type, x.rows, x.cols, x.stride, h.codes, h.codes_stride, h.scales, h.scales_stride, ht.codes, ht.codes_stride, ht.scales, ht.scales_stride, stream);
  Py_END_ALLOW_THREADS
  return answer(st);
}

// (d_codes, d_scales, d_out, stream)
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Matrix out;
  Held h;
  void* stream;
  if (n_args != 4 || !matrix(a[2], out) || !held(a[0], a[1], out.rows, out.cols, h) || !stream_of(a[3], stream)) return not_this_way();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = g_calls.dequantize(h.codes, h.codes_stride, h.scales, h.scales_stride, out.rows, out.cols, out.at, out.type, out.stride, stream);
  Py_END_ALLOW_THREADS
  return answer(st);
}

// (d_a_codes, d_a_scales, d_b_codes, d_b_scales, k, d_out, d_ws, d_bias, add, stream)
PyObject* product(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Matrix out;
  Held x, w;
  const float* bias;
  void *ws, *stream;
  size_t ws_bytes;
  if (n_args != 10 || !PyLong_CheckExact(a[4])) return not_this_way();
  const long long k = PyLong_AsLongLong(a[4]);
  if (k < 0 || k > 0x7fffffff) {
    PyErr_Clear();
    return not_this_way();
  }
  if (!matrix(a[5], out) || !held(a[0], a[1], out.rows, size_t(k), x) || !held(a[2], a[3], out.cols, size_t(k), w) || !workspace_of(a[6], ws, ws_bytes) ||
      !bias_of(a[7], out.cols, bias) || !stream_of(a[9], stream))
    return not_this_way();
  const int add = PyObject_IsTrue(a[8]);
  if (add < 0) return nullptr;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = g_calls.product(x.codes, x.codes_stride, x.scales, x.scales_stride, w.codes, w.codes_stride, w.scales, w.scales_stride, out.rows, out.cols, size_t(k), bias, out.at, out.type,
                       out.stride, add ? ZC_MX_ADD : 0u, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return answer(st);
}

// (d_x, d_w_codes, d_w_scales, d_out, d_ws, d_bias, add, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Matrix x, out;
  Held w;
  const float* bias;
  void *ws, *stream;
  size_t ws_bytes;
  if (n_args != 8 || !matrix(a[0], x) || !matrix(a[3], out) || out.rows != x.rows || !held(a[1], a[2], out.cols, x.cols, w) || !workspace_of(a[4], ws, ws_bytes) ||
      !bias_of(a[5], out.cols, bias) || !stream_of(a[7], stream))
    return not_this_way();
  const int add = PyObject_IsTrue(a[6]);
  if (add < 0) return nullptr;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = g_calls.linear(x.at, x.type, x.stride, w.codes, w.codes_stride, w.scales, w.scales_stride, out.rows, out.cols, x.cols, bias, out.at, out.type, out.stride,
                      add ? ZC_MX_ADD : 0u, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return answer(st);
}

// A list's tensors, of one type and contiguous; sizes are written or, `same`, compared.
bool list_of(PyObject* list, Py_ssize_t k, bool same, std::vector<size_t>& sizes, void** to, int& type) {
  if (!PyList_CheckExact(list) || PyList_GET_SIZE(list) != k) return false;
  for (Py_ssize_t i = 0; i < k; ++i) {                    // (nothing of Python runs that could change the list)
    const at::Tensor* const t = tensor(PyList_GET_ITEM(list, i));
    if (!t || !t->is_contiguous()) return false;
    const int kind = type_of(*t);
    if (kind < 0 || (i && kind != type)) return false;
    type = kind;
    if (same && sizes[size_t(i)] != size_t(t->numel())) return false;
    sizes[size_t(i)] = size_t(t->numel());
    to[i] = t->data_ptr();
  }
  return true;
}

bool real(PyObject* o, double& v) {
  if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
  v = PyFloat_AsDouble(o);
  return !PyErr_Occurred();
}
bool word(PyObject* o, uint64_t& v) {
  if (!PyLong_CheckExact(o)) return false;
  v = PyLong_AsUnsignedLongLong(o);
  if (!PyErr_Occurred()) return true;
  PyErr_Clear();
  return false;
}

// (d_params, d_grads, d_state, step, lr, beta1, beta2, eps, weight_decay, state_bits, seed, d_copies, d_grad_scale, stream)
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  uint64_t step, bits, seed;
  double c[5];
  void *state, *stream;
  size_t state_bytes;
  const float* scale;
  if (n_args != 14 || !PyList_CheckExact(a[0]) || !PyList_GET_SIZE(a[0])) return not_this_way();
  const Py_ssize_t k = PyList_GET_SIZE(a[0]);
  if (k > 0x7fffffff || !word(a[3], step) || !word(a[9], bits) || bits > 32 || !word(a[10], seed)) return not_this_way();
  for (int i = 0; i < 5; ++i)
    if (!real(a[4 + i], c[i])) return not_this_way();
  std::vector<size_t> sizes(static_cast<size_t>(k));
  std::vector<void*> at(static_cast<size_t>(3 * k));
  int types[3] = {ZC_F32, ZC_F32, ZC_F32};
  const bool copies = a[11] != Py_None;
  if (!list_of(a[0], k, false, sizes, at.data(), types[0]) || !list_of(a[1], k, true, sizes, at.data() + k, types[1]) ||
      (copies && !list_of(a[11], k, true, sizes, at.data() + 2 * k, types[2])) || !workspace_of(a[2], state, state_bytes) || !bias_of(a[12], 1, scale) ||
      !stream_of(a[13], stream))
    return not_this_way();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = g_calls.adamw(int(k), sizes.data(), at.data(), types[0], const_cast<const void* const*>(at.data() + k), types[1], copies ? at.data() + 2 * k : nullptr, types[2], state,
                     state_bytes, int(bits), step, c[0], c[1], c[2], c[3], c[4], scale, seed, stream);
  Py_END_ALLOW_THREADS
  return answer(st);
}

// (addresses of the five calls in the order of Calls, torch's version): whether the module can be used.
PyObject* setup_layers(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  uint64_t at[5];
  if (n_args != 6 || !PyUnicode_Check(a[5])) {
    PyErr_SetString(PyExc_TypeError, "setup_layers takes five addresses and a version");
    return nullptr;
  }
  for (int i = 0; i < 5; ++i)
    if (!word(a[i], at[i]) || !at[i]) {
      PyErr_SetString(PyExc_ValueError, "setup_layers: the address of a call is missing");
      return nullptr;
    }
  if (PyUnicode_CompareWithASCIIString(a[5], TORCH_VERSION) != 0) Py_RETURN_FALSE;
  g_calls.adamw = reinterpret_cast<decltype(g_calls.adamw)>(at[0]);
  g_calls.quantize = reinterpret_cast<decltype(g_calls.quantize)>(at[1]);
  g_calls.dequantize = reinterpret_cast<decltype(g_calls.dequantize)>(at[2]);
  g_calls.product = reinterpret_cast<decltype(g_calls.product)>(at[3]);
  g_calls.linear = reinterpret_cast<decltype(g_calls.linear)>(at[4]);
  Py_RETURN_TRUE;
}

// (torch's current device, its raw current stream)
PyObject* setup_streams(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 2) {
    PyErr_SetString(PyExc_TypeError, "setup_streams takes two functions");
    return nullptr;
  }
  g_streams.set(a[0], a[1]);
  Py_RETURN_NONE;
}

// (A tensor without memory of its own throws when it is asked for its address, and a list may be too long for the memory that is left.)
using Call = PyObject*(PyObject*, PyObject* const*, Py_ssize_t);
template <Call* F>
PyObject* caught(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(self, a, n);
  } catch (...) {
    return not_this_way();
  }
}
template <Call* F>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&caught<F>)), METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {method<setup_layers>("setup_layers"), method<setup_streams>("setup_streams"), method<adamw>("adamw"), method<quantize>("quantize"),
                           method<dequantize>("dequantize"), method<product>("product"), method<linear>("linear"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_zc_layer_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__zc_layer_calls() {
  g_streams.cuda_stream = PyUnicode_InternFromString("cuda_stream");
  return g_streams.cuda_stream ? PyModule_Create(&g_module) : nullptr;
}
