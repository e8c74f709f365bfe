// The Python binding's short way into the paged calls: reads the tensors' attributes, checks them and calls the C
// ABI, in one step.  A serving step makes these calls once per layer, and through ctypes with the checks in
// Python one took 9 to 14 us of host time, two to five times what its kernels run.
//
// Each function returns the call's status, or None where an argument is not what the call takes (or is
// of another kind than the common one): the caller then goes the long way, which says what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>

#include "aatc.h"

namespace {

PyObject *s_is_cuda, *s_dtype, *s_shape, *s_stride, *s_data_ptr;
PyObject *g_int32, *g_float32, *g_bf16, *g_f16;               // torch's dtypes
PyObject *g_raw_stream, *g_device;                            // the current stream's handle

struct View {
  int ndim;
  int64_t size[4], stride[4];
  void* ptr;
  bool contiguous() const {
    int64_t n = 1;
    for (int i = ndim - 1; i >= 0; --i) {
      if (size[i] > 1 && stride[i] != n) return false;
      n *= size[i];
    }
    return true;
  }
};

bool longs(PyObject* t, int n, int64_t* out) {
  for (int i = 0; i < n; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    if (out[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

// A CUDA tensor of `dtype` with `ndim` dimensions; false (with or without a Python error) for anything else.
bool view_of(PyObject* t, PyObject* dtype, int ndim, View* v) {
  PyObject* x = PyObject_GetAttr(t, s_is_cuda);
  if (!x) return false;
  Py_DECREF(x);
  if (x != Py_True) return false;
  x = PyObject_GetAttr(t, s_dtype);
  if (!x) return false;
  Py_DECREF(x);
  if (x != dtype) return false;
  x = PyObject_GetAttr(t, s_shape);
  if (!x) return false;
  bool ok = PyTuple_Check(x) && PyTuple_GET_SIZE(x) == ndim && longs(x, ndim, v->size);
  Py_DECREF(x);
  if (!ok) return false;
  x = PyObject_CallMethodNoArgs(t, s_stride);
  if (!x) return false;
  ok = PyTuple_Check(x) && PyTuple_GET_SIZE(x) == ndim && longs(x, ndim, v->stride);
  Py_DECREF(x);
  if (!ok) return false;
  x = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!x) return false;
  v->ptr = PyLong_AsVoidPtr(x);
  Py_DECREF(x);
  v->ndim = ndim;
  return !PyErr_Occurred();
}

bool heads(PyObject* t, PyObject* dtype, View* v, aatc_heads_t* h) {
  if (!view_of(t, dtype, 3, v) || v->size[2] != AATC_HEAD_DIM || v->stride[2] != 1) return false;
  h->x = v->ptr;
  h->token_stride = v->size[0] > 1 ? v->stride[0] : 0;        // (a stride of one row or head means nothing)
  h->head_stride = v->size[1] > 1 ? v->stride[1] : 0;
  return true;
}

// A contiguous vector or array of the given sizes; `out` stays null for None.
bool flat(PyObject* t, PyObject* dtype, int ndim, int64_t n0, int64_t n1, int64_t n2, void** out) {
  *out = nullptr;
  if (t == Py_None) return true;
  View v;
  const int64_t n[3] = {n0, n1, n2};
  if (!view_of(t, dtype, ndim, &v) || !v.contiguous()) return false;
  for (int i = 0; i < ndim; ++i)
    if (v.size[i] != n[i]) return false;
  *out = v.ptr;
  return true;
}

struct Table {
  const int32_t* ids;
  int32_t rows, stride, pages;
};
bool table_of(PyObject* t, Table* out) {
  View v;
  if (!view_of(t, g_int32, 2, &v) || v.size[0] > INT32_MAX || v.size[1] > INT32_MAX || v.stride[0] > INT32_MAX ||
      (v.size[1] > 1 && v.stride[1] != 1))
    return false;
  out->ids = static_cast<const int32_t*>(v.ptr);
  out->rows = static_cast<int32_t>(v.size[0]);
  out->pages = static_cast<int32_t>(v.size[1]);
  out->stride = static_cast<int32_t>(v.size[0] > 1 ? v.stride[0] : v.size[1]);
  return true;
}

bool address(PyObject* x, void** out) {
  *out = x == Py_None ? nullptr : PyLong_AsVoidPtr(x);
  return !PyErr_Occurred();
}
bool int32_of(PyObject* x, int32_t* out) {
  const long v = PyLong_AsLong(x);
  if ((v == -1 && PyErr_Occurred()) || v < INT32_MIN || v > INT32_MAX) return false;
  *out = static_cast<int32_t>(v);
  return true;
}
bool float_of(PyObject* x, float* out) {
  const double v = PyFloat_AsDouble(x);
  *out = static_cast<float>(v);
  return !(v == -1.0 && PyErr_Occurred());
}

// The handle of a torch.cuda.Stream (its cuda_stream, given as an int), or of the current stream for None.
bool stream_of(PyObject* x, void** out) {
  if (x != Py_None) return address(x, out);
  PyObject* dev = PyObject_CallNoArgs(g_device);
  if (!dev) return false;
  PyObject* s = PyObject_CallOneArg(g_raw_stream, dev);
  Py_DECREF(dev);
  if (!s) return false;
  *out = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !PyErr_Occurred();
}

PyObject* not_taken() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// The status of a call, made without holding up Python's other threads.
template <typename F>
PyObject* answer(F call) {
  aatc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// rotate(rope address, x, positions, out, backward, stream)
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *rope, *positions, *stream;
  View x, o;
  aatc_heads_t xh, oh;
  if (n != 6 || !address(a[0], &rope)) return not_taken();
  PyObject* dtype = PyObject_GetAttr(a[1], s_dtype);
  if (!dtype) return not_taken();
  Py_DECREF(dtype);                                           // (torch keeps its dtypes)
  if ((dtype != g_bf16 && dtype != g_f16) || !heads(a[1], dtype, &x, &xh) || x.size[0] > INT32_MAX ||
      x.size[1] > INT32_MAX || !flat(a[2], g_int32, 1, x.size[0], 0, 0, &positions) || !positions ||
      !heads(a[3], dtype, &o, &oh) || o.size[0] != x.size[0] || o.size[1] != x.size[1] || !stream_of(a[5], &stream))
    return not_taken();
  const int32_t code = dtype == g_bf16 ? AATC_BF16 : AATC_F16, backward = PyObject_IsTrue(a[4]);
  if (backward < 0) return not_taken();
  return answer([&] { return aatc_rotate(static_cast<const aatc_rotary_t*>(rope), code, xh.x, xh.token_stride, xh.head_stride,
                                     static_cast<const int32_t*>(positions), static_cast<int32_t>(x.size[0]),
                                     static_cast<int32_t>(x.size[1]), backward, const_cast<void*>(oh.x), oh.token_stride,
                                     oh.head_stride, stream); });
}

// append(descriptor, layer address, flags address, dtype, n_kv_heads, k, v, table, index, rows, positions, rope address, q,
// q_out, stream)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *desc, *base, *flags, *index, *rows, *positions, *rope, *out = nullptr, *stream;
  int32_t n_kv, n_q = 0;
  View k, v, q;
  aatc_heads_t kh, vh, qh;
  Table t;
  if (n != 15 || !address(a[0], &desc) || !address(a[1], &base) || !address(a[2], &flags) || !int32_of(a[4], &n_kv) ||
      !heads(a[5], a[3], &k, &kh) || k.size[1] != n_kv || k.size[0] > INT32_MAX || !heads(a[6], a[3], &v, &vh) ||
      v.size[0] != k.size[0] || v.size[1] != n_kv || !table_of(a[7], &t) ||
      !flat(a[8], g_int32, 1, k.size[0], 0, 0, &index) || !index || !flat(a[9], g_int32, 1, k.size[0], 0, 0, &rows) ||
      (!rows && k.size[0] > t.rows) || !flat(a[10], g_int32, 1, k.size[0], 0, 0, &positions) || !address(a[11], &rope) ||
      (a[12] == Py_None) != (a[13] == Py_None) || !stream_of(a[14], &stream))
    return not_taken();
  if (a[12] != Py_None) {
    if (!rope || !heads(a[12], a[3], &q, &qh) || q.size[0] != k.size[0] || q.size[1] > INT32_MAX) return not_taken();
    if (a[13] == a[12]) out = q.ptr;
    else if (!flat(a[13], a[3], 3, q.size[0], q.size[1], AATC_HEAD_DIM, &out)) return not_taken();
    n_q = static_cast<int32_t>(q.size[1]);
  }
  return answer([&] { return aatc_paged_append(
      static_cast<const aatc_pages_t*>(desc), base, t.ids, t.rows, t.stride, t.pages, static_cast<const int32_t*>(rows),
      static_cast<const int32_t*>(index), static_cast<const int32_t*>(positions), static_cast<int32_t>(k.size[0]), &kh, &vh,
      static_cast<const aatc_rotary_t*>(rope), out ? &qh : nullptr, n_q, out, static_cast<int32_t*>(flags), stream); });
}

// decode(descriptor, layer address, flags address, dtype, q, table, lens, out, lse, prior out, prior lse, scale, cap, window,
// slopes, workspace, stream)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *desc, *base, *flags, *lens, *out, *lse, *prior_out, *prior_lse, *slopes, *stream;
  View q, ws;
  aatc_heads_t qh;
  Table t;
  aatc_paged_decode_t how;
  if (n != 17 || !address(a[0], &desc) || !address(a[1], &base) || !address(a[2], &flags) || !heads(a[4], a[3], &q, &qh) ||
      q.size[0] < 1 || q.size[0] > INT32_MAX || q.size[1] > INT32_MAX || !table_of(a[5], &t) || t.rows != q.size[0] ||
      !flat(a[6], g_int32, 1, q.size[0], 0, 0, &lens) || !lens ||
      !flat(a[7], g_float32, 3, q.size[0], q.size[1], AATC_HEAD_DIM, &out) || !out ||
      !flat(a[8], g_float32, 2, q.size[0], q.size[1], 0, &lse) ||
      !flat(a[9], g_float32, 3, q.size[0], q.size[1], AATC_HEAD_DIM, &prior_out) ||
      !flat(a[10], g_float32, 2, q.size[0], q.size[1], 0, &prior_lse) || !prior_out != !prior_lse ||
      !float_of(a[11], &how.scale) || !float_of(a[12], &how.cap) || !int32_of(a[13], &how.window) ||
      !flat(a[14], g_float32, 1, q.size[1], 0, 0, &slopes) || !view_of(a[15], g_float32, 1, &ws) || !ws.contiguous() ||
      !stream_of(a[16], &stream))
    return not_taken();
  how.slopes = static_cast<const float*>(slopes);
  how.prior_out = static_cast<const float*>(prior_out);
  how.prior_lse = static_cast<const float*>(prior_lse);
  return answer([&] { return aatc_paged_decode_attention(
      static_cast<const aatc_pages_t*>(desc), base, t.ids, t.stride, t.pages, static_cast<const int32_t*>(lens), t.rows, &qh,
      static_cast<int32_t>(q.size[1]), &how, static_cast<float*>(out), static_cast<float*>(lse), ws.ptr,
      static_cast<size_t>(ws.size[0]) * sizeof(float), static_cast<int32_t*>(flags), stream); });
}

// gather(descriptor, layer address, flags address, dtype, n_kv_heads, table, first, n_tokens, lens, k, v, stream)
PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *desc, *base, *flags, *lens, *stream;
  int32_t n_kv, first, tokens;
  View k, v;
  Table t;
  if (n != 12 || !address(a[0], &desc) || !address(a[1], &base) || !address(a[2], &flags) || !int32_of(a[4], &n_kv) ||
      !table_of(a[5], &t) || !int32_of(a[6], &first) || !int32_of(a[7], &tokens) ||
      !flat(a[8], g_int32, 1, t.rows, 0, 0, &lens) || !view_of(a[9], a[3], 4, &k) || !view_of(a[10], a[3], 4, &v) ||
      !stream_of(a[11], &stream))
    return not_taken();
  const int64_t want[4] = {t.rows, tokens, n_kv, AATC_HEAD_DIM};
  for (int i = 0; i < 4; ++i)
    if (k.size[i] != want[i] || v.size[i] != want[i]) return not_taken();
  if (!k.contiguous() || !v.contiguous()) return not_taken();
  return answer([&] { return aatc_paged_gather(static_cast<const aatc_pages_t*>(desc), base, t.ids, t.rows, t.stride, t.pages, first,
                                           tokens, static_cast<const int32_t*>(lens), k.ptr, v.ptr,
                                           static_cast<int32_t*>(flags), stream); });
}

// copy(descriptor, first layer's address, n_layers, bytes of a layer, pairs, stream); pairs: a C-contiguous int32 buffer [n][2]
PyObject* copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *desc, *base, *stream;
  int32_t layers;
  if (n != 6 || !address(a[0], &desc) || !address(a[1], &base) || !int32_of(a[2], &layers) || !stream_of(a[5], &stream))
    return not_taken();
  const size_t layer_bytes = PyLong_AsSize_t(a[3]);
  Py_buffer pairs;
  if (PyErr_Occurred() || PyObject_GetBuffer(a[4], &pairs, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) < 0) return not_taken();
  PyObject* got = nullptr;
  if (pairs.ndim == 2 && pairs.shape[1] == 2 && pairs.itemsize == 4 && pairs.shape[0] <= INT32_MAX && pairs.format &&
      pairs.format[0] == 'i' && !pairs.format[1])
    got = answer([&] { return aatc_pages_copy(static_cast<const aatc_pages_t*>(desc), base, layers, layer_bytes,
                                              static_cast<const int32_t*>(pairs.buf), static_cast<int32_t>(pairs.shape[0]),
                                              stream); });
  PyBuffer_Release(&pairs);
  return got ? got : not_taken();
}

// setup(torch.int32, torch.float32, torch.bfloat16, torch.float16, current raw stream of a device, current device)
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "setup takes six objects");
    return nullptr;
  }
  PyObject** to[6] = {&g_int32, &g_float32, &g_bf16, &g_f16, &g_raw_stream, &g_device};
  for (int i = 0; i < 6; ++i) Py_XSETREF(*to[i], Py_NewRef(a[i]));
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"rotate", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rotate)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(append)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(decode)), METH_FASTCALL, nullptr},
    {"gather", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gather)), METH_FASTCALL, nullptr},
    {"copy", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(copy)), METH_FASTCALL, nullptr},
    {"setup", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(setup)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  if (!s_is_cuda || !s_dtype || !s_shape || !s_stride || !s_data_ptr) return nullptr;
  return PyModule_Create(&module);
}
