// Native half of binding.py: argument marshalling between Python objects and the C ABI (adaption.h), and
// nothing else.  A layer call through ctypes cost 8 to 12 us of interpreter time in front of a launch, more
// than the small layers take on the GPU; here it costs about 1 us.
//
// The library itself is opened by path (bind), so that this module holds no link dependency on it.
// Tensors are read through their own attributes at every call (data_ptr() of the planes, formats,
// pitch): nothing about an argument is kept from one call to the next.  The interpreter lock is released
// around every call into the library.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <dlfcn.h>

#include <cstring>

#include "adaption.h"

namespace {

// the library's entry points
#define ADAPTION_FUNCTIONS(X)                                                                                        \
  X(adaption_measure_range) X(adaption_quantize) X(adaption_quantize_batch) X(adaption_quantize_batch_stochastic)    \
  X(adaption_quantize_stochastic) X(adaption_lp_act) X(adaption_lp_act_stochastic) X(adaption_bit_histogram)         \
  X(adaption_width_histogram) X(adaption_lp_conv_workspace_bytes) X(adaption_lp_conv_fwd)                            \
  X(adaption_lp_conv_fwd_stochastic) X(adaption_lp_conv_pool_workspace_bytes) X(adaption_lp_conv_pool_fwd)           \
  X(adaption_lp_ip_workspace_bytes) X(adaption_lp_ip_fwd) X(adaption_lp_ip_fwd_stochastic)                           \
  X(adaption_lp_ip_fwd_static_ws) X(adaption_maxpool2x2)                                                             \
  X(adaption_fp4_scale_bytes) X(adaption_fp4_quantize) X(adaption_fp4_dequantize) X(adaption_fp4_ip_fwd) X(adaption_fp4_act_ip_fwd)
#define DECLARE(f) decltype(&::f) p_##f = nullptr;
ADAPTION_FUNCTIONS(DECLARE)
#undef DECLARE

PyObject* g_error = nullptr;        // AdaptionError
PyObject* g_device = nullptr;       // () -> current device ordinal
PyObject* g_stream = nullptr;       // (device) -> raw handle of the current stream
PyObject* g_tensor = nullptr;        // the tensor class
PyObject* g_dtypes[3] = {};         // the tensor types ADAPTION_F32, ADAPTION_F16, ADAPTION_BF16

// The part of DLPack's C exchange interface (version 1.3) that describes a Python tensor in one call, without Python objects in
// between: 0.06 us where pointer, type, shape, strides and device through attributes take 0.37.
struct DlTensor {
  void* data;
  struct { int32_t type, id; } device;
  int32_t ndim;
  struct { uint8_t code, bits; uint16_t lanes; } dtype;
  int64_t *shape, *strides;
  uint64_t byte_offset;
};
struct DlExchange {
  struct { uint32_t major, minor; void* previous; } header;
  void *allocate, *from_object, *to_object;
  int (*view)(void* object, DlTensor* out);
};
const DlExchange* g_exchange = nullptr;   // null: tensors are read through their attributes
constexpr int32_t kDlCuda = 2;

PyObject *s_lo, *s_hi, *s_q16, *s_n_bits, *s_frac_bits, *s_c_stride, *s_outer, *s_inner, *s_data_ptr, *s_numel, *s_itemsize,
    *s_codes, *s_scales, *s_block, *s_exp, *s_dtype, *s_shape, *s_stride, *s_get_device;

bool attr_i64(PyObject* o, PyObject* name, long long* out) {
  PyObject* v = PyObject_GetAttr(o, name);
  if (v == nullptr) return false;
  *out = PyLong_AsLongLong(v);
  Py_DECREF(v);
  return !(*out == -1 && PyErr_Occurred());
}
// tensor (or None) -> device pointer
bool tensor_ptr(PyObject* t, void** out) {
  *out = nullptr;
  if (t == Py_None) return true;
  PyObject* v = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (v == nullptr) return false;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !(*out == nullptr && PyErr_Occurred());
}
bool attr_ptr(PyObject* o, PyObject* name, void** out) {
  PyObject* t = PyObject_GetAttr(o, name);
  if (t == nullptr) return false;
  const bool ok = tensor_ptr(t, out);
  Py_DECREF(t);
  return ok;
}
// QTensor -> descriptor
bool qtensor(PyObject* o, adaption_qtensor* q) {
  long long n, f, cs;
  void* q16;
  if (!attr_ptr(o, s_hi, &q->hi) || !attr_ptr(o, s_lo, &q->lo) || !attr_ptr(o, s_q16, &q16) || !attr_i64(o, s_n_bits, &n) ||
      !attr_i64(o, s_frac_bits, &f) || !attr_i64(o, s_c_stride, &cs))
    return false;
  q->q16 = static_cast<int16_t*>(q16);
  q->fmt.n_bits = (int32_t)n;
  q->fmt.frac_bits = (int32_t)f;
  q->c_stride = cs;
  return true;
}
bool i64(PyObject* o, long long* out) {
  *out = PyLong_AsLongLong(o);
  return !(*out == -1 && PyErr_Occurred());
}
bool i32(PyObject* o, int32_t* out) {
  long long v;
  if (!i64(o, &v)) return false;
  *out = (int32_t)v;
  return true;
}
bool truth(PyObject* o, int32_t* out) {
  const int t = PyObject_IsTrue(o);
  *out = t;
  return t >= 0;
}
bool u64(PyObject* o, uint64_t* out) {         // modulo 2^64
  PyObject* i = PyNumber_Index(o);
  if (i == nullptr) return false;
  *out = PyLong_AsUnsignedLongLongMask(i);
  Py_DECREF(i);
  return !PyErr_Occurred();
}
bool current_stream(void** out) {
  PyObject* d = PyObject_CallNoArgs(g_device);
  if (d == nullptr) return false;
  PyObject* s = PyObject_CallOneArg(g_stream, d);
  Py_DECREF(d);
  if (s == nullptr) return false;
  *out = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !(*out == nullptr && PyErr_Occurred());
}
bool numel(PyObject* t, long long* out) {
  PyObject* n = PyObject_CallMethodNoArgs(t, s_numel);
  if (n == nullptr) return false;
  *out = PyLong_AsLongLong(n);
  Py_DECREF(n);
  return !(*out == -1 && PyErr_Occurred());
}
// bytes of a tensor (workspace), 0 for None
bool workspace(PyObject* t, void** p, size_t* bytes) {
  *bytes = 0;
  if (!tensor_ptr(t, p)) return false;
  if (t == Py_None) return true;
  long long n, item;
  if (!numel(t, &n) || !attr_i64(t, s_itemsize, &item)) return false;
  *bytes = (size_t)(n * item);
  return true;
}
// read-only view of a ctypes structure
struct Buffer {
  Py_buffer b;
  bool held = false;
  ~Buffer() {
    if (held) PyBuffer_Release(&b);
  }
  bool get(PyObject* o, size_t need, const char* what, int flags = PyBUF_SIMPLE) {
    if (PyObject_GetBuffer(o, &b, flags) != 0) return false;
    held = true;
    if ((size_t)b.len < need) {
      PyErr_Format(PyExc_TypeError, "%s: a structure of %zu bytes is expected", what, need);
      return false;
    }
    return true;
  }
};

PyObject* answer(int rc, const char* where) {
  if (rc == ADAPTION_OK) Py_RETURN_NONE;
  PyObject* e = PyObject_CallFunction(g_error, "is", rc, where);
  if (e != nullptr) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return nullptr;
}

#define ARGS(n)                                                                        \
  if (nargs != (n)) {                                                                  \
    PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", (n), nargs);       \
    return nullptr;                                                                    \
  }
#define CALL(expr)            \
  int rc;                     \
  Py_BEGIN_ALLOW_THREADS rc = (expr); \
  Py_END_ALLOW_THREADS

// x, n_bits, d_max_abs, d_fmt_out
PyObject* measure_range(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(4)
  void *x, *mx, *fmt, *st;
  long long count;
  int32_t n;
  if (!tensor_ptr(a[0], &x) || !numel(a[0], &count) || !i32(a[1], &n) || !tensor_ptr(a[2], &mx) || !tensor_ptr(a[3], &fmt) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_measure_range((const float*)x, (size_t)count, n, (float*)mx, (adaption_qfmt*)fmt, st))
  return answer(rc, "adaption_measure_range");
}

// x, outer, inner, out, d_fmt, rounding, d_stats
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(7)
  void *x, *fmt, *stats, *st;
  long long outer, inner;
  int32_t rounding;
  adaption_qtensor q;
  if (!tensor_ptr(a[0], &x) || !i64(a[1], &outer) || !i64(a[2], &inner) || !qtensor(a[3], &q) || !tensor_ptr(a[4], &fmt) ||
      !i32(a[5], &rounding) || !tensor_ptr(a[6], &stats) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_quantize((const float*)x, (size_t)outer, (size_t)inner, q, (const adaption_qfmt*)fmt, rounding,
                           (adaption_stats*)stats, st))
  return answer(rc, "adaption_quantize");
}

// items (ctypes array, filled here), entries: (x, outer, inner, out, d_fmt or None) each
PyObject* fill_items(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(2)
  PyObject* seq = PySequence_Fast(a[1], "a sequence of entries is expected");
  if (seq == nullptr) return nullptr;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  Buffer b;
  bool ok = b.get(a[0], (size_t)n * sizeof(adaption_quantize_item), "items", PyBUF_WRITABLE);
  for (Py_ssize_t k = 0; ok && k < n; ++k) {
    adaption_quantize_item& it = static_cast<adaption_quantize_item*>(b.b.buf)[k];
    PyObject* e = PySequence_Fast(PySequence_Fast_GET_ITEM(seq, k), "an entry is a sequence");
    if (e == nullptr) { ok = false; break; }
    if (PySequence_Fast_GET_SIZE(e) != 5) {
      PyErr_SetString(PyExc_ValueError, "an entry is (x, outer, inner, out, d_fmt)");
      ok = false;
    } else {
      PyObject** v = PySequence_Fast_ITEMS(e);
      void *x, *fmt;
      long long outer, inner;
      ok = tensor_ptr(v[0], &x) && i64(v[1], &outer) && i64(v[2], &inner) && qtensor(v[3], &it.q) && tensor_ptr(v[4], &fmt);
      if (ok) {
        it.d_x = (const float*)x;
        it.outer = outer;
        it.inner = inner;
        it.d_fmt = (const adaption_qfmt*)fmt;
      }
    }
    Py_DECREF(e);
  }
  Py_DECREF(seq);
  if (!ok) return nullptr;
  Py_RETURN_NONE;
}

// items (None: a null pointer, which the library takes with n = 0 and refuses otherwise), n
PyObject* quantize_batch(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(2)
  int32_t n;
  void* st;
  Buffer b;
  if (!i32(a[1], &n) ||
      (a[0] != Py_None && !b.get(a[0], n > 0 ? (size_t)n * sizeof(adaption_quantize_item) : 0, "items")) ||
      !current_stream(&st))
    return nullptr;
  CALL(p_adaption_quantize_batch(b.held ? (const adaption_quantize_item*)b.b.buf : nullptr, n, st))
  return answer(rc, "adaption_quantize_batch");
}

// items, seeds (ctypes array of uint64), n
PyObject* quantize_batch_stochastic(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(3)
  int32_t n;
  void* st;
  Buffer b, s;
  if (!i32(a[2], &n) || !b.get(a[0], (size_t)n * sizeof(adaption_quantize_item), "items") ||
      !s.get(a[1], (size_t)n * sizeof(uint64_t), "seeds") || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_quantize_batch_stochastic((const adaption_quantize_item*)b.b.buf, (const uint64_t*)s.b.buf, n, st))
  return answer(rc, "adaption_quantize_batch_stochastic");
}

// x, outer, inner, out, seed, relu, d_fmt, d_stats
PyObject* quantize_stochastic(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(8)
  void *x, *fmt, *stats, *st;
  long long outer, inner;
  int32_t relu;
  uint64_t seed;
  adaption_qtensor q;
  if (!tensor_ptr(a[0], &x) || !i64(a[1], &outer) || !i64(a[2], &inner) || !qtensor(a[3], &q) || !u64(a[4], &seed) ||
      !truth(a[5], &relu) || !tensor_ptr(a[6], &fmt) || !tensor_ptr(a[7], &stats) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_quantize_stochastic((const float*)x, (size_t)outer, (size_t)inner, q, (const adaption_qfmt*)fmt, relu, seed,
                                      (adaption_stats*)stats, st))
  return answer(rc, "adaption_quantize_stochastic");
}

// x_f32, x_q, outer, inner, relu, out, d_fmt, rounding, d_stats
PyObject* lp_act(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(9)
  void *x, *fmt, *stats, *st;
  long long outer, inner;
  int32_t relu, rounding;
  adaption_qtensor xq, q;
  if (!tensor_ptr(a[0], &x) || (a[1] != Py_None && !qtensor(a[1], &xq)) || !i64(a[2], &outer) || !i64(a[3], &inner) ||
      !truth(a[4], &relu) || !qtensor(a[5], &q) || !tensor_ptr(a[6], &fmt) || !i32(a[7], &rounding) ||
      !tensor_ptr(a[8], &stats) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_lp_act((const float*)x, a[1] == Py_None ? nullptr : &xq, (size_t)outer, (size_t)inner, relu, q,
                         (const adaption_qfmt*)fmt, rounding, (adaption_stats*)stats, st))
  return answer(rc, "adaption_lp_act");
}

// x_f32, x_q, outer, inner, relu, out, seed, d_fmt, d_stats
PyObject* lp_act_stochastic(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(9)
  void *x, *fmt, *stats, *st;
  long long outer, inner;
  int32_t relu;
  uint64_t seed;
  adaption_qtensor xq, q;
  if (!tensor_ptr(a[0], &x) || (a[1] != Py_None && !qtensor(a[1], &xq)) || !i64(a[2], &outer) || !i64(a[3], &inner) ||
      !truth(a[4], &relu) || !qtensor(a[5], &q) || !u64(a[6], &seed) || !tensor_ptr(a[7], &fmt) || !tensor_ptr(a[8], &stats) ||
      !current_stream(&st))
    return nullptr;
  CALL(p_adaption_lp_act_stochastic((const float*)x, a[1] == Py_None ? nullptr : &xq, (size_t)outer, (size_t)inner, relu, q,
                                    (const adaption_qfmt*)fmt, seed, (adaption_stats*)stats, st))
  return answer(rc, "adaption_lp_act_stochastic");
}

// x, d_hist
PyObject* bit_histogram(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(2)
  void *x, *h, *st;
  long long count;
  if (!tensor_ptr(a[0], &x) || !numel(a[0], &count) || !tensor_ptr(a[1], &h) || !current_stream(&st)) return nullptr;
  CALL(p_adaption_bit_histogram((const float*)x, (size_t)count, (uint64_t*)h, st))
  return answer(rc, "adaption_bit_histogram");
}

// x (QTensor), d_hist
PyObject* width_histogram(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(2)
  adaption_qtensor q;
  long long outer, inner;
  void *h, *st;
  if (!qtensor(a[0], &q) || !attr_i64(a[0], s_outer, &outer) || !attr_i64(a[0], s_inner, &inner) || !tensor_ptr(a[1], &h) ||
      !current_stream(&st))
    return nullptr;
  CALL(p_adaption_width_histogram(q, (size_t)outer, (size_t)inner, (uint64_t*)h, st))
  return answer(rc, "adaption_width_histogram");
}

// shape, x (QTensor), w (QTensor), algo
PyObject* conv_workspace(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(4)
  Buffer shape;
  long long xn, xf, wn, wf, cs;
  int32_t algo;
  if (!shape.get(a[0], sizeof(adaption_conv_shape), "shape") || !attr_i64(a[1], s_n_bits, &xn) ||
      !attr_i64(a[1], s_frac_bits, &xf) || !attr_i64(a[1], s_c_stride, &cs) || !attr_i64(a[2], s_n_bits, &wn) ||
      !attr_i64(a[2], s_frac_bits, &wf) || !i32(a[3], &algo))
    return nullptr;
  const adaption_qfmt fx{(int32_t)xn, (int32_t)xf}, fw{(int32_t)wn, (int32_t)wf};
  return PyLong_FromSize_t(p_adaption_lp_conv_workspace_bytes((const adaption_conv_shape*)shape.b.buf, fx, fw, cs, algo));
}

// shape, x, w, y (QTensors), algo
PyObject* conv_pool_workspace(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(5)
  Buffer shape;
  long long xn, xf, wn, wf, yn, yf, cs, ycs;
  int32_t algo;
  if (!shape.get(a[0], sizeof(adaption_conv_shape), "shape") || !attr_i64(a[1], s_n_bits, &xn) ||
      !attr_i64(a[1], s_frac_bits, &xf) || !attr_i64(a[1], s_c_stride, &cs) || !attr_i64(a[2], s_n_bits, &wn) ||
      !attr_i64(a[2], s_frac_bits, &wf) || !attr_i64(a[3], s_n_bits, &yn) || !attr_i64(a[3], s_frac_bits, &yf) ||
      !attr_i64(a[3], s_c_stride, &ycs) || !i32(a[4], &algo))
    return nullptr;
  const adaption_qfmt fx{(int32_t)xn, (int32_t)xf}, fw{(int32_t)wn, (int32_t)wf}, fy{(int32_t)yn, (int32_t)yf};
  return PyLong_FromSize_t(
      p_adaption_lp_conv_pool_workspace_bytes((const adaption_conv_shape*)shape.b.buf, fx, fw, fy, cs, ycs, algo));
}

// B, K, O, x, w (QTensors), algo
PyObject* ip_workspace(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(6)
  long long B, K, O, xn, xf, wn, wf;
  int32_t algo;
  if (!i64(a[0], &B) || !i64(a[1], &K) || !i64(a[2], &O) || !attr_i64(a[3], s_n_bits, &xn) || !attr_i64(a[3], s_frac_bits, &xf) ||
      !attr_i64(a[4], s_n_bits, &wn) || !attr_i64(a[4], s_frac_bits, &wf) || !i32(a[5], &algo))
    return nullptr;
  const adaption_qfmt fx{(int32_t)xn, (int32_t)xf}, fw{(int32_t)wn, (int32_t)wf};
  return PyLong_FromSize_t(p_adaption_lp_ip_workspace_bytes(B, K, O, fx, fw, algo));
}

// shape, x, w, bias_q, bias_frac_bits, relu, mode, algo, y or None, d_stats, workspace
PyObject* conv_fwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(11)
  Buffer shape;
  adaption_qtensor x, w, y{};
  void *bias, *stats, *ws, *st;
  size_t wsb;
  int32_t bf, relu, mode, algo;
  if (!shape.get(a[0], sizeof(adaption_conv_shape), "shape") || !qtensor(a[1], &x) || !qtensor(a[2], &w) ||
      !tensor_ptr(a[3], &bias) || !i32(a[4], &bf) || !truth(a[5], &relu) || !i32(a[6], &mode) || !i32(a[7], &algo) ||
      (a[8] != Py_None && !qtensor(a[8], &y)) || !tensor_ptr(a[9], &stats) || !workspace(a[10], &ws, &wsb) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_lp_conv_fwd((const adaption_conv_shape*)shape.b.buf, x, w, (const int16_t*)bias, bf, relu, mode, algo, y,
                              (adaption_stats*)stats, ws, wsb, st))
  return answer(rc, "adaption_lp_conv_fwd");
}

// shape, x, w, bias_q, bias_frac_bits, relu, algo, y, seed, d_stats, workspace
PyObject* conv_fwd_stochastic(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(11)
  Buffer shape;
  adaption_qtensor x, w, y;
  void *bias, *stats, *ws, *st;
  size_t wsb;
  int32_t bf, relu, algo;
  uint64_t seed;
  if (!shape.get(a[0], sizeof(adaption_conv_shape), "shape") || !qtensor(a[1], &x) || !qtensor(a[2], &w) ||
      !tensor_ptr(a[3], &bias) || !i32(a[4], &bf) || !truth(a[5], &relu) || !i32(a[6], &algo) || !qtensor(a[7], &y) ||
      !u64(a[8], &seed) || !tensor_ptr(a[9], &stats) || !workspace(a[10], &ws, &wsb) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_lp_conv_fwd_stochastic((const adaption_conv_shape*)shape.b.buf, x, w, (const int16_t*)bias, bf, relu, algo, y,
                                         seed, (adaption_stats*)stats, ws, wsb, st))
  return answer(rc, "adaption_lp_conv_fwd_stochastic");
}

// shape, x, w, bias_q, bias_frac_bits, relu, algo, y, d_stats, workspace, phases
PyObject* conv_pool_fwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(11)
  Buffer shape;
  adaption_qtensor x, w, y;
  void *bias, *stats, *ws, *st;
  size_t wsb;
  int32_t bf, relu, algo, phases;
  if (!shape.get(a[0], sizeof(adaption_conv_shape), "shape") || !qtensor(a[1], &x) || !qtensor(a[2], &w) ||
      !tensor_ptr(a[3], &bias) || !i32(a[4], &bf) || !truth(a[5], &relu) || !i32(a[6], &algo) || !qtensor(a[7], &y) ||
      !tensor_ptr(a[8], &stats) || !workspace(a[9], &ws, &wsb) || !i32(a[10], &phases) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_lp_conv_pool_fwd((const adaption_conv_shape*)shape.b.buf, x, w, (const int16_t*)bias, bf, relu, algo, phases,
                                   y, (adaption_stats*)stats, ws, wsb, st))
  return answer(rc, "adaption_lp_conv_pool_fwd");
}

// B, K, O, x, w, bias_q, bias_frac_bits, relu, mode, algo, y or None, d_stats, workspace
PyObject* ip_fwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(13)
  adaption_qtensor x, w, y{};
  void *bias, *stats, *ws, *st;
  size_t wsb;
  long long B, K, O;
  int32_t bf, relu, mode, algo;
  if (!i64(a[0], &B) || !i64(a[1], &K) || !i64(a[2], &O) || !qtensor(a[3], &x) || !qtensor(a[4], &w) || !tensor_ptr(a[5], &bias) ||
      !i32(a[6], &bf) || !truth(a[7], &relu) || !i32(a[8], &mode) || !i32(a[9], &algo) || (a[10] != Py_None && !qtensor(a[10], &y)) ||
      !tensor_ptr(a[11], &stats) || !workspace(a[12], &ws, &wsb) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_lp_ip_fwd(B, K, O, x, w, (const int16_t*)bias, bf, relu, mode, algo, y, (adaption_stats*)stats, ws, wsb, st))
  return answer(rc, "adaption_lp_ip_fwd");
}

// B, K, O, x, w, bias_q, bias_frac_bits, relu, algo, y, seed, d_stats, workspace
PyObject* ip_fwd_stochastic(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(13)
  adaption_qtensor x, w, y;
  void *bias, *stats, *ws, *st;
  size_t wsb;
  long long B, K, O;
  int32_t bf, relu, algo;
  uint64_t seed;
  if (!i64(a[0], &B) || !i64(a[1], &K) || !i64(a[2], &O) || !qtensor(a[3], &x) || !qtensor(a[4], &w) || !tensor_ptr(a[5], &bias) ||
      !i32(a[6], &bf) || !truth(a[7], &relu) || !i32(a[8], &algo) || !qtensor(a[9], &y) || !u64(a[10], &seed) ||
      !tensor_ptr(a[11], &stats) || !workspace(a[12], &ws, &wsb) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_lp_ip_fwd_stochastic(B, K, O, x, w, (const int16_t*)bias, bf, relu, algo, y, seed, (adaption_stats*)stats, ws,
                                       wsb, st))
  return answer(rc, "adaption_lp_ip_fwd_stochastic");
}

// B, K, O, x, w, bias_q, bias_frac_bits, relu, mode, algo, y or None, d_stats
PyObject* ip_fwd_static_ws(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(12)
  adaption_qtensor x, w, y{};
  void *bias, *stats, *st;
  long long B, K, O;
  int32_t bf, relu, mode, algo;
  if (!i64(a[0], &B) || !i64(a[1], &K) || !i64(a[2], &O) || !qtensor(a[3], &x) || !qtensor(a[4], &w) || !tensor_ptr(a[5], &bias) ||
      !i32(a[6], &bf) || !truth(a[7], &relu) || !i32(a[8], &mode) || !i32(a[9], &algo) || (a[10] != Py_None && !qtensor(a[10], &y)) ||
      !tensor_ptr(a[11], &stats) || !current_stream(&st))
    return nullptr;
  CALL(p_adaption_lp_ip_fwd_static_ws(B, K, O, x, w, (const int16_t*)bias, bf, relu, mode, algo, y, (adaption_stats*)stats, st))
  return answer(rc, "adaption_lp_ip_fwd_static_ws");
}

// x, N, H, W, C, y
PyObject* maxpool(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(6)
  adaption_qtensor x, y;
  int32_t N, H, W, C;
  void* st;
  if (!qtensor(a[0], &x) || !i32(a[1], &N) || !i32(a[2], &H) || !i32(a[3], &W) || !i32(a[4], &C) || !qtensor(a[5], &y) ||
      !current_stream(&st))
    return nullptr;
  CALL(p_adaption_maxpool2x2(x, N, H, W, C, y, st))
  return answer(rc, "adaption_maxpool2x2");
}

// ---- microscaled 4-bit floating point.  These calls take tensors of several types and any pitch, so what the C ABI cannot see
// is checked here: type, shape, contiguous rows, and that the tensors lie on the current device.

PyObject* refuse(const char* where) { return answer(ADAPTION_ERR_INVALID_ARG, where); }

// the current device and its stream
bool device_stream(long long* device, void** out) {
  PyObject* d = PyObject_CallNoArgs(g_device);
  if (d == nullptr) return false;
  *device = PyLong_AsLongLong(d);
  PyObject* s = *device == -1 && PyErr_Occurred() ? nullptr : PyObject_CallOneArg(g_stream, d);
  Py_DECREF(d);
  if (s == nullptr) return false;
  *out = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !(*out == nullptr && PyErr_Occurred());
}
// What the calls below look at in a tensor.
struct View {
  void* data;
  long long device;                    // -1: not on a GPU
  int dtype;                           // ADAPTION_F32, _F16 or _BF16, or 3
  int ndim;                            // shape and strides of at most two dimensions
  long long shape[2], stride[2];
  long long bytes, item;               // of all elements, of one
  bool contiguous;
};
// Whether elements lie one after the other; called for every dimension, the last one first, with n = 1 at the start.
bool dense(long long size, long long stride, long long* n) {
  const bool ok = size == 1 || stride == *n;
  *n *= size;
  return ok;
}

bool view_by_attributes(PyObject* t, View* v) {
  PyObject* d = PyObject_CallMethodNoArgs(t, s_get_device);
  if (d == nullptr) return false;
  v->device = PyLong_AsLongLong(d);
  Py_DECREF(d);
  if (v->device == -1 && PyErr_Occurred()) return false;
  d = PyObject_GetAttr(t, s_dtype);
  if (d == nullptr) return false;
  Py_DECREF(d);                        // (types live as long as torch)
  for (v->dtype = 0; v->dtype < 3 && g_dtypes[v->dtype] != d; ++v->dtype) {
  }
  PyObject* shape = PyObject_GetAttr(t, s_shape);
  PyObject* stride = shape == nullptr ? nullptr : PyObject_CallMethodNoArgs(t, s_stride);
  bool ok = stride != nullptr && PyTuple_Check(shape) && PyTuple_Check(stride);
  if (ok) {
    v->ndim = (int)PyTuple_GET_SIZE(shape);
    v->contiguous = true;
    long long n = 1;
    for (int k = v->ndim - 1; ok && k >= 0; --k) {
      long long size, step;
      ok = i64(PyTuple_GET_ITEM(shape, k), &size) && i64(PyTuple_GET_ITEM(stride, k), &step);
      if (!ok) break;
      if (k < 2) {
        v->shape[k] = size;
        v->stride[k] = step;
      }
      v->contiguous = dense(size, step, &n) && v->contiguous;
    }
    v->contiguous = v->contiguous || n == 0;
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_TypeError, "a tensor is expected");
  }
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  long long n = 0;
  if (!ok || !numel(t, &n) || !attr_i64(t, s_itemsize, &v->item)) return false;
  v->bytes = n * v->item;
  return tensor_ptr(t, &v->data);
}
bool view_of(PyObject* t, View* v) {
  DlTensor d{};
  if (g_exchange == nullptr || g_exchange->view(t, &d) != 0) {
    PyErr_Clear();
    return view_by_attributes(t, v);
  }
  v->data = static_cast<char*>(d.data) + d.byte_offset;
  v->device = d.device.type == kDlCuda ? d.device.id : -1;
  const int type = d.dtype.lanes != 1 ? 0 : d.dtype.code * 256 + d.dtype.bits;
  v->dtype = type == 2 * 256 + 32 ? ADAPTION_F32 : type == 2 * 256 + 16 ? ADAPTION_F16 : type == 4 * 256 + 16 ? ADAPTION_BF16 : 3;
  v->ndim = d.ndim;
  v->contiguous = true;
  long long n = 1;
  for (int k = d.ndim - 1; k >= 0; --k) {
    const long long step = d.strides != nullptr ? d.strides[k] : n;
    if (k < 2) {
      v->shape[k] = d.shape[k];
      v->stride[k] = step;
    }
    v->contiguous = dense(d.shape[k], step, &n) && v->contiguous;
  }
  v->contiguous = v->contiguous || n == 0;
  v->item = (long long)d.dtype.bits * d.dtype.lanes / 8;
  v->bytes = n * v->item;
  return true;
}
// 2-D tensor of rows x cols -> descriptor: 1, 0 (refused) or -1 (exception)
int matrix(PyObject* t, long long rows, long long cols, long long device, adaption_matrix* m) {
  View v;
  if (!view_of(t, &v)) return -1;
  if (v.device != device || v.dtype == 3 || v.ndim != 2 || v.shape[0] != rows || v.shape[1] != cols) return 0;
  if (cols > 1 && v.stride[1] != 1) return 0;
  m->data = v.data;
  m->dtype = v.dtype;
  m->reserved = 0;
  // (the pitch of a single row means nothing)
  m->stride = rows > 1 ? v.stride[0] : (v.stride[0] > cols ? v.stride[0] : cols);
  return 1;
}
// a tensor's address (null for None) if it lies on the device and holds its elements one after the other; `bytes`: its size
int address(PyObject* t, long long device, void** out, size_t* bytes = nullptr) {
  *out = nullptr;
  if (bytes != nullptr) *bytes = 0;
  if (t == Py_None) return 1;
  View v;
  if (!view_of(t, &v)) return -1;
  if (v.device != device || !v.contiguous) return 0;
  *out = v.data;
  if (bytes != nullptr) *bytes = (size_t)v.bytes;
  return 1;
}
int attr_address(PyObject* o, PyObject* name, long long device, void** out, size_t* bytes = nullptr) {
  PyObject* t = PyObject_GetAttr(o, name);
  if (t == nullptr) return -1;
  const int r = address(t, device, out, bytes);
  Py_DECREF(t);
  return r;
}
// A byte plane of a fixed-point tensor (null for None): on the device and, where `need` bytes of it are read, holding them one after
// the other.
int plane_address(PyObject* o, PyObject* name, long long device, unsigned __int128 need, void** out) {
  *out = nullptr;
  PyObject* t = PyObject_GetAttr(o, name);
  if (t == nullptr) return -1;
  View v;
  const int r = t == Py_None ? 0 : (view_of(t, &v) ? 1 : -1);
  Py_DECREF(t);
  if (r <= 0) return r < 0 ? -1 : 1;
  if (v.device != device || (need > 0 && (v.item != 1 || !v.contiguous || (unsigned __int128)v.bytes < need))) return 0;
  *out = v.data;
  return 1;
}
// QTensor of at least rows x cols as a source
int fixed_source(PyObject* o, long long rows, long long cols, long long device, adaption_qtensor* q) {
  long long outer, inner, n, f, cs;
  if (!attr_i64(o, s_outer, &outer) || !attr_i64(o, s_inner, &inner) || !attr_i64(o, s_n_bits, &n) || !attr_i64(o, s_frac_bits, &f) ||
      !attr_i64(o, s_c_stride, &cs))
    return -1;
  if (outer < rows || inner < cols || cs < cols || n < 1 || n > 16 || f < 0 || f > 15) return 0;
  const unsigned __int128 need = (unsigned __int128)rows * (unsigned long long)cs;
  q->q16 = nullptr;
  q->fmt.n_bits = (int32_t)n;
  q->fmt.frac_bits = (int32_t)f;
  q->c_stride = cs;
  const int r = plane_address(o, s_lo, device, need, &q->lo);
  return r > 0 ? plane_address(o, s_hi, device, n > 8 ? need : 0, &q->hi) : r;
}
// adaption_stats, or None
int stats_address(PyObject* t, long long device, void** out) {
  size_t bytes;
  const int r = address(t, device, out, &bytes);
  return r > 0 && *out != nullptr && bytes < sizeof(adaption_stats) ? 0 : r;
}
// Fp4Tensor of at least rows x cols
int fp4tensor(PyObject* o, long long rows, long long cols, long long device, adaption_fp4tensor* f) {
  long long outer, inner, cs, block, exp;
  if (!attr_i64(o, s_outer, &outer) || !attr_i64(o, s_inner, &inner) || !attr_i64(o, s_c_stride, &cs) ||
      !attr_i64(o, s_block, &block) || !attr_i64(o, s_exp, &exp))
    return -1;
  // (the scale tiles follow from the row length, so a tensor is used at its own)
  if (outer < rows || inner != cols || cs < 0 || cs > (1ll << 40) || rows > (1ll << 40)) return 0;
  f->c_stride = cs;
  f->block = (int32_t)block;
  f->exp = exp < -1000 || exp > 1000 ? 1000 : (int32_t)exp;
  size_t codes = 0, scales = 0;
  int r = attr_address(o, s_codes, device, &f->codes, &codes);
  if (r > 0) r = attr_address(o, s_scales, device, &f->scales, &scales);
  if (r <= 0) return r;
  // (attributes can be given other tensors later)
  return (unsigned __int128)rows * (unsigned long long)(cs / 2) <= codes && p_adaption_fp4_scale_bytes(rows, cols, f->block) <= scales;
}
// fp32 vector of at least n elements, or None
int bias_vector(PyObject* t, long long n, long long device, void** out) {
  *out = nullptr;
  if (t == Py_None) return 1;
  View v;
  if (!view_of(t, &v)) return -1;
  if (v.device != device || v.dtype != ADAPTION_F32 || v.ndim != 1 || v.shape[0] < n || (n > 1 && v.stride[0] != 1)) return 0;
  *out = v.data;
  return 1;
}
#define TAKE(expr, where)                     \
  {                                           \
    const int taken = (expr);                 \
    if (taken < 0) return nullptr;            \
    if (taken == 0) return refuse(where);     \
  }

// x (tensor or QTensor), outer, inner, out, relu, d_stats
PyObject* fp4_quantize(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(6)
  const char* const where = "adaption_fp4_quantize";
  long long outer, inner, dev;
  int32_t relu;
  void *stats, *st;
  adaption_matrix x{};
  adaption_qtensor q{};
  adaption_fp4tensor out;
  if (!i64(a[1], &outer) || !i64(a[2], &inner) || !truth(a[4], &relu) || !device_stream(&dev, &st)) return nullptr;
  if (outer < 0 || inner < 0) return refuse(where);
  const bool fixed = !PyObject_TypeCheck(a[0], (PyTypeObject*)g_tensor) && PyObject_HasAttr(a[0], s_n_bits);
  if (fixed) {
    TAKE(fixed_source(a[0], outer, inner, dev, &q), where)
  } else {
    TAKE(matrix(a[0], outer, inner, dev, &x), where)
  }
  TAKE(fp4tensor(a[3], outer, inner, dev, &out), where)
  TAKE(stats_address(a[5], dev, &stats), where)
  CALL(p_adaption_fp4_quantize(x, fixed ? &q : nullptr, (size_t)outer, (size_t)inner, relu, out, (adaption_stats*)stats, st))
  return answer(rc, where);
}

// x, outer, inner, y
PyObject* fp4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(4)
  const char* const where = "adaption_fp4_dequantize";
  long long outer, inner, dev;
  void* st;
  adaption_fp4tensor x;
  adaption_matrix y;
  if (!i64(a[1], &outer) || !i64(a[2], &inner) || !device_stream(&dev, &st)) return nullptr;
  if (outer < 0 || inner < 0) return refuse(where);
  TAKE(fp4tensor(a[0], outer, inner, dev, &x), where)
  TAKE(matrix(a[3], outer, inner, dev, &y), where)
  CALL(p_adaption_fp4_dequantize(x, (size_t)outer, (size_t)inner, y, st))
  return answer(rc, where);
}

// B, K, O, x, w, bias, relu, y, d_stats
PyObject* fp4_ip_fwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(9)
  const char* const where = "adaption_fp4_ip_fwd";
  long long B, K, O, dev;
  int32_t relu;
  void *bias, *stats, *st;
  adaption_fp4tensor x, w;
  adaption_matrix y;
  if (!i64(a[0], &B) || !i64(a[1], &K) || !i64(a[2], &O) || !truth(a[6], &relu) || !device_stream(&dev, &st)) return nullptr;
  TAKE(fp4tensor(a[3], B, K, dev, &x), where)
  TAKE(fp4tensor(a[4], O, K, dev, &w), where)
  TAKE(bias_vector(a[5], O, dev, &bias), where)
  TAKE(matrix(a[7], B, O, dev, &y), where)
  TAKE(stats_address(a[8], dev, &stats), where)
  CALL(p_adaption_fp4_ip_fwd(B, K, O, x, w, (const float*)bias, relu, y, (adaption_stats*)stats, st))
  return answer(rc, where);
}

// B, K, O, x, x_exp, w, bias, relu, y, d_stats, workspace
PyObject* fp4_act_ip_fwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(11)
  const char* const where = "adaption_fp4_act_ip_fwd";
  long long B, K, O, dev, x_exp;
  int32_t relu;
  size_t wsb;
  void *bias, *stats, *ws, *st;
  adaption_fp4tensor w;
  adaption_matrix x, y;
  if (!i64(a[0], &B) || !i64(a[1], &K) || !i64(a[2], &O) || !i64(a[4], &x_exp) || !truth(a[7], &relu) ||
      !device_stream(&dev, &st))
    return nullptr;
  if (x_exp < -1000 || x_exp > 1000) return refuse(where);
  TAKE(matrix(a[3], B, K, dev, &x), where)
  TAKE(fp4tensor(a[5], O, K, dev, &w), where)
  TAKE(bias_vector(a[6], O, dev, &bias), where)
  TAKE(matrix(a[8], B, O, dev, &y), where)
  TAKE(stats_address(a[9], dev, &stats), where)
  TAKE(address(a[10], dev, &ws, &wsb), where)
  CALL(p_adaption_fp4_act_ip_fwd(B, K, O, x, (int32_t)x_exp, w, (const float*)bias, relu, y, (adaption_stats*)stats, ws, wsb, st))
  return answer(rc, where);
}

// Whether the exchange interface says of a tensor what its attributes say.
bool views_agree(PyObject* t) {
  View a, b;
  memset(&a, 0, sizeof(a));
  memset(&b, 0, sizeof(b));
  DlTensor d{};
  if (g_exchange->view(t, &d) != 0 || !view_of(t, &a) || !view_by_attributes(t, &b)) {
    PyErr_Clear();
    return false;
  }
  return a.data == b.data && a.device == b.device && a.dtype == b.dtype && a.ndim == b.ndim && a.bytes == b.bytes &&
         a.item == b.item && a.contiguous == b.contiguous && memcmp(a.shape, b.shape, sizeof(a.shape)) == 0 && memcmp(a.stride, b.stride, sizeof(a.stride)) == 0;
}

// library path, AdaptionError, current device, stream of device, the types of ADAPTION_F32, _F16 and _BF16, the tensor class, its
// DLPack exchange capsule or None, tensors to try that on
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(10)
  if (!PyType_Check(a[7]) || !PyTuple_Check(a[9])) {
    PyErr_SetString(PyExc_TypeError, "a class and a tuple are expected");
    return nullptr;
  }
  const char* path = PyUnicode_AsUTF8(a[0]);
  if (path == nullptr) return nullptr;
  void* lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
  if (lib == nullptr) {
    PyErr_Format(PyExc_RuntimeError, "%s cannot be opened: %s", path, dlerror());
    return nullptr;
  }
#define RESOLVE(f)                                                        \
  p_##f = reinterpret_cast<decltype(p_##f)>(dlsym(lib, #f));              \
  if (p_##f == nullptr) {                                                 \
    PyErr_SetString(PyExc_RuntimeError, "the library lacks " #f);         \
    return nullptr;                                                       \
  }
  ADAPTION_FUNCTIONS(RESOLVE)
#undef RESOLVE
  for (int k = 1; k < 7; ++k) Py_INCREF(a[k]);
  for (int k = 0; k < 3; ++k) Py_XSETREF(g_dtypes[k], a[4 + k]);
  Py_INCREF(a[7]);
  Py_XSETREF(g_tensor, a[7]);
  g_exchange = nullptr;
  if (PyCapsule_IsValid(a[8], "dlpack_exchange_api")) {
    const DlExchange* e = static_cast<const DlExchange*>(PyCapsule_GetPointer(a[8], "dlpack_exchange_api"));
    if (e->header.major == 1 && e->header.minor >= 3 && e->view != nullptr) {
      g_exchange = e;
      for (Py_ssize_t k = 0; g_exchange != nullptr && k < PyTuple_GET_SIZE(a[9]); ++k)
        if (!views_agree(PyTuple_GET_ITEM(a[9], k))) g_exchange = nullptr;
    }
  }
  Py_XSETREF(g_error, a[1]);
  Py_XSETREF(g_device, a[2]);
  Py_XSETREF(g_stream, a[3]);
  Py_RETURN_NONE;
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(measure_range), METHOD(quantize), METHOD(fill_items), METHOD(quantize_batch),
                         METHOD(quantize_batch_stochastic), METHOD(quantize_stochastic), METHOD(lp_act),
                         METHOD(lp_act_stochastic), METHOD(bit_histogram), METHOD(width_histogram), METHOD(conv_workspace),
                         METHOD(conv_pool_workspace), METHOD(ip_workspace), METHOD(conv_fwd), METHOD(conv_fwd_stochastic),
                         METHOD(conv_pool_fwd), METHOD(ip_fwd), METHOD(ip_fwd_stochastic), METHOD(ip_fwd_static_ws),
                         METHOD(maxpool), METHOD(fp4_quantize), METHOD(fp4_dequantize), METHOD(fp4_ip_fwd), METHOD(fp4_act_ip_fwd),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_adaption_native", "Argument marshalling of the C ABI.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__adaption_native() {
  struct { PyObject** o; const char* s; } names[] = {
      {&s_lo, "lo"}, {&s_hi, "hi"}, {&s_q16, "q16"}, {&s_n_bits, "n_bits"}, {&s_frac_bits, "frac_bits"},
      {&s_c_stride, "c_stride"}, {&s_outer, "outer"}, {&s_inner, "inner"}, {&s_data_ptr, "data_ptr"}, {&s_numel, "numel"},
      {&s_itemsize, "itemsize"}, {&s_codes, "codes"}, {&s_scales, "scales"}, {&s_block, "block"}, {&s_exp, "exp"},
      {&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_get_device, "get_device"}};
  for (auto& n : names) {
    *n.o = PyUnicode_InternFromString(n.s);
    if (*n.o == nullptr) return nullptr;
  }
  return PyModule_Create(&module);
}
