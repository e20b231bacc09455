// The layer calls of the Python binding without its interpreter time: arguments checked and taken
// from the tensors here, one native call.  A layer of a small batch is 3 us of GPU time; through
// ctypes its call took 5.6 us of host time, of which the launch itself is 2.3.
//
// Only marshalling, as in binding.py: device tensors, contiguous, of the stated type (None: a null
// pointer); tensors of exactly torch.Tensor's type are read directly, others through the binding's
// own _ptr.  The functions called are the ones that the binding loaded (their addresses are handed
// over by bind()), on the current device's current stream; the interpreter lock is released during
// the call, as ctypes does.  Each function returns the library's return code.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include "../../include/q8conv.h"

namespace {

PyObject *g_ptr, *g_device, *g_stream, *g_desc_type, *g_int8, *g_int32, *g_float32, *g_uint8;
enum {
  kInt8, kU8, kPerChannel, kReal, kF32, kMaxabs, kQuantize, kDequantize, kLayerFunctions,
  kRows = kLayerFunctions, kLinearInt8, kLinear, kPackedBytes, kPages, kKv4Write, kKv4Read, kKv4Attend,
  kKv8Write, kKv8Read, kKv8Attend, kPageSelect, kPageCompact, kPageCopy, kFunctions
};
void* g_fn[kFunctions];

// One call's arguments, read in order; `ok` turns false with a Python exception set.
struct Args {
  PyObject* const* a;
  bool ok = true;
  Py_buffer desc_buffer{};

  ~Args() {
    if (desc_buffer.obj) PyBuffer_Release(&desc_buffer);
  }
  const q8_conv_desc* desc(int i) {
    if (!ok) return nullptr;
    if (!PyObject_TypeCheck(a[i], (PyTypeObject*)g_desc_type)) {
      PyErr_SetString(PyExc_TypeError, "expected a ConvDesc");
      ok = false;
    } else if (PyObject_GetBuffer(a[i], &desc_buffer, PyBUF_SIMPLE) != 0) {
      ok = false;
    } else if (desc_buffer.len < (Py_ssize_t)sizeof(q8_conv_desc)) {
      PyErr_SetString(PyExc_TypeError, "ConvDesc is too small");
      ok = false;
    }
    return ok ? static_cast<const q8_conv_desc*>(desc_buffer.buf) : nullptr;
  }
  // Address of the tensor; elements: their number.
  // (type Undefined: any type)
  template <typename T>
  T* tensor(int i, at::ScalarType type, PyObject* dtype, long* elements = nullptr) {
    if (elements) *elements = 0;
    if (!ok || a[i] == Py_None) return nullptr;
    if (Py_TYPE(a[i]) == (PyTypeObject*)THPVariableClass) {
      const at::Tensor& t = THPVariable_Unpack(a[i]);
      try {
        if (t.is_cuda() && t.has_storage() && t.is_contiguous() &&
            (type == at::ScalarType::Undefined || t.scalar_type() == type)) {
          T* const p = static_cast<T*>(t.mutable_data_ptr());
          if (elements) *elements = t.numel();
          return p;
        }
      } catch (...) {        // (none may leave through the interpreter's frames)
      }
    }
    // The binding's own checks, and their exceptions: also for tensors of that type without storage,
    // as a function under vmap, grad or functionalize sees them.
    PyObject* address = PyObject_CallFunctionObjArgs(g_ptr, a[i], dtype, nullptr);
    void* p = address ? PyLong_AsVoidPtr(address) : nullptr;
    Py_XDECREF(address);
    if (elements && !PyErr_Occurred()) {
      PyObject* n = PyObject_CallMethod(a[i], "numel", nullptr);
      if (n) *elements = PyLong_AsLong(n);
      Py_XDECREF(n);
    }
    if (PyErr_Occurred()) ok = false;
    return ok ? static_cast<T*>(p) : nullptr;
  }
  // A tensor whose elements count: None has no number of them, and is none of length 0.
  template <typename T>
  T* counted(int i, at::ScalarType type, PyObject* dtype, long* elements) {
    if (ok && a[i] == Py_None) {
      Py_XDECREF(PyObject_GetAttrString(a[i], "numel"));       // the exception that this raises
      ok = false;
    }
    return tensor<T>(i, type, dtype, elements);
  }
  int8_t* i8(int i) { return tensor<int8_t>(i, at::kChar, g_int8); }
  int32_t* i32(int i) { return tensor<int32_t>(i, at::kInt, g_int32); }
  float* f32(int i) { return tensor<float>(i, at::kFloat, g_float32); }
  // The number inside an object of that ctypes type; null, with the exception as it is, for any other.
  static PyObject* boxed(PyObject* v, const char* type) {
    PyObject *kind, *error, *trace;
    PyErr_Fetch(&kind, &error, &trace);
    PyObject* ctypes = PyImport_ImportModule("ctypes");
    PyObject* t = ctypes ? PyObject_GetAttrString(ctypes, type) : nullptr;
    PyObject* n = t && PyObject_IsInstance(v, t) == 1 ? PyObject_GetAttrString(v, "value") : nullptr;
    Py_XDECREF(ctypes);
    Py_XDECREF(t);
    PyErr_Clear();
    if (!n) {
      PyErr_Restore(kind, error, trace);
      return nullptr;
    }
    Py_XDECREF(kind);
    Py_XDECREF(error);
    Py_XDECREF(trace);
    return n;
  }
  // As ctypes takes a c_float: whatever has __float__ or __index__, and its own objects.
  float factor(int i) {
    if (!ok) return 0.0f;
    double v = PyFloat_AsDouble(a[i]);
    if (v == -1.0 && PyErr_Occurred()) {
      PyObject* n = boxed(a[i], "c_float");
      if (n) v = PyFloat_AsDouble(n);
      Py_XDECREF(n);
    }
    if (PyErr_Occurred()) ok = false;
    return (float)v;
  }
  int integer(int i) {                       // ... and a c_int: whatever has __index__
    if (!ok) return 0;
    PyObject* n = PyNumber_Index(a[i]);
    if (!n) n = boxed(a[i], "c_int");
    const int v = n ? (int)PyLong_AsUnsignedLongMask(n) : 0;
    Py_XDECREF(n);
    if (PyErr_Occurred()) ok = false;
    return v;
  }
  int flag(int i) {
    if (!ok) return 0;
    PyObject* n = PyNumber_Long(a[i]);      // as int() takes it
    const int v = n ? (int)PyLong_AsUnsignedLongMask(n) : 0;
    Py_XDECREF(n);
    if (PyErr_Occurred()) ok = false;
    return v;
  }
  void* stream() {
    if (!ok) return nullptr;
    PyObject* d = PyObject_CallNoArgs(g_device);
    PyObject* s = d ? PyObject_CallOneArg(g_stream, d) : nullptr;
    void* p = s ? PyLong_AsVoidPtr(s) : nullptr;
    Py_XDECREF(d);
    Py_XDECREF(s);
    if (PyErr_Occurred()) ok = false;
    return p;
  }
};

bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

template <typename F>
PyObject* finish(Args& g, F call) {
  if (!g.ok) return nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (desc, x, w, bias, q_x, q_w, q_out, residual, q_res, out, acc_dump, workspace)
PyObject* conv_int8(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 12)) return nullptr;
  Args g{args};
  const q8_conv_desc* d = g.desc(0);
  const int8_t *x = g.i8(1), *w = g.i8(2);
  const int32_t* b = g.i32(3);
  const float q_x = g.factor(4), q_w = g.factor(5), q_out = g.factor(6);
  const int8_t* res = g.i8(7);
  const float q_res = g.factor(8);
  int8_t* y = g.i8(9);
  int32_t* dump = g.i32(10);
  long bytes = 0;
  void* ws = g.tensor<uint8_t>(11, at::kByte, g_uint8, &bytes);
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_conv_int8))g_fn[kInt8])(d, x, w, b, q_x, q_w, q_out, res, q_res, y, dump, ws,
                                                  (size_t)bytes, s);
  });
}

// (desc, in_u8, out_u8, res_u8, x, w, bias, taps, q_x, q_w, q_out, residual, q_res, out, acc_dump)
PyObject* conv_u8(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 15)) return nullptr;
  Args g{args};
  const q8_conv_desc* d = g.desc(0);
  const int in = g.flag(1), out = g.flag(2), ru = g.flag(3);
  const int8_t *x = g.i8(4), *w = g.i8(5);
  const int32_t *b = g.i32(6), *taps = g.i32(7);
  const float q_x = g.factor(8), q_w = g.factor(9), q_out = g.factor(10);
  const int8_t* res = g.i8(11);
  const float q_res = g.factor(12);
  int8_t* y = g.i8(13);
  int32_t* dump = g.i32(14);
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_conv_u8))g_fn[kU8])(d, in, out, ru, x, w, b, taps, q_x, q_w, q_out, res, q_res, y,
                                              dump, s);
  });
}

// (desc, x, w, bias, m, q_out, residual, q_res, out, acc_dump)
PyObject* conv_per_channel(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 10)) return nullptr;
  Args g{args};
  const q8_conv_desc* d = g.desc(0);
  const int8_t *x = g.i8(1), *w = g.i8(2);
  const int32_t* b = g.i32(3);
  const float* m = g.f32(4);
  const float q_out = g.factor(5);
  const int8_t* res = g.i8(6);
  const float q_res = g.factor(7);
  int8_t* y = g.i8(8);
  int32_t* dump = g.i32(9);
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_conv_int8_per_channel))g_fn[kPerChannel])(d, x, w, b, m, q_out, res, q_res, y, dump, s);
  });
}

// (desc, x, w, bias, q_x, q_w, residual, q_res, out)
PyObject* conv_real(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  Args g{args};
  const q8_conv_desc* d = g.desc(0);
  const int8_t* x = g.i8(1);
  const void* w = g.tensor<void>(2, at::ScalarType::Undefined, Py_None);
  const int32_t* b = g.i32(3);
  const float q_x = g.factor(4), q_w = g.factor(5);
  const int8_t* res = g.i8(6);
  const float q_res = g.factor(7);
  float* y = g.f32(8);
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_conv_int8_real_output))g_fn[kReal])(d, x, w, b, q_x, q_w, res, q_res, y, s);
  });
}

// (desc, x, w, bias, residual, out, maxabs_sum, maxabs_out, copies)
PyObject* conv_f32(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  Args g{args};
  const q8_conv_desc* d = g.desc(0);
  const float *x = g.f32(1), *w = g.f32(2), *b = g.f32(3), *res = g.f32(4);
  float *y = g.f32(5), *m_sum = g.f32(6), *m_out = g.f32(7);
  const int copies = g.ok ? (int)PyLong_AsLong(args[8]) : 0;
  if (PyErr_Occurred()) g.ok = false;
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_conv_f32_observed_spread))g_fn[kF32])(d, x, w, b, res, y, m_sum, m_out, copies, s);
  });
}

// (x, maximum)
PyObject* maxabs(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 2)) return nullptr;
  Args g{args};
  long len = 0;
  const float* x = g.counted<float>(0, at::kFloat, g_float32, &len);
  float* m = g.f32(1);
  void* s = g.stream();
  return finish(g, [&] { return ((decltype(&q8_calibrate_maxabs))g_fn[kMaxabs])(x, (size_t)len, m, s); });
}

// (r, q, p, z)
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 4)) return nullptr;
  Args g{args};
  long len = 0;
  const float* r = g.counted<float>(0, at::kFloat, g_float32, &len);
  const float q = g.factor(1);
  const int p = g.integer(2);
  int8_t* z = g.i8(3);
  void* s = g.stream();
  return finish(g, [&] { return ((decltype(&q8_quantize))g_fn[kQuantize])(r, (size_t)len, q, p, z, s); });
}

// (z, q, r)
PyObject* dequantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 3)) return nullptr;
  Args g{args};
  long len = 0;
  const int8_t* z = g.counted<int8_t>(0, at::kChar, g_int8, &len);
  const float q = g.factor(1);
  float* r = g.f32(2);
  void* s = g.stream();
  return finish(g, [&] { return ((decltype(&q8_dequantize))g_fn[kDequantize])(z, (size_t)len, q, r, s); });
}

// ---- the operators on rows, on the caches and on their pages: tensors with strides, of several types.  What a call cannot pass on
// raises an AssertionError; tensors' subclasses (parameters) are taken as tensors.
struct Strided {
  void* p = nullptr;
  long size[4] = {0, 0, 0, 0}, stride[4] = {0, 0, 0, 0}, n = 0;
  int type = -1, dims = 0;             // Q8_* of real values
  int device = -1;
};
struct TensorArgs : Args {
  explicit TensorArgs(PyObject* const* args) : Args{args} {}
  void refuse(int i, const char* what) {
    if (ok && !PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "argument %d: %s", i, what);
    ok = false;
  }
  // A device tensor of that type (Undefined: fp32, fp16 or bf16) and number of dimensions (-1: any) whose last `dense`
  // ones are dense (-1: all).
  Strided get(int i, at::ScalarType type, int dims, int dense, bool none = false) {
    Strided s;
    if (!ok || (none && a[i] == Py_None)) return s;
    if (!THPVariable_Check(a[i])) {
      refuse(i, "expected a tensor");
      return s;
    }
    try {
      const at::Tensor& t = THPVariable_Unpack(a[i]);
      if (!t.is_cuda() || !t.has_storage() || t.layout() != at::kStrided) {
        refuse(i, "expected a device tensor");
        return s;
      }
      const at::ScalarType st = t.scalar_type();
      s.type = st == at::kFloat ? Q8_F32 : st == at::kHalf ? Q8_F16 : st == at::kBFloat16 ? Q8_BF16 : -1;
      if (type == at::ScalarType::Undefined ? s.type < 0 : st != type) refuse(i, "type of its elements");
      if (dims >= 0 && t.dim() != dims) refuse(i, "number of dimensions");
      if (!ok) return s;
      if (dense < 0 && !t.is_contiguous()) refuse(i, "expected a contiguous tensor");
      long run = 1;
      for (int d = (int)t.dim() - 1; d >= 0; --d) {
        if (d < 4) s.size[d] = t.size(d), s.stride[d] = t.stride(d);
        if (d > 0 && t.size(d) > 0x7fffffff) refuse(i, "more than an int counts");       // (the first: as the call says)
        if (d >= t.dim() - dense && t.size(d) > 1 && t.stride(d) != run && t.numel() > 0) refuse(i, "expected dense rows");
        run *= t.size(d);
      }
      s.n = t.numel();
      s.dims = (int)t.dim();
      s.device = t.get_device();
      s.p = t.mutable_data_ptr();
    } catch (...) {            // (none may leave through the interpreter's frames)
      refuse(i, "expected a device tensor with storage");
    }
    return s;
  }
  // Elements between the rows of [M][cols], also where there is one row only.
  static size_t row_stride(const Strided& s) { return s.size[0] > 1 ? s.stride[0] : s.size[1] > 1 ? s.size[1] : 1; }
  // Codes [M][K]: the storage holds the last row up to a multiple of 16 bytes.
  Strided codes(int i, size_t* stride) {
    const Strided s = get(i, at::kChar, 2, 1);
    if (!ok) return s;
    const long K16 = (s.size[1] + 15) / 16 * 16;
    const long between = s.size[0] > 1 ? s.stride[0] : K16;
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (s.size[0] > 0 && t.storage_offset() + (s.size[0] - 1) * between + K16 > (long)t.storage().nbytes())
      refuse(i, "codes: rows to a multiple of 16 bytes");
    *stride = between;
    return s;
  }
  void check(bool fine, int i, const char* what) {
    if (ok && !fine) refuse(i, what);
  }
  // All of them on the device whose stream the call takes.
  void check_device(std::initializer_list<const Strided*> all) {
    if (!ok) return;
    PyObject* d = PyObject_CallNoArgs(g_device);
    const long current = d ? PyLong_AsLong(d) : -1;
    Py_XDECREF(d);
    if (PyErr_Occurred()) ok = false;
    for (const Strided* s : all) check(s->device < 0 || s->device == current, 0, "every tensor on the current device");
  }
};

// (x, codes, factors)
PyObject* quantize_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 3)) return nullptr;
  TensorArgs g{args};
  const Strided x = g.get(0, at::ScalarType::Undefined, 2, 1), q = g.get(2, at::kFloat, -1, -1);
  size_t z_stride = 0;
  const Strided z = g.codes(1, &z_stride);
  g.check(z.size[0] == x.size[0] && z.size[1] == x.size[1], 1, "shape");
  g.check(q.n == x.size[0], 2, "one factor for each row");
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_quantize_rows))g_fn[kRows])(x.p, x.type, x.size[0], (int)x.size[1], g.row_stride(x),
                                                      (int8_t*)z.p, z_stride, (float*)q.p, s);
  });
}

// Weights, factors, bias and output from argument i on, for M rows of K values.
struct Product {
  Strided w, q_w, bias, y;
  Product(TensorArgs& g, int i, long M, long K)
      : w(g.get(i, at::kChar, -1, -1)), q_w(g.get(i + 1, at::kFloat, -1, -1)),
        bias(g.get(i + 2, at::kFloat, -1, -1, true)), y(g.get(i + 3, at::ScalarType::Undefined, 2, 1)) {
    if (!g.ok) return;
    const size_t bytes = ((decltype(&q8_linear_packed_bytes))g_fn[kPackedBytes])((int)q_w.n, (int)K);
    // (as linear_pack leaves them, [blocks of 16 outputs][blocks of 64 values][bytes], or any memory that holds as much)
    const bool blocks = w.dims != 3 || (w.size[0] == (q_w.n + 15) / 16 && w.size[1] == (K + 63) / 64);
    g.check(q_w.n < 0x7fffffff && blocks && (size_t)w.n >= bytes, i, "weights packed for other sizes");
    g.check(!bias.p || bias.n == q_w.n, i + 2, "one bias for each output");
    g.check(y.size[0] == M && y.size[1] == q_w.n, i + 3, "shape");
  }
};

// (codes, q_x, w, q_w, bias, out, variant)
PyObject* linear_int8(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 7)) return nullptr;
  TensorArgs g{args};
  size_t z_stride = 0;
  const Strided z = g.codes(0, &z_stride), q_x = g.get(1, at::kFloat, -1, -1);
  g.check(q_x.n == z.size[0], 1, "one factor for each row");
  const Product p(g, 2, z.size[0], z.size[1]);
  const int variant = g.integer(6);
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_linear_int8_variant))g_fn[kLinearInt8])(
        (const int8_t*)z.p, z_stride, (const float*)q_x.p, z.size[0], (int)p.q_w.n, (int)z.size[1], p.w.p,
        (const float*)p.q_w.p, (const float*)p.bias.p, p.y.p, p.y.type, g.row_stride(p.y), variant, s);
  });
}

// (x, w, q_w, bias, out, workspace)
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 6)) return nullptr;
  TensorArgs g{args};
  const Strided x = g.get(0, at::ScalarType::Undefined, 2, 1), ws = g.get(5, at::kByte, -1, -1);
  const Product p(g, 1, x.size[0], x.size[1]);
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_linear))g_fn[kLinear])(x.p, x.type, g.row_stride(x), x.size[0], (int)p.q_w.n, (int)x.size[1],
                                                 p.w.p, (const float*)p.q_w.p, (const float*)p.bias.p, p.y.p, p.y.type,
                                                 g.row_stride(p.y), ws.p, ws.n, s);
  });
}

// (lengths, added, page, free, table, slots, positions, starts, grown, counts)
PyObject* page_tables(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 10)) return nullptr;
  TensorArgs g{args};
  const Strided len = g.get(0, at::kInt, -1, -1), add = g.get(1, at::kInt, -1, -1), fr = g.get(3, at::kInt, -1, -1),
                table = g.get(4, at::kInt, 2, 1), slots = g.get(5, at::kLong, -1, -1),
                pos = g.get(6, at::kInt, -1, -1), starts = g.get(7, at::kInt, -1, -1), grown = g.get(8, at::kInt, -1, -1),
                counts = g.get(9, at::kInt, -1, -1);
  const int page = g.integer(2);
  g.check(add.n == len.n, 1, "one number for each request");
  g.check(table.size[0] == len.n, 4, "one row for each request");
  g.check(pos.n == slots.n, 6, "one position for each slot");
  g.check(starts.n == len.n + 1 && grown.n == len.n && counts.n == 3, 7, "starts, lengths and counts");
  g.check((len.n | fr.n | slots.n | table.size[1]) < 0x7fffffff, 0, "sizes");
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_page_tables))g_fn[kPages])(
        (const int32_t*)len.p, (const int32_t*)add.p, (int)len.n, page, (const int32_t*)fr.p, (int)fr.n,
        (int32_t*)table.p, (int)table.size[1],
        table.size[0] > 1 ? (size_t)table.stride[0] : (size_t)table.size[1], (int64_t*)slots.p, (int32_t*)pos.p,
        (int)slots.n, (int32_t*)starts.p, (int32_t*)grown.p, (int32_t*)counts.p, s);
  });
}

// A cache uint8 [pages][heads][page / 16][18 D] (4 bits) or [32 D + 64] (8 bits).
struct Cache {
  Strided c;
  int heads, page, D;
  Cache(TensorArgs& g, int i, int bits = 4) : c(g.get(i, at::kByte, 4, -1)) {
    const long per = bits == 4 ? 18 : 32, more = bits == 4 ? 0 : 64, channels = c.size[3] - more;
    g.check(channels >= 0 && channels % per == 0 && c.size[2] <= 0x7ffffff, i, "the cache's shape");
    heads = (int)c.size[1], page = (int)(c.size[2] * 16), D = (int)(channels / per);
  }
};
// [tokens][heads][D]: elements between tokens and between heads, also where there is one only.
struct Tokens {
  Strided t;
  size_t token, head;
  Tokens(TensorArgs& g, int i) : t(g.get(i, at::ScalarType::Undefined, 3, 1)) {
    token = t.size[0] > 1 ? t.stride[0] : t.size[1] * t.size[2];
    head = t.size[1] > 1 ? t.stride[1] : t.size[2];
  }
};

void check_tokens(TensorArgs& g, const Cache& c, const Tokens& k, const Tokens& v, const Strided& slots, int i) {
  for (const Tokens* t : {&k, &v})
    g.check(t->t.size[0] == slots.n && t->t.size[1] == c.heads && t->t.size[2] == c.D, i, "[slots, heads, D] each");
  g.check(k.t.type == v.t.type, i, "keys and values of one type");
}

// (cache, k, v, slots)
PyObject* kv4_write(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 4)) return nullptr;
  TensorArgs g{args};
  const Cache c(g, 0);
  const Tokens k(g, 1), v(g, 2);
  const Strided slots = g.get(3, at::kLong, -1, -1);
  check_tokens(g, c, k, v, slots, 1);
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_kv4_write))g_fn[kKv4Write])(k.t.p, v.t.p, k.t.type, slots.n, c.heads, c.D, k.token, k.head,
                                                      v.token, v.head, (const int64_t*)slots.p, c.c.p, c.c.size[0],
                                                      c.page, s);
  });
}

// (cache, slots, k, v)
PyObject* kv4_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 4)) return nullptr;
  TensorArgs g{args};
  const Cache c(g, 0);
  const Strided slots = g.get(1, at::kLong, -1, -1);
  const Tokens k(g, 2), v(g, 3);
  check_tokens(g, c, k, v, slots, 2);
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_kv4_read))g_fn[kKv4Read])(c.c.p, c.c.size[0], c.page, (const int64_t*)slots.p, slots.n,
                                                    c.heads, c.D, k.t.p, v.t.p, k.t.type, k.token, k.head, v.token,
                                                    v.head, s);
  });
}

// (q, cache, table, lengths, starts, scale, window, out, workspace)
PyObject* kv4_attend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  TensorArgs g{args};
  const Tokens q(g, 0);
  const Cache c(g, 1);
  const Strided table = g.get(2, at::kInt, 2, 1), len = g.get(3, at::kInt, -1, -1),
                starts = g.get(4, at::kInt, -1, -1, true);
  const float scale = g.factor(5);
  const int window = g.integer(6);
  const Tokens out(g, 7);
  const Strided ws = g.get(8, at::kByte, -1, -1, true);
  g.check(q.t.size[2] == c.D && c.heads > 0 && q.t.size[1] % c.heads == 0, 0, "[tokens, a multiple of the heads, D]");
  g.check(out.t.size[0] == q.t.size[0] && out.t.size[1] == q.t.size[1] && out.t.size[2] == q.t.size[2], 7, "shape");
  g.check(out.t.type == q.t.type, 7, "queries and outputs of one type");
  g.check(table.size[0] == len.n && len.n < 0x7fffffff && table.size[1] < 0x7fffffff, 2, "one row for each request");
  if (g.ok && g.a[4] == Py_None) g.check(q.t.size[0] == len.n, 0, "one row for each request");
  else g.check(starts.n == len.n + 1, 4, "one start for each request, and the end");
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_kv4_attend))g_fn[kKv4Attend])(
        q.t.p, q.t.type, q.t.size[0], c.heads, (int)(q.t.size[1] / c.heads), c.D, q.token, q.head, c.c.p, c.c.size[0],
        c.page, (const int32_t*)table.p, (int)table.size[1],
        table.size[0] > 1 ? (size_t)table.stride[0] : (size_t)table.size[1], (const int32_t*)len.p,
        (const int32_t*)starts.p, (int)len.n, scale, window, out.t.p, out.token, out.head, ws.p, ws.n, s);
  });
}

// (cache, k, v, slots)
PyObject* kv8_write(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 4)) return nullptr;
  TensorArgs g{args};
  const Cache c(g, 0, 8);
  const Tokens k(g, 1), v(g, 2);
  const Strided slots = g.get(3, at::kLong, -1, -1);
  check_tokens(g, c, k, v, slots, 1);
  g.check_device({&c.c, &k.t, &v.t, &slots});
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_kv8_write))g_fn[kKv8Write])(k.t.p, v.t.p, k.t.type, slots.n, c.heads, c.D, k.token, k.head,
                                                      v.token, v.head, (const int64_t*)slots.p, c.c.p, c.c.size[0],
                                                      c.page, s);
  });
}

// (cache, slots, k, v)
PyObject* kv8_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 4)) return nullptr;
  TensorArgs g{args};
  const Cache c(g, 0, 8);
  const Strided slots = g.get(1, at::kLong, -1, -1);
  const Tokens k(g, 2), v(g, 3);
  check_tokens(g, c, k, v, slots, 2);
  g.check_device({&c.c, &k.t, &v.t, &slots});
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_kv8_read))g_fn[kKv8Read])(c.c.p, c.c.size[0], c.page, (const int64_t*)slots.p, slots.n,
                                                    c.heads, c.D, k.t.p, v.t.p, k.t.type, k.token, k.head, v.token,
                                                    v.head, s);
  });
}

// (q, cache, table, lengths, starts, scale, window, causal, out, workspace)
PyObject* kv8_attend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 10)) return nullptr;
  TensorArgs g{args};
  const Tokens q(g, 0);
  const Cache c(g, 1, 8);
  const Strided table = g.get(2, at::kInt, 2, 1), len = g.get(3, at::kInt, -1, -1),
                starts = g.get(4, at::kInt, -1, -1, true);
  const float scale = g.factor(5);
  const int window = g.integer(6), causal = g.integer(7);
  const Tokens out(g, 8);
  const Strided ws = g.get(9, at::kByte, -1, -1, true);
  g.check(q.t.size[2] == c.D && c.heads > 0 && q.t.size[1] % c.heads == 0, 0, "[tokens, a multiple of the heads, D]");
  g.check(out.t.size[0] == q.t.size[0] && out.t.size[1] == q.t.size[1] && out.t.size[2] == q.t.size[2], 8, "shape");
  g.check(out.t.type == q.t.type, 8, "queries and outputs of one type");
  g.check(table.size[0] == len.n && len.n < 0x7fffffff && table.size[1] < 0x7fffffff, 2, "one row for each request");
  if (g.ok && g.a[4] == Py_None) g.check(q.t.size[0] == len.n, 0, "one row for each request");
  else g.check(starts.n == len.n + 1, 4, "one start for each request, and the end");
  g.check_device({&q.t, &c.c, &table, &len, &starts, &out.t, &ws});
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_kv8_attend))g_fn[kKv8Attend])(
        q.t.p, q.t.type, q.t.size[0], c.heads, (int)(q.t.size[1] / c.heads), c.D, q.token, q.head, c.c.p, c.c.size[0],
        c.page, (const int32_t*)table.p, (int)table.size[1], g.row_stride(table), (const int32_t*)len.p,
        (const int32_t*)starts.p, (int)len.n, scale, window, causal, out.t.p, out.token, out.head, ws.p, ws.n, s);
  });
}

// (parents, lengths, table, page, pages, out table, out lengths, free, copies, counts, workspace)
PyObject* page_select(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 11)) return nullptr;
  TensorArgs g{args};
  const Strided parents = g.get(0, at::kInt, -1, -1), len = g.get(1, at::kInt, -1, -1), table = g.get(2, at::kInt, 2, 1),
                rows = g.get(5, at::kInt, 2, 1), grown = g.get(6, at::kInt, -1, -1), fr = g.get(7, at::kInt, -1, -1),
                copies = g.get(8, at::kInt, 2, -1), counts = g.get(9, at::kInt, -1, -1), ws = g.get(10, at::kByte, -1, -1);
  const int page = g.integer(3), pool = g.integer(4);
  g.check(table.size[0] == len.n, 2, "one row for each request");
  g.check(rows.size[0] == parents.n && rows.size[1] == table.size[1] && grown.n == parents.n, 5,
          "one row, as long as the requests', and one length for each parent");
  g.check(pool >= 0 && fr.n == pool, 7, "as many places as pages");
  g.check(copies.size[0] == parents.n && copies.size[1] == 2, 8, "one pair for each parent");
  g.check(counts.n == 4, 9, "four counts");
  g.check((len.n | parents.n) < 0x7fffffff, 0, "sizes");
  g.check_device({&parents, &len, &table, &rows, &grown, &fr, &copies, &counts, &ws});
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_page_select))g_fn[kPageSelect])(
        (const int32_t*)parents.p, (int)parents.n, (const int32_t*)len.p, (const int32_t*)table.p, g.row_stride(table),
        (int)len.n, (int)table.size[1], page, (size_t)pool, (int32_t*)rows.p, g.row_stride(rows), (int32_t*)grown.p,
        (int32_t*)fr.p, (int32_t*)copies.p, (int32_t*)counts.p, ws.p, ws.n, s);
  });
}

// (lengths, table, page, pages, out table, free, copies, counts, workspace)
PyObject* page_compact(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  TensorArgs g{args};
  const Strided len = g.get(0, at::kInt, -1, -1), table = g.get(1, at::kInt, 2, 1), rows = g.get(4, at::kInt, 2, 1),
                fr = g.get(5, at::kInt, -1, -1), copies = g.get(6, at::kInt, 2, -1), counts = g.get(7, at::kInt, -1, -1),
                ws = g.get(8, at::kByte, -1, -1);
  const int page = g.integer(2), pool = g.integer(3);
  g.check(table.size[0] == len.n, 1, "one row for each request");
  g.check(rows.size[0] == table.size[0] && rows.size[1] == table.size[1], 4, "shape");
  g.check(pool >= 0 && fr.n == pool, 5, "as many places as pages");
  g.check(copies.size[0] == pool / 2 && copies.size[1] == 2, 6, "one pair for two pages");
  g.check(counts.n == 4, 7, "four counts");
  g.check(len.n < 0x7fffffff, 0, "sizes");
  g.check_device({&len, &table, &rows, &fr, &copies, &counts, &ws});
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_page_compact))g_fn[kPageCompact])(
        (const int32_t*)len.p, (const int32_t*)table.p, g.row_stride(table), (int)len.n, (int)table.size[1], page,
        (size_t)pool, (int32_t*)rows.p, g.row_stride(rows), (int32_t*)fr.p, (int32_t*)copies.p, (int32_t*)counts.p, ws.p,
        ws.n, s);
  });
}

// (cache [pages, ..], pairs)
PyObject* page_copy(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 2)) return nullptr;
  TensorArgs g{args};
  const Strided c = g.get(0, at::kByte, -1, -1), pairs = g.get(1, at::kInt, 2, -1);
  g.check(c.dims >= 1, 0, "number of dimensions");
  g.check(pairs.size[1] == 2 && pairs.size[0] < 0x7fffffff, 1, "pairs of pages");
  g.check_device({&c, &pairs});
  void* s = g.stream();
  return finish(g, [&] {
    return ((decltype(&q8_page_copy))g_fn[kPageCopy])(c.p, c.size[0], c.size[0] ? c.n / c.size[0] : 0,
                                                      (const int32_t*)pairs.p, (int)pairs.size[0], s);
  });
}

bool bind_functions(PyObject* const* args, int first, int end) {
  for (int i = first; i < end; ++i) {
    g_fn[i] = PyLong_AsVoidPtr(args[i - first]);
    if (PyErr_Occurred()) return false;
  }
  return true;
}

// bind(_ptr, get_device, get_stream, ConvDesc, int8, int32, float32, uint8, eight addresses)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, 8 + kLayerFunctions)) return nullptr;
  PyObject** keep[] = {&g_ptr, &g_device, &g_stream, &g_desc_type, &g_int8, &g_int32, &g_float32, &g_uint8};
  for (int i = 0; i < 8; ++i) {
    Py_INCREF(args[i]);
    *keep[i] = args[i];
  }
  if (!bind_functions(args + 8, 0, kLayerFunctions)) return nullptr;
  Py_RETURN_NONE;
}

// bind_rows(the addresses of the operators on rows, on the caches and on their pages)
PyObject* bind_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count(n, kFunctions - kLayerFunctions)) return nullptr;
  if (!bind_functions(args, kLayerFunctions, kFunctions)) return nullptr;
  Py_RETURN_NONE;
}

#define Q8_METHOD(F) {#F, (PyCFunction)(void (*)(void))F, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {Q8_METHOD(conv_int8), Q8_METHOD(conv_u8), Q8_METHOD(conv_per_channel),
                         Q8_METHOD(conv_real), Q8_METHOD(conv_f32), Q8_METHOD(maxabs), Q8_METHOD(quantize),
                         Q8_METHOD(dequantize), Q8_METHOD(quantize_rows), Q8_METHOD(linear_int8), Q8_METHOD(linear),
                         Q8_METHOD(page_tables), Q8_METHOD(kv4_write), Q8_METHOD(kv4_read), Q8_METHOD(kv4_attend),
                         Q8_METHOD(kv8_write), Q8_METHOD(kv8_read), Q8_METHOD(kv8_attend), Q8_METHOD(page_select),
                         Q8_METHOD(page_compact), Q8_METHOD(page_copy),
                         Q8_METHOD(bind), Q8_METHOD(bind_rows), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_q8call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__q8call(void) { return PyModule_Create(&module); }
