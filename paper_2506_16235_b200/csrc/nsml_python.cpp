// The 8-bit operators for Python: checks tensors and makes the call.  A call for a few tokens is bound by the host, and most of
// that was the interpreter and ctypes: attributes of up to eight tensors and up to 23 arguments, 3 to 8 us beside a launch of two.
// Tensors are reached through their Python attributes, so nothing here depends on torch's headers.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "nsml.h"

namespace {

PyObject *s_shape, *s_stride, *s_dtype, *s_get_device, *s_data_ptr, *s_numel;
PyObject *t_f32, *t_bf16, *t_int8;           // torch's types
PyObject *current_device, *current_stream;   // () -> index, (index) -> stream

constexpr int64_t kAny = -1;
enum Type { kFloat, kF32, kBf16, kInt8 };    // kFloat: either of the next two

struct Call {
  PyObject* index = nullptr;  // the current device's
  long device = 0;
  bool begin() {
    index = PyObject_CallNoArgs(current_device);
    if (index == nullptr) return false;
    device = PyLong_AsLong(index);
    return !(device == -1 && PyErr_Occurred());
  }
  bool stream(void** out) const {
    PyObject* s = PyObject_CallOneArg(current_stream, index);
    if (s == nullptr) return false;
    *out = reinterpret_cast<void*>((uintptr_t)PyLong_AsUnsignedLongLong(s));
    Py_DECREF(s);
    return PyErr_Occurred() == nullptr;
  }
  ~Call() { Py_XDECREF(index); }
};

bool integer(PyObject* o, int64_t* out) {  // takes the reference
  if (o == nullptr) return false;
  *out = PyLong_AsLongLong(o);
  Py_DECREF(o);
  return !(*out == -1 && PyErr_Occurred());
}

bool pointer(PyObject* t, void** out) {
  PyObject* o = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (o == nullptr) return false;
  *out = reinterpret_cast<void*>((uintptr_t)PyLong_AsUnsignedLongLong(o));
  Py_DECREF(o);
  return PyErr_Occurred() == nullptr;
}

bool on_device(PyObject* t, const char* what, const Call& call) {
  int64_t device;
  if (!integer(PyObject_CallMethodNoArgs(t, s_get_device), &device)) return false;
  if (device == call.device) return true;
  PyErr_Format(PyExc_ValueError, "%s must be a tensor of the current CUDA device", what);
  return false;
}

// The type's number among the library's (0 for codes).
bool typed(PyObject* t, const char* what, Type want, int* dtype) {
  PyObject* d = PyObject_GetAttr(t, s_dtype);
  if (d == nullptr) return false;
  bool ok = true;
  *dtype = d == t_bf16 ? NSML_BF16 : NSML_F32;
  if (want == kFloat) {
    if (d != t_f32 && d != t_bf16) {
      PyErr_SetString(PyExc_TypeError, "matrices must be float32 or bfloat16");
      ok = false;
    }
  } else {
    PyObject* wanted = want == kF32 ? t_f32 : want == kBf16 ? t_bf16 : t_int8;
    if (d != wanted) {
      PyErr_Format(PyExc_TypeError, "%s must be %S, not %S", what, wanted, d);
      ok = false;
    }
  }
  Py_DECREF(d);
  return ok;
}

struct Matrix {
  void* ptr = nullptr;
  int64_t rows = 0, cols = 0, ld = 0;
  int dtype = 0;
  Type type() const { return dtype == NSML_BF16 ? kBf16 : kF32; }

  // A 2-D tensor of the current device with contiguous rows, of that shape where it is given.
  bool from(PyObject* t, const char* what, const Call& call, Type want, int64_t want_rows = kAny, int64_t want_cols = kAny) {
    PyObject *shape = PyObject_GetAttr(t, s_shape), *stride = shape == nullptr ? nullptr : PyObject_CallMethodNoArgs(t, s_stride);
    bool ok = stride != nullptr;
    int64_t inner = 1;
    if (ok && (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != 2 || !PyTuple_Check(stride) || PyTuple_GET_SIZE(stride) != 2)) {
      PyErr_Format(PyExc_ValueError, "%s must be a 2-D tensor with contiguous rows", what);
      ok = false;
    }
    if (ok) {
      rows = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0));
      cols = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 1));
      ld = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 0));
      inner = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 1));
      ok = PyErr_Occurred() == nullptr;
    }
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    if (!ok) return false;
    if (inner != 1 && cols > 1) {
      PyErr_Format(PyExc_ValueError, "%s must be a 2-D tensor with contiguous rows", what);
      return false;
    }
    if ((want_rows != kAny && rows != want_rows) || (want_cols != kAny && cols != want_cols)) {
      PyErr_Format(PyExc_ValueError, "%s must have shape (%lld, %lld), not (%lld, %lld)", what, (long long)(want_rows == kAny ? rows : want_rows),
                   (long long)(want_cols == kAny ? cols : want_cols), (long long)rows, (long long)cols);
      return false;
    }
    return typed(t, what, want, &dtype) && on_device(t, what, call) && pointer(t, &ptr);
  }
};

// A contiguous 1-D tensor of n elements.
bool vector(PyObject* t, const char* what, const Call& call, Type want, int64_t n, void** ptr, int* dtype) {
  PyObject *shape = PyObject_GetAttr(t, s_shape), *stride = shape == nullptr ? nullptr : PyObject_CallMethodNoArgs(t, s_stride);
  bool ok = stride != nullptr;
  if (ok) {
    ok = PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 1 && PyTuple_Check(stride) && PyTuple_GET_SIZE(stride) == 1 &&
         PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0)) == n && (n <= 1 || PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 0)) == 1);
    if (!ok && !PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s must be a contiguous 1-D tensor of %lld elements", what, (long long)n);
  }
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  return ok && typed(t, what, want, dtype) && on_device(t, what, call) && pointer(t, ptr);
}
bool scales(PyObject* t, const char* what, const Call& call, int64_t n, float** ptr) {
  int dtype;
  return vector(t, what, call, kF32, n, reinterpret_cast<void**>(ptr), &dtype);
}

bool scratch(PyObject* t, const Call& call, void** ptr, int64_t* bytes) {
  return on_device(t, "workspace", call) && pointer(t, ptr) && integer(PyObject_CallMethodNoArgs(t, s_numel), bytes);
}

bool arguments(Py_ssize_t got, Py_ssize_t want) {
  if (got == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected", want);
  return false;
}

// The call, without the interpreter's lock (a launch may wait for room in the stream).
template <class F>
PyObject* result(F call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

int8_t* codes_of(const Matrix& m) { return static_cast<int8_t*>(m.ptr); }

PyObject* pack(PyObject*, PyObject* const* a, Py_ssize_t n) {  // x, codes, scales
  Call call;
  Matrix x, q;
  float* s;
  void* st;
  if (!arguments(n, 3) || !call.begin() || !x.from(a[0], "x", call, kFloat) || !q.from(a[1], "codes", call, kInt8, x.rows, x.cols) ||
      !scales(a[2], "scales", call, x.rows, &s) || !call.stream(&st))
    return nullptr;
  return result([&] { return nsml_q8_pack(x.ptr, x.rows, x.cols, x.ld, x.dtype, codes_of(q), q.ld, s, st); });
}

PyObject* unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {  // codes, scales, out
  Call call;
  Matrix q, out;
  float* s;
  void* st;
  if (!arguments(n, 3) || !call.begin() || !q.from(a[0], "codes", call, kInt8) || !scales(a[1], "scales", call, q.rows, &s) ||
      !out.from(a[2], "out", call, kFloat, q.rows, q.cols) || !call.stream(&st))
    return nullptr;
  return result([&] { return nsml_q8_unpack(codes_of(q), q.ld, s, q.rows, q.cols, out.ptr, out.ld, out.dtype, st); });
}

PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {  // x, weight, eps, residual, h, codes, scales, rstd
  Call call;
  Matrix x, r, h, q;
  void *w, *st;
  float *s, *rstd;
  int wtype;
  if (!arguments(n, 8) || !call.begin() || !x.from(a[0], "x", call, kFloat) || !vector(a[1], "weight", call, kFloat, x.cols, &w, &wtype)) return nullptr;
  const double eps = PyFloat_AsDouble(a[2]);
  if (eps == -1.0 && PyErr_Occurred()) return nullptr;
  if ((a[3] != Py_None && !r.from(a[3], "residual", call, x.type(), x.rows, x.cols)) || (a[4] != Py_None && !h.from(a[4], "h", call, x.type(), x.rows, x.cols)) ||
      !q.from(a[5], "codes", call, kInt8, x.rows, x.cols) || !scales(a[6], "scales", call, x.rows, &s) || !scales(a[7], "rstd", call, x.rows, &rstd) ||
      !call.stream(&st))
    return nullptr;
  return result([&] {
    return nsml_q8_rms_norm(x.ptr, x.ld, r.ptr, r.ld, x.rows, x.cols, x.dtype, w, wtype, eps, h.ptr, h.ld, codes_of(q), q.ld, s, rstd, st);
  });
}

// dy, weight, rstd, h, codes, scales, dh, dx, dweight, zero_first, workspace
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call call;
  Matrix dy, h, q, dh, dx;
  void *w, *dw, *ws, *st;
  float *s = nullptr, *rstd;
  int wtype, dwtype;
  int64_t bytes;
  if (!arguments(n, 11) || !call.begin() || !dy.from(a[0], "dy", call, kFloat)) return nullptr;
  if ((a[3] == Py_None) == (a[4] == Py_None)) {
    PyErr_SetString(PyExc_ValueError, "give h, or codes and scales");
    return nullptr;
  }
  const int zero_first = PyObject_IsTrue(a[9]);
  if (zero_first < 0 || !vector(a[1], "weight", call, kFloat, dy.cols, &w, &wtype) || !scales(a[2], "rstd", call, dy.rows, &rstd) ||
      (a[3] != Py_None && !h.from(a[3], "h", call, dy.type(), dy.rows, dy.cols)) ||
      (a[4] != Py_None && (!q.from(a[4], "codes", call, kInt8, dy.rows, dy.cols) || !scales(a[5], "scales", call, dy.rows, &s))) ||
      (a[6] != Py_None && !dh.from(a[6], "dh", call, dy.type(), dy.rows, dy.cols)) || !dx.from(a[7], "dx", call, dy.type(), dy.rows, dy.cols) ||
      !vector(a[8], "dweight", call, kFloat, dy.cols, &dw, &dwtype) || !scratch(a[10], call, &ws, &bytes) || !call.stream(&st))
    return nullptr;
  return result([&] {
    return nsml_q8_rms_norm_backward(dy.ptr, dy.ld, dh.ptr, dh.ld, h.ptr, h.ld, codes_of(q), q.ld, s, rstd, dy.rows, dy.cols, dy.dtype, w, wtype, dx.ptr, dx.ld, dw,
                                     dwtype, zero_first, ws, (size_t)bytes, st);
  });
}

PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {  // a, a_scales, b, b_scales, out, workspace
  Call call;
  Matrix x, y, out;
  float *sx, *sy;
  void *ws, *st;
  int64_t bytes;
  if (!arguments(n, 6) || !call.begin() || !x.from(a[0], "a", call, kInt8) || !y.from(a[2], "b", call, kInt8, kAny, x.cols) ||
      !scales(a[1], "a_scales", call, x.rows, &sx) || !scales(a[3], "b_scales", call, y.rows, &sy) || !out.from(a[4], "out", call, kFloat, x.rows, y.rows) ||
      !scratch(a[5], call, &ws, &bytes) || !call.stream(&st))
    return nullptr;
  return result([&] {
    return nsml_q8_matmul(codes_of(x), x.ld, sx, codes_of(y), y.ld, sy, x.rows, y.rows, x.cols, out.ptr, out.ld, out.dtype, ws, (size_t)bytes, st);
  });
}

PyObject* grad_input(PyObject*, PyObject* const* a, Py_ssize_t n) {  // dy, b, b_scales, dx, workspace
  Call call;
  Matrix dy, b, dx;
  float* s;
  void *ws, *st;
  int64_t bytes;
  if (!arguments(n, 5) || !call.begin() || !dy.from(a[0], "dy", call, kBf16) || !b.from(a[1], "b", call, kInt8, dy.cols) ||
      !scales(a[2], "b_scales", call, dy.cols, &s) || !dx.from(a[3], "dx", call, kFloat, dy.rows, b.cols) || !scratch(a[4], call, &ws, &bytes) || !call.stream(&st))
    return nullptr;
  return result([&] {
    return nsml_q8_matmul_grad_input(dy.ptr, dy.ld, codes_of(b), b.ld, s, dy.rows, dy.cols, b.cols, dx.ptr, dx.ld, dx.dtype, ws, (size_t)bytes, st);
  });
}

PyObject* grad_weight(PyObject*, PyObject* const* a, Py_ssize_t n) {  // dy, a, a_scales, dw, zero_first, workspace
  Call call;
  Matrix dy, x, dw;
  float* s;
  void *ws, *st;
  int64_t bytes;
  if (!arguments(n, 6) || !call.begin() || !dy.from(a[0], "dy", call, kBf16) || !x.from(a[1], "a", call, kInt8, dy.rows) ||
      !scales(a[2], "a_scales", call, dy.rows, &s) || !dw.from(a[3], "dw", call, kFloat, dy.cols, x.cols))
    return nullptr;
  const int zero_first = PyObject_IsTrue(a[4]);
  if (zero_first < 0 || !scratch(a[5], call, &ws, &bytes) || !call.stream(&st)) return nullptr;
  return result([&] {
    return nsml_q8_matmul_grad_weight(dy.ptr, dy.ld, codes_of(x), x.ld, s, dy.rows, dy.cols, x.cols, dw.ptr, dw.ld, dw.dtype, zero_first, ws, (size_t)bytes, st);
  });
}

// float32, bfloat16 and int8 as tensors name them, and the callables for the current device's index and its current stream
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 5)) return nullptr;
  PyObject** const to[5] = {&t_f32, &t_bf16, &t_int8, &current_device, &current_stream};
  for (int i = 0; i < 5; ++i) {
    Py_INCREF(a[i]);
    Py_XSETREF(*to[i], a[i]);
  }
  Py_RETURN_NONE;
}

#define NSML_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {NSML_METHOD(setup), NSML_METHOD(pack), NSML_METHOD(unpack), NSML_METHOD(rms_norm), NSML_METHOD(rms_norm_backward),
                         NSML_METHOD(matmul), NSML_METHOD(grad_input), NSML_METHOD(grad_weight), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "The 8-bit operators' calls: tensors are checked, the result is the library's status.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
  struct { PyObject** to; const char* name; } const names[] = {{&s_shape, "shape"}, {&s_stride, "stride"}, {&s_dtype, "dtype"},
                                                               {&s_get_device, "get_device"}, {&s_data_ptr, "data_ptr"}, {&s_numel, "numel"}};
  for (const auto& n : names)
    if ((*n.to = PyUnicode_InternFromString(n.name)) == nullptr) return nullptr;
  return PyModule_Create(&module);
}
