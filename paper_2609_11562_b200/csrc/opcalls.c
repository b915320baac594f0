/* Arguments of the operators beside the fused call (entwine_ops.h), from torch tensors to the C entry points: checks
 * of device, type, shape and strides, then the call.  The smallest calls last a few microseconds on the GPU; the same
 * checks in Python with a ctypes call took 6.7 to 8.4 us, of which 3.2 are the launch.
 *
 * The module knows neither torch nor the library: bind() hands it the entry points' addresses, torch's dtype objects,
 * the error class and how to ask for the current device and stream.  Tensors are used through their Python methods. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdarg.h>
#include <stdint.h>
#include <string.h>

enum { BF16, FP16, FP32, I8, I32, I64, U8, DTYPES };  /* the first four as in entwine_ops.h */
enum { LEAST_DTYPES = U8 };  /* bind() may be given no uint8: nothing is of that type then */
enum { FLOATING = 1 << BF16 | 1 << FP16 | 1 << FP32, ANY = FLOATING | 1 << I8, IDS = 1 << I32 | 1 << I64 };

static PyObject *dtypes[DTYPES], *error_class, *current_device, *current_stream;
static PyObject *s_get_device, *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_is_contiguous, *s_cuda_stream;

typedef int (*quant_fn)(const void*, int, int64_t, int64_t, int64_t, void*, int64_t, float*, void*);
typedef int (*gemm_fn)(const void*, int64_t, const float*, const void*, int64_t, const float*, const float*, void*, int,
                       int64_t, int64_t, int64_t, int64_t, void*);
typedef int (*grouped_fn)(const void*, int64_t, const float*, const void*, int64_t, int64_t, const float*, const float*,
                          const int32_t*, void*, int, int64_t, int64_t, int64_t, int64_t, int64_t, void*);
typedef int (*dispatch_fn)(const void*, int, int64_t, int64_t, int64_t, const float*, const void*, int, int64_t, int64_t,
                           void*, int64_t, float*, int32_t*, int32_t*, void*);
typedef int (*dispatch_bwd_fn)(const void*, int, int64_t, int64_t, int64_t, const int32_t*, int64_t, int64_t, void*,
                               int64_t, void*);
typedef int (*combine_fn)(const void*, int, int64_t, int64_t, int64_t, const float*, const int32_t*, int64_t, int64_t,
                          void*, int64_t, void*);
typedef int (*combine_bwd_fn)(const void*, int, int64_t, int64_t, int64_t, const void*, int64_t, int64_t, const float*,
                              const int32_t*, int64_t, void*, int64_t, float*, void*);

typedef int (*quant4_fn)(const void*, int, int64_t, int64_t, int64_t, void*, int64_t, void*, int64_t, void*);
typedef int (*dequant4_fn)(const void*, int64_t, const void*, int64_t, int64_t, int64_t, void*, int, int64_t, void*);
typedef int (*gemm4_fn)(const void*, int64_t, const void*, int64_t, const void*, int64_t, const void*, int64_t, const float*,
                        void*, int, int64_t, int64_t, int64_t, int64_t, void*);
typedef int (*grouped4_fn)(const void*, int64_t, const void*, int64_t, const void*, int64_t, int64_t, const void*, int64_t,
                           int64_t, const float*, const int32_t*, void*, int, int64_t, int64_t, int64_t, int64_t, int64_t,
                           void*);
typedef int (*dropout_fn)(const void*, int, int64_t, int64_t, int64_t, const void*, int64_t, double, const int64_t*, int64_t,
                          void*, int64_t, void*);
typedef int (*norm_fn)(const void*, int, int64_t, int64_t, int64_t, const void*, int64_t, double, const int64_t*, int64_t,
                       const void*, const void*, int, float, void*, int64_t, void*, int64_t, float*, float*, void*);
typedef int (*norm_bwd_fn)(const void*, int, int64_t, int64_t, int64_t, const void*, int64_t, const void*, int, const float*,
                           const float*, const void*, int64_t, double, const int64_t*, int64_t, void*, int64_t, void*,
                           int64_t, float*, float*, float*, int64_t, void*);

static quant_fn quant;
static gemm_fn gemm;
static grouped_fn grouped;
static dispatch_fn dispatch;
static dispatch_bwd_fn dispatch_bwd;
static combine_fn combine;
static combine_bwd_fn combine_bwd;
static quant4_fn quant4;
static dequant4_fn dequant4;
static gemm4_fn gemm4;
static grouped4_fn grouped4;
static dropout_fn dropout;
static norm_fn norm;
static norm_bwd_fn norm_bwd;

/* What bind() has to be given is fetched at the first call, by a function that calls it: until then the package needs no
 * torch. */
static PyObject* binder;
static int bound(void) {
  PyObject* o;
  if (error_class) return 1;
  if (!binder) {
    PyErr_SetString(PyExc_RuntimeError, "_opcalls: neither bind() nor on_first_call() has been called");
    return 0;
  }
  o = PyObject_CallNoArgs(binder);
  if (!o) return 0;
  Py_DECREF(o);
  if (error_class) return 1;
  PyErr_SetString(PyExc_RuntimeError, "_opcalls: the function of on_first_call() did not call bind()");
  return 0;
}
static PyObject* py_on_first_call(PyObject* self, PyObject* f) {
  Py_XSETREF(binder, Py_NewRef(f));
  Py_CLEAR(error_class); /* bound anew at the next call (a reloaded package has another error class) */
  Py_RETURN_NONE;
}

/* Raises EntwineError(code, what). */
static PyObject* fail(int code, const char* what) {
  PyObject* e = PyObject_CallFunction(error_class, "is", code, what);
  if (e) {
    PyErr_SetObject(error_class, e);
    Py_DECREF(e);
  }
  return NULL;
}
static int refuse(const char* format, ...) {
  char what[256];
  va_list args;
  va_start(args, format);
  vsnprintf(what, sizeof(what), format, args);
  va_end(args);
  PyErr_Clear();
  fail(-1, what); /* ENTWINE_ERR_INVALID */
  return 0;
}

/* The current device, on which the first argument has to lie; the others are compared with it.  -1: refused. */
static long device_of(PyObject* t) {
  PyObject* d = PyObject_CallMethodNoArgs(t, s_get_device);
  if (!d) return -1;
  const long v = PyLong_AsLong(d);
  Py_DECREF(d);
  return v;
}
static long first_device(PyObject* t, const char* name) {
  const long dev = device_of(t);
  long now = -2;
  if (dev >= 0) {
    PyObject* d = PyObject_CallNoArgs(current_device);
    if (!d) return -1;
    now = PyLong_AsLong(d);
    Py_DECREF(d);
  }
  if (dev < 0 || dev != now) {
    refuse("%s must be a tensor on the current CUDA device", name);
    return -1;
  }
  return dev;
}

/* Device and type of a tensor; its address. */
static int tensor(PyObject* t, const char* name, unsigned allowed, long dev, int* dtype, void** at) {
  int i;
  PyObject* o;
  if (device_of(t) != dev) return refuse("%s must be a tensor on the current CUDA device", name);
  o = PyObject_GetAttr(t, s_dtype);
  if (!o) return refuse("%s must be a tensor", name);
  Py_DECREF(o); /* (the bound dtype objects live on) */
  for (i = 0; i < DTYPES && o != dtypes[i]; ++i) {} /* (a slot that bind() was not given is NULL) */
  if (i == DTYPES || !(allowed >> i & 1)) return refuse("%s is of a type that this argument cannot have", name);
  *dtype = i;
  o = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!o) return 0;
  *at = PyLong_AsVoidPtr(o);
  Py_DECREF(o);
  return !PyErr_Occurred();
}
/* n numbers of a tuple; takes the reference. */
static int numbers(PyObject* tuple, int n, int64_t* out) {
  int i, ok = tuple && PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == n;
  for (i = 0; ok && i < n; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
    ok = !(out[i] == -1 && PyErr_Occurred());
  }
  Py_XDECREF(tuple);
  return ok;
}

typedef struct {
  void* at;
  int dtype;
  int64_t rows, cols, ld;
} Matrix;

/* A matrix whose rows are contiguous and do not overlap. */
static int matrix(PyObject* t, const char* name, unsigned allowed, long dev, Matrix* m) {
  int64_t shape[2], stride[2];
  if (!tensor(t, name, allowed, dev, &m->dtype, &m->at)) return 0;
  if (!numbers(PyObject_GetAttr(t, s_shape), 2, shape) || !numbers(PyObject_CallMethodNoArgs(t, s_stride), 2, stride))
    return refuse("%s must be a matrix", name);
  m->rows = shape[0];
  m->cols = shape[1];
  if ((stride[1] != 1 && m->cols > 1) || (stride[0] < m->cols && m->rows > 1))
    return refuse("%s must have contiguous rows that do not overlap (strides %lld, %lld)", name, (long long)stride[0],
                  (long long)stride[1]);
  m->ld = stride[0] > m->cols ? stride[0] : m->cols;
  return 1;
}
/* The same of known size. */
static int result(PyObject* t, const char* name, unsigned allowed, long dev, int64_t rows, int64_t cols, Matrix* m) {
  if (!matrix(t, name, allowed, dev, m)) return 0;
  if (m->rows != rows || m->cols != cols)
    return refuse("%s must be (%lld, %lld), not (%lld, %lld)", name, (long long)rows, (long long)cols, (long long)m->rows,
                  (long long)m->cols);
  return 1;
}
/* A contiguous tensor of n dimensions, which have to be a and b. */
static int dense(PyObject* t, const char* name, unsigned allowed, long dev, int n, int64_t a, int64_t b, void** at,
                 int* dtype) {
  int64_t shape[2];
  PyObject* o;
  int ok, ignored;
  if (!tensor(t, name, allowed, dev, dtype ? dtype : &ignored, at)) return 0;
  if (!numbers(PyObject_GetAttr(t, s_shape), n, shape) || shape[0] != a || (n == 2 && shape[1] != b))
    return n == 2 ? refuse("%s must be (%lld, %lld)", name, (long long)a, (long long)b)
                  : refuse("%s must be (%lld,)", name, (long long)a);
  o = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  ok = o == Py_True;
  Py_XDECREF(o);
  return ok ? 1 : refuse("%s must be contiguous", name);
}
static int optional(PyObject* t, const char* name, long dev, int n, int64_t a, int64_t b, void** at) {
  *at = NULL;
  return t == Py_None || dense(t, name, 1 << FP32, dev, n, a, b, at, NULL);
}
/* The two extents of the routing, [T, k]. */
static int routing(PyObject* t, const char* name, int64_t* extents) {
  return numbers(PyObject_GetAttr(t, s_shape), 2, extents) ? 1 : refuse("%s must be a tensor [T, k]", name);
}

/* A stream: None (the current one), a raw handle, or an object that has one. */
static int stream_of(PyObject* s, long dev, void** out) {
  PyObject* o;
  if (s == Py_None) o = PyObject_CallFunction(current_stream, "l", dev);
  else if (PyLong_Check(s)) o = Py_NewRef(s);
  else o = PyObject_GetAttr(s, s_cuda_stream);
  if (!o) return 0;
  *out = PyLong_AsVoidPtr(o);
  Py_DECREF(o);
  return !PyErr_Occurred();
}

static int count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return 1;
  PyErr_Format(PyExc_TypeError, "takes %zd arguments, not %zd", want, n);
  return 0;
}
#define CALL(name, ...)                     \
  do {                                      \
    int code;                               \
    Py_BEGIN_ALLOW_THREADS                  \
    code = __VA_ARGS__;                     \
    Py_END_ALLOW_THREADS                    \
    if (code != 0) return fail(code, name); \
    Py_RETURN_NONE;                         \
  } while (0)

/* (x, q, scale, stream) */
static PyObject* py_quant_i8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, q;
  void *scale, *stream;
  long dev;
  if (!bound() || !count_is(n, 4) || (dev = first_device(a[0], "x")) < 0 || !matrix(a[0], "x", FLOATING, dev, &x) ||
      !result(a[1], "q", 1 << I8, dev, x.rows, x.cols, &q) ||
      !dense(a[2], "scale", 1 << FP32, dev, 1, x.rows, 0, &scale, NULL) || !stream_of(a[3], dev, &stream))
    return NULL;
  CALL("entwine_quant_i8", quant(x.at, x.dtype, x.rows, x.cols, x.ld, q.at, q.ld, scale, stream));
}

/* (a, scale_a, b, scale_b, out, bias, stream) */
static PyObject* py_gemm_i8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, w, c;
  void *sx, *sw, *bias, *stream;
  long dev;
  if (!bound() || !count_is(n, 7) || (dev = first_device(a[0], "a")) < 0 || !matrix(a[0], "a", 1 << I8, dev, &x) ||
      !matrix(a[2], "b", 1 << I8, dev, &w))
    return NULL;
  if (x.cols != w.cols) return refuse("a and b must have rows of one length"), NULL;
  if (!result(a[4], "out", FLOATING, dev, x.rows, w.rows, &c) ||
      !dense(a[1], "scale_a", 1 << FP32, dev, 1, x.rows, 0, &sx, NULL) ||
      !dense(a[3], "scale_b", 1 << FP32, dev, 1, w.rows, 0, &sw, NULL) ||
      !optional(a[5], "bias", dev, 1, w.rows, 0, &bias) || !stream_of(a[6], dev, &stream))
    return NULL;
  CALL("entwine_gemm_i8", gemm(x.at, x.ld, sx, w.at, w.ld, sw, bias, c.at, c.dtype, c.ld, x.rows, w.rows, x.cols, stream));
}

/* (a, scale_a, b, scale_b, offsets, out, bias, stream) */
static PyObject* py_gemm_i8_grouped(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, c;
  void *w, *sx, *sw, *bias, *offsets, *stream;
  int64_t s[3], d[3];
  int dtype;
  long dev;
  if (!bound() || !count_is(n, 8) || (dev = first_device(a[0], "a")) < 0 || !matrix(a[0], "a", 1 << I8, dev, &x) ||
      !tensor(a[2], "b", 1 << I8, dev, &dtype, &w))
    return NULL;
  if (!numbers(PyObject_GetAttr(a[2], s_shape), 3, s) || !numbers(PyObject_CallMethodNoArgs(a[2], s_stride), 3, d) ||
      s[0] < 1 || s[1] < 1 || s[2] != x.cols)
    return refuse("b must be [G, N, %lld]", (long long)x.cols), NULL;
  if ((d[2] != 1 && s[2] > 1) || (d[1] < s[2] && s[1] > 1) || (d[0] < (s[1] - 1) * d[1] + s[2] && s[0] > 1))
    return refuse("b must be matrices of contiguous rows that do not overlap"), NULL;
  if (!result(a[5], "out", FLOATING, dev, x.rows, s[1], &c) ||
      !dense(a[1], "scale_a", 1 << FP32, dev, 1, x.rows, 0, &sx, NULL) ||
      !dense(a[3], "scale_b", 1 << FP32, dev, 2, s[0], s[1], &sw, NULL) ||
      !dense(a[4], "offsets", 1 << I32, dev, 1, s[0] + 1, 0, &offsets, NULL) ||
      !optional(a[6], "bias", dev, 2, s[0], s[1], &bias) || !stream_of(a[7], dev, &stream))
    return NULL;
  CALL("entwine_gemm_i8_grouped", grouped(x.at, x.ld, sx, w, d[1] > s[2] ? d[1] : s[2], d[0], sw, bias, offsets, c.at,
                                          c.dtype, c.ld, x.rows, s[1], x.cols, s[0], stream));
}

/* (x, ids, n_experts, rows, offsets, row_of, x_scale, row_scale, stream) */
static PyObject* py_moe_dispatch(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, r;
  void *ids, *offsets, *row_of, *x_scale = NULL, *row_scale = NULL, *stream;
  int64_t e[2];
  long long experts;
  int id_type;
  long dev;
  if (!bound() || !count_is(n, 9) || (dev = first_device(a[0], "x")) < 0 || !matrix(a[0], "x", ANY, dev, &x) ||
      !routing(a[1], "ids", e))
    return NULL;
  experts = PyLong_AsLongLong(a[2]);
  if (experts == -1 && PyErr_Occurred()) return NULL;
  if (experts < 1 || experts > INT32_MAX - 1) return refuse("n_experts must be positive"), NULL;
  if (e[1] > INT32_MAX) return refuse("ids must be [T, k]"), NULL;
  if (!dense(a[1], "ids", IDS, dev, 2, x.rows, e[1], &ids, &id_type) ||
      !result(a[3], "rows", 1u << x.dtype, dev, x.rows * e[1], x.cols, &r) ||
      !dense(a[4], "offsets", 1 << I32, dev, 1, experts + 1, 0, &offsets, NULL) ||
      !dense(a[5], "row_of", 1 << I32, dev, 2, x.rows, e[1], &row_of, NULL))
    return NULL;
  if ((a[6] == Py_None) != (a[7] == Py_None)) return refuse("x_scale and row_scale go together"), NULL;
  if (!optional(a[6], "x_scale", dev, 1, x.rows, 0, &x_scale) ||
      !optional(a[7], "row_scale", dev, 1, x.rows * e[1], 0, &row_scale) || !stream_of(a[8], dev, &stream))
    return NULL;
  CALL("entwine_moe_dispatch", dispatch(x.at, x.dtype, x.rows, x.cols, x.ld, x_scale, ids, id_type == I64, e[1], experts,
                                        r.at, r.ld, row_scale, offsets, row_of, stream));
}

/* (d_rows, row_of, dx, stream) */
static PyObject* py_moe_dispatch_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix r, x;
  void *row_of, *stream;
  int64_t e[2];
  long dev;
  if (!bound() || !count_is(n, 4) || (dev = first_device(a[0], "d_rows")) < 0 || !matrix(a[0], "d_rows", FLOATING, dev, &r) ||
      !routing(a[1], "row_of", e) || !dense(a[1], "row_of", 1 << I32, dev, 2, e[0], e[1], &row_of, NULL) ||
      !result(a[2], "dx", 1u << r.dtype, dev, e[0], r.cols, &x) || !stream_of(a[3], dev, &stream))
    return NULL;
  CALL("entwine_moe_dispatch_bwd",
       dispatch_bwd(r.at, r.dtype, r.rows, r.cols, r.ld, row_of, e[0], e[1], x.at, x.ld, stream));
}

/* (y, weights, row_of, out, stream) */
static PyObject* py_moe_combine(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix y, o;
  void *w, *row_of, *stream;
  int64_t e[2];
  long dev;
  if (!bound() || !count_is(n, 5) || (dev = first_device(a[0], "y")) < 0 || !matrix(a[0], "y", FLOATING, dev, &y) ||
      !routing(a[2], "row_of", e) || !dense(a[2], "row_of", 1 << I32, dev, 2, e[0], e[1], &row_of, NULL) ||
      !dense(a[1], "weights", 1 << FP32, dev, 2, e[0], e[1], &w, NULL) ||
      !result(a[3], "out", 1u << y.dtype, dev, e[0], y.cols, &o) || !stream_of(a[4], dev, &stream))
    return NULL;
  CALL("entwine_moe_combine", combine(y.at, y.dtype, y.rows, y.cols, y.ld, w, row_of, e[0], e[1], o.at, o.ld, stream));
}

/* (dout, y, weights, row_of, dy, dw, stream) */
static PyObject* py_moe_combine_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix g, y, dy;
  void *w, *row_of, *dw, *stream;
  int64_t e[2];
  long dev;
  if (!bound() || !count_is(n, 7) || (dev = first_device(a[0], "dout")) < 0 || !matrix(a[0], "dout", FLOATING, dev, &g) ||
      !routing(a[3], "row_of", e) || !dense(a[3], "row_of", 1 << I32, dev, 2, g.rows, e[1], &row_of, NULL) ||
      !matrix(a[1], "y", 1u << g.dtype, dev, &y))
    return NULL;
  if (y.cols != g.cols) return refuse("y must have rows as long as dout's"), NULL;
  if (!result(a[4], "dy", 1u << g.dtype, dev, y.rows, y.cols, &dy) ||
      !dense(a[2], "weights", 1 << FP32, dev, 2, g.rows, e[1], &w, NULL) ||
      !dense(a[5], "dw", 1 << FP32, dev, 2, g.rows, e[1], &dw, NULL) || !stream_of(a[6], dev, &stream))
    return NULL;
  CALL("entwine_moe_combine_bwd", combine_bwd(g.at, g.dtype, g.rows, g.cols, g.ld, y.at, y.rows, y.ld, w, row_of, e[1],
                                              dy.at, dy.ld, dw, stream));
}

/* Codes of rows of `cols` elements, or of as many as two a byte make, and their scales. */
static int codes(PyObject* q, const char* q_name, PyObject* scale, const char* scale_name, long dev, int64_t rows,
                 int64_t cols, Matrix* m, Matrix* s) {
  if (rows < 0) {
    if (!matrix(q, q_name, 1 << U8, dev, m)) return 0;
  } else if (!result(q, q_name, 1 << U8, dev, rows, (cols + 1) / 2, m)) {
    return 0;
  }
  return result(scale, scale_name, 1 << U8, dev, m->rows, (rows < 0 ? 2 * m->cols + 31 : cols + 31) / 32, s);
}

/* (x, q, scale, stream) */
static PyObject* py_quant_mxf4(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, q, s;
  void* stream;
  long dev;
  if (!bound() || !count_is(n, 4) || (dev = first_device(a[0], "x")) < 0 || !matrix(a[0], "x", FLOATING, dev, &x) ||
      !codes(a[1], "q", a[2], "scale", dev, x.rows, x.cols, &q, &s) || !stream_of(a[3], dev, &stream))
    return NULL;
  CALL("entwine_quant_mxf4", quant4(x.at, x.dtype, x.rows, x.cols, x.ld, q.at, q.ld, s.at, s.ld, stream));
}

/* (q, scale, x, stream) */
static PyObject* py_dequant_mxf4(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, q, s;
  void* stream;
  long dev;
  if (!bound() || !count_is(n, 4) || (dev = first_device(a[0], "q")) < 0 || !matrix(a[2], "x", FLOATING, dev, &x) ||
      !codes(a[0], "q", a[1], "scale", dev, x.rows, x.cols, &q, &s) || !stream_of(a[3], dev, &stream))
    return NULL;
  CALL("entwine_dequant_mxf4", dequant4(q.at, q.ld, s.at, s.ld, x.rows, x.cols, x.at, x.dtype, x.ld, stream));
}

/* (a, scale_a, b, scale_b, out, bias, stream) */
static PyObject* py_gemm_mxf4(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, sx, w, sw, c;
  void *bias, *stream;
  long dev;
  if (!bound() || !count_is(n, 7) || (dev = first_device(a[0], "a")) < 0 ||
      !codes(a[0], "a", a[1], "scale_a", dev, -1, 0, &x, &sx) || !codes(a[2], "b", a[3], "scale_b", dev, -1, 0, &w, &sw))
    return NULL;
  if (x.cols != w.cols) return refuse("a and b must have rows of one length"), NULL;
  if (!result(a[4], "out", FLOATING, dev, x.rows, w.rows, &c) || !optional(a[5], "bias", dev, 1, w.rows, 0, &bias) ||
      !stream_of(a[6], dev, &stream))
    return NULL;
  CALL("entwine_gemm_mxf4", gemm4(x.at, x.ld, sx.at, sx.ld, w.at, w.ld, sw.at, sw.ld, bias, c.at, c.dtype, c.ld, x.rows,
                                  w.rows, 2 * x.cols, stream));
}

/* Matrices [G, N, cols] whose rows are contiguous and do not overlap. */
static int stacked(PyObject* t, const char* name, long dev, int64_t cols, void** at, int64_t* s, int64_t* d) {
  int dtype;
  if (!tensor(t, name, 1 << U8, dev, &dtype, at)) return 0;
  if (!numbers(PyObject_GetAttr(t, s_shape), 3, s) || !numbers(PyObject_CallMethodNoArgs(t, s_stride), 3, d) || s[0] < 1 ||
      s[1] < 1 || s[2] != cols)
    return refuse("%s must be [G, N, %lld]", name, (long long)cols);
  if ((d[2] != 1 && s[2] > 1) || (d[1] < s[2] && s[1] > 1) || (d[0] < (s[1] - 1) * d[1] + s[2] && s[0] > 1))
    return refuse("%s must be matrices of contiguous rows that do not overlap", name);
  if (d[1] < s[2]) d[1] = s[2];
  return 1;
}

/* (a, scale_a, b, scale_b, offsets, out, bias, stream) */
static PyObject* py_gemm_mxf4_grouped(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, sx, c;
  void *w, *sw, *bias, *offsets, *stream;
  int64_t s[3], d[3], ss[3], sd[3];
  long dev;
  if (!bound() || !count_is(n, 8) || (dev = first_device(a[0], "a")) < 0 ||
      !codes(a[0], "a", a[1], "scale_a", dev, -1, 0, &x, &sx) || !stacked(a[2], "b", dev, x.cols, &w, s, d) ||
      !stacked(a[3], "scale_b", dev, sx.cols, &sw, ss, sd))
    return NULL;
  if (ss[0] != s[0] || ss[1] != s[1]) return refuse("b and scale_b must have as many experts and rows"), NULL;
  if (!result(a[5], "out", FLOATING, dev, x.rows, s[1], &c) ||
      !dense(a[4], "offsets", 1 << I32, dev, 1, s[0] + 1, 0, &offsets, NULL) ||
      !optional(a[6], "bias", dev, 2, s[0], s[1], &bias) || !stream_of(a[7], dev, &stream))
    return NULL;
  CALL("entwine_gemm_mxf4_grouped", grouped4(x.at, x.ld, sx.at, sx.ld, w, d[1], d[0], sw, sd[1], sd[0], bias, offsets, c.at,
                                             c.dtype, c.ld, x.rows, s[1], 2 * x.cols, s[0], stream));
}

/* p, the generator's state and the first row's number. */
typedef struct {
  double p;
  void* rng;
  long long row0;
} Drop;
static int drop_of(PyObject* p, PyObject* rng, PyObject* row0, long dev, Drop* d) {
  d->p = PyFloat_AsDouble(p);
  if (d->p == -1.0 && PyErr_Occurred()) return 0;
  d->row0 = PyLong_AsLongLong(row0);
  if (d->row0 == -1 && PyErr_Occurred()) {
    if (!PyErr_ExceptionMatches(PyExc_OverflowError)) return 0;
    return refuse("row0 is out of range");
  }
  d->rng = NULL;
  if (!(d->p >= 0.0 && d->p < 1.0)) return refuse("p must be at least 0 and below 1");
  if (rng == Py_None) return d->p == 0.0 ? 1 : refuse("rng must be a tensor where p is not 0");
  return dense(rng, "rng", 1 << I64, dev, 1, 2, 0, &d->rng, NULL);
}
/* A matrix of known size, or None. */
static int optional_matrix(PyObject* t, const char* name, unsigned allowed, long dev, int64_t rows, int64_t cols, Matrix* m) {
  memset(m, 0, sizeof(*m));
  return t == Py_None || result(t, name, allowed, dev, rows, cols, m);
}

/* (x, out, p, rng, row0, residual, stream) */
static PyObject* py_dropout(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, o, r;
  Drop d;
  void* stream;
  long dev;
  if (!bound() || !count_is(n, 7) || (dev = first_device(a[0], "x")) < 0 || !matrix(a[0], "x", FLOATING, dev, &x) ||
      !result(a[1], "out", 1u << x.dtype, dev, x.rows, x.cols, &o) ||
      !optional_matrix(a[5], "residual", 1u << x.dtype, dev, x.rows, x.cols, &r) || !drop_of(a[2], a[3], a[4], dev, &d) ||
      !stream_of(a[6], dev, &stream))
    return NULL;
  CALL("entwine_dropout", dropout(x.at, x.dtype, x.rows, x.cols, x.ld, r.at, r.ld, d.p, d.rng, d.row0, o.at, o.ld, stream));
}

/* (x, weight, bias, out, eps, mean, rstd, residual, hidden, p, rng, row0, stream) */
static PyObject* py_layer_norm(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix x, o, r, h;
  Drop d;
  void *w, *b = NULL, *mean, *rstd, *stream;
  int w_type;
  double eps;
  long dev;
  if (!bound() || !count_is(n, 13) || (dev = first_device(a[0], "x")) < 0 || !matrix(a[0], "x", FLOATING, dev, &x) ||
      !dense(a[1], "weight", 1u << x.dtype | 1 << FP32, dev, 1, x.cols, 0, &w, &w_type) ||
      (a[2] != Py_None && !dense(a[2], "bias", 1u << w_type, dev, 1, x.cols, 0, &b, NULL)) ||
      !result(a[3], "out", 1u << x.dtype, dev, x.rows, x.cols, &o))
    return NULL;
  eps = PyFloat_AsDouble(a[4]);
  if (eps == -1.0 && PyErr_Occurred()) return NULL;
  if (!optional(a[5], "mean", dev, 1, x.rows, 0, &mean) || !optional(a[6], "rstd", dev, 1, x.rows, 0, &rstd) ||
      !optional_matrix(a[7], "residual", 1u << x.dtype, dev, x.rows, x.cols, &r) ||
      !optional_matrix(a[8], "hidden", 1u << x.dtype, dev, x.rows, x.cols, &h) ||
      !drop_of(a[9], a[10], a[11], dev, &d) || !stream_of(a[12], dev, &stream))
    return NULL;
  CALL("entwine_layer_norm", norm(x.at, x.dtype, x.rows, x.cols, x.ld, r.at, r.ld, d.p, d.rng, d.row0, w, b, w_type,
                                  (float)eps, h.at, h.ld, o.at, o.ld, mean, rstd, stream));
}

/* (dout, hidden, weight, mean, rstd, dx, dweight, dbias, work, dhidden, dresidual, p, rng, row0, stream) */
static PyObject* py_layer_norm_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Matrix g, h, dx, dh, dr;
  Drop d;
  void *w, *mean, *rstd, *dw, *db, *work, *stream;
  int64_t floats[1];
  int w_type;
  long dev;
  if (!bound() || !count_is(n, 15) || (dev = first_device(a[0], "dout")) < 0 || !matrix(a[0], "dout", FLOATING, dev, &g) ||
      !result(a[1], "hidden", 1u << g.dtype, dev, g.rows, g.cols, &h) ||
      !dense(a[2], "weight", 1u << g.dtype | 1 << FP32, dev, 1, g.cols, 0, &w, &w_type) ||
      !dense(a[3], "mean", 1 << FP32, dev, 1, g.rows, 0, &mean, NULL) ||
      !dense(a[4], "rstd", 1 << FP32, dev, 1, g.rows, 0, &rstd, NULL) ||
      !result(a[5], "dx", 1u << g.dtype, dev, g.rows, g.cols, &dx) ||
      !dense(a[6], "dweight", 1 << FP32, dev, 1, g.cols, 0, &dw, NULL) || !optional(a[7], "dbias", dev, 1, g.cols, 0, &db))
    return NULL;
  if (!numbers(PyObject_GetAttr(a[8], s_shape), 1, floats)) return refuse("work must have one dimension"), NULL;
  if (!dense(a[8], "work", 1 << FP32, dev, 1, floats[0], 0, &work, NULL) ||
      !optional_matrix(a[9], "dhidden", 1u << g.dtype, dev, g.rows, g.cols, &dh) ||
      !optional_matrix(a[10], "dresidual", 1u << g.dtype, dev, g.rows, g.cols, &dr) ||
      !drop_of(a[11], a[12], a[13], dev, &d) || !stream_of(a[14], dev, &stream))
    return NULL;
  CALL("entwine_layer_norm_bwd",
       norm_bwd(g.at, g.dtype, g.rows, g.cols, g.ld, h.at, h.ld, w, w_type, mean, rstd, dh.at, dh.ld, d.p, d.rng, d.row0, dx.at,
                dx.ld, dr.at, dr.ld, dw, db, work, floats[0], stream));
}

static int entry(PyObject* addresses, const char* name, void* out) {
  PyObject* o = PyDict_GetItemString(addresses, name); /* borrowed */
  void* p;
  if (!o) {
    PyErr_Format(PyExc_KeyError, "no address of %s", name);
    return 0;
  }
  p = PyLong_AsVoidPtr(o);
  memcpy(out, &p, sizeof(p));
  return !PyErr_Occurred();
}

/* bind(addresses, dtypes, error, current_device, current_stream) */
static PyObject* py_bind(PyObject* self, PyObject* args) {
  PyObject *addresses, *types, *error, *device, *stream;
  int i;
  if (!PyArg_ParseTuple(args, "O!O!OOO", &PyDict_Type, &addresses, &PyTuple_Type, &types, &error, &device, &stream))
    return NULL;
  if (PyTuple_GET_SIZE(types) < LEAST_DTYPES || PyTuple_GET_SIZE(types) > DTYPES)
    return PyErr_Format(PyExc_ValueError, "%d to %d dtypes", LEAST_DTYPES, DTYPES);
  if (!entry(addresses, "entwine_quant_i8", &quant) || !entry(addresses, "entwine_gemm_i8", &gemm) ||
      !entry(addresses, "entwine_gemm_i8_grouped", &grouped) || !entry(addresses, "entwine_moe_dispatch", &dispatch) ||
      !entry(addresses, "entwine_moe_dispatch_bwd", &dispatch_bwd) ||
      !entry(addresses, "entwine_moe_combine", &combine) || !entry(addresses, "entwine_moe_combine_bwd", &combine_bwd) ||
      !entry(addresses, "entwine_quant_mxf4", &quant4) || !entry(addresses, "entwine_dequant_mxf4", &dequant4) ||
      !entry(addresses, "entwine_gemm_mxf4", &gemm4) || !entry(addresses, "entwine_gemm_mxf4_grouped", &grouped4) ||
      !entry(addresses, "entwine_dropout", &dropout) || !entry(addresses, "entwine_layer_norm", &norm) ||
      !entry(addresses, "entwine_layer_norm_bwd", &norm_bwd))
    return NULL;
  for (i = 0; i < DTYPES; ++i)
    Py_XSETREF(dtypes[i], i < PyTuple_GET_SIZE(types) ? Py_NewRef(PyTuple_GET_ITEM(types, i)) : NULL);
  Py_XSETREF(error_class, Py_NewRef(error));
  Py_XSETREF(current_device, Py_NewRef(device));
  Py_XSETREF(current_stream, Py_NewRef(stream));
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, "bind(addresses, dtypes, error, current_device, current_stream)"},
    {"on_first_call", py_on_first_call, METH_O, "on_first_call(f): f() is called before the first operator and calls bind()"},
    {"quant_i8", (PyCFunction)(void (*)(void))py_quant_i8, METH_FASTCALL, "(x, q, scale, stream)"},
    {"gemm_i8", (PyCFunction)(void (*)(void))py_gemm_i8, METH_FASTCALL, "(a, scale_a, b, scale_b, out, bias, stream)"},
    {"gemm_i8_grouped", (PyCFunction)(void (*)(void))py_gemm_i8_grouped, METH_FASTCALL,
     "(a, scale_a, b, scale_b, offsets, out, bias, stream)"},
    {"moe_dispatch", (PyCFunction)(void (*)(void))py_moe_dispatch, METH_FASTCALL,
     "(x, ids, n_experts, rows, offsets, row_of, x_scale, row_scale, stream)"},
    {"moe_dispatch_bwd", (PyCFunction)(void (*)(void))py_moe_dispatch_bwd, METH_FASTCALL, "(d_rows, row_of, dx, stream)"},
    {"moe_combine", (PyCFunction)(void (*)(void))py_moe_combine, METH_FASTCALL, "(y, weights, row_of, out, stream)"},
    {"moe_combine_bwd", (PyCFunction)(void (*)(void))py_moe_combine_bwd, METH_FASTCALL,
     "(dout, y, weights, row_of, dy, dw, stream)"},
    {"quant_mxf4", (PyCFunction)(void (*)(void))py_quant_mxf4, METH_FASTCALL, "(x, q, scale, stream)"},
    {"dequant_mxf4", (PyCFunction)(void (*)(void))py_dequant_mxf4, METH_FASTCALL, "(q, scale, x, stream)"},
    {"gemm_mxf4", (PyCFunction)(void (*)(void))py_gemm_mxf4, METH_FASTCALL, "(a, scale_a, b, scale_b, out, bias, stream)"},
    {"gemm_mxf4_grouped", (PyCFunction)(void (*)(void))py_gemm_mxf4_grouped, METH_FASTCALL,
     "(a, scale_a, b, scale_b, offsets, out, bias, stream)"},
    {"dropout", (PyCFunction)(void (*)(void))py_dropout, METH_FASTCALL, "(x, out, p, rng, row0, residual, stream)"},
    {"layer_norm", (PyCFunction)(void (*)(void))py_layer_norm, METH_FASTCALL,
     "(x, weight, bias, out, eps, mean, rstd, residual, hidden, p, rng, row0, stream)"},
    {"layer_norm_bwd", (PyCFunction)(void (*)(void))py_layer_norm_bwd, METH_FASTCALL,
     "(dout, hidden, weight, mean, rstd, dx, dweight, dbias, work, dhidden, dresidual, p, rng, row0, stream)"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_opcalls",
                                    "Argument marshalling of the operators beside the fused call.", -1, methods};

PyMODINIT_FUNC PyInit__opcalls(void) {
  s_get_device = PyUnicode_InternFromString("get_device");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  return PyModule_Create(&module);
}
