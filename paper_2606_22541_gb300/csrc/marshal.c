/* Argument marshalling of the calls that are short enough for it to count: the
 * e4m3 operators on plain tensors.  A Python wrapper spends 2.5 to 4 us on
 * attributes, checks and ctypes conversions, more than the launch itself (2.5
 * us); this takes about 1.
 *
 * The operators around a training step's expert products come second; they also
 * look at the device, which has to be the current one.
 *
 * Each function reads its tensors through their Python attributes (shape,
 * dtype, is_cuda, stride(), data_ptr()), calls the library's entry point with
 * the GIL released and returns its code.  Whatever is not as the entry point
 * wants it (another rank, type, stride or size, an empty extent) returns None
 * and calls nothing: the caller then goes through the checks that name what is
 * wrong. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef int (*quantize_fn)(const void*, int64_t, int32_t, int32_t, void*, int64_t, float*, int64_t, void*);
typedef int (*swiglu_fn)(const void*, const void*, int64_t, int32_t, int32_t, void*, int64_t, float*, int64_t, void*);
typedef int (*matmul_fn)(const void*, int64_t, const float*, int64_t, const void*, int64_t, const float*, int64_t, void*,
                         int64_t, int32_t, int32_t, int32_t, uint32_t*, void*);

static quantize_fn call_quantize;
static swiglu_fn call_swiglu;
static matmul_fn call_matmul;
static PyObject *bf16, *f32, *f8, *u8;            /* the dtypes' objects */
static PyObject *current_device, *current_stream; /* device index; raw handle of a device's stream */
static PyObject *n_shape, *n_dtype, *n_is_cuda, *n_stride, *n_data_ptr, *n_cuda_stream;

typedef struct {
  long long rows, cols, ld;
  void* ptr;
} Mat;

/* Two elements of a tuple of integers. */
static int two(PyObject* t, long long* a, long long* b) {
  int ok = t && PyTuple_Check(t) && PyTuple_GET_SIZE(t) == 2;
  if (ok) {
    *a = PyLong_AsLongLong(PyTuple_GET_ITEM(t, 0));
    *b = PyLong_AsLongLong(PyTuple_GET_ITEM(t, 1));
    ok = !PyErr_Occurred();
  }
  Py_XDECREF(t);
  return ok;
}

static int pointer(PyObject* t, void** p) {
  PyObject* v = PyObject_CallMethodNoArgs(t, n_data_ptr);
  if (!v) return 0;
  *p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

/* A 2-D CUDA tensor of dtype a (or b) with contiguous columns, neither extent
 * empty nor over 2^30.  A single row's stride says nothing: one that any row
 * may have is put in its place. */
static int matrix(PyObject* t, PyObject* a, PyObject* b, Mat* m) {
  long long s0, s1;
  PyObject* v = PyObject_GetAttr(t, n_dtype);
  if (!v) return 0;
  Py_DECREF(v); /* (compared by identity only) */
  if (v != a && v != b) return 0;
  v = PyObject_GetAttr(t, n_is_cuda);
  if (!v) return 0;
  Py_DECREF(v);
  if (v != Py_True) return 0;
  if (!two(PyObject_GetAttr(t, n_shape), &m->rows, &m->cols)) return 0;
  if (m->rows < 1 || m->cols < 1 || m->rows > (1 << 30) || m->cols > (1 << 30)) return 0;
  if (!two(PyObject_CallMethodNoArgs(t, n_stride), &s0, &s1)) return 0;
  if (s1 != 1 && m->cols > 1) return 0;
  m->ld = m->rows > 1 ? s0 : (m->cols + 15) / 16 * 16;
  return m->ld != 0 && pointer(t, &m->ptr);
}

static int stream_of(PyObject* stream, void** p) {
  PyObject* v;
  if (stream == Py_None) {
    PyObject* d = PyObject_CallNoArgs(current_device);
    if (!d) return 0;
    v = PyObject_CallOneArg(current_stream, d);
    Py_DECREF(d);
  } else {
    v = PyObject_GetAttr(stream, n_cuda_stream);
  }
  if (!v) return 0;
  *p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

static PyObject* not_mine(void) {
  PyErr_Clear();
  Py_RETURN_NONE;
}

static int scales_fit(const Mat* s, long long rows, long long cols) {
  return s->rows == rows && s->cols == (cols + 127) / 128;
}

/* quantize(x, q, scales, stream) */
static PyObject* quantize(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Mat x, q, s;
  void* st;
  int code;
  (void)self;
  if (n != 4 || !call_quantize || !matrix(a[0], bf16, bf16, &x) || !matrix(a[1], f8, u8, &q) ||
      !matrix(a[2], f32, f32, &s) || q.rows != x.rows || q.cols != x.cols || !scales_fit(&s, x.rows, x.cols) ||
      !stream_of(a[3], &st))
    return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_quantize(x.ptr, x.ld, (int32_t)x.rows, (int32_t)x.cols, q.ptr, q.ld, (float*)s.ptr, s.ld, st);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* swiglu_quantize(gate, up, q, scales, stream) */
static PyObject* swiglu_quantize(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Mat g, u, q, s;
  void* st;
  int code;
  (void)self;
  if (n != 5 || !call_swiglu || !matrix(a[0], bf16, bf16, &g) || !matrix(a[1], bf16, bf16, &u) ||
      !matrix(a[2], f8, u8, &q) || !matrix(a[3], f32, f32, &s) || u.rows != g.rows || u.cols != g.cols ||
      u.ld != g.ld || q.rows != g.rows || q.cols != g.cols || !scales_fit(&s, g.rows, g.cols) || !stream_of(a[4], &st))
    return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_swiglu(g.ptr, u.ptr, g.ld, (int32_t)g.rows, (int32_t)g.cols, q.ptr, q.ld, (float*)s.ptr, s.ld, st);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* matmul(a, a_scales, b, b_scales, out, stream, status); the caller has checked status */
static PyObject* matmul(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Mat x, sx, w, sw, o;
  void *st, *status = NULL;
  int code;
  (void)self;
  if (n != 7 || !call_matmul || !matrix(a[0], f8, u8, &x) || !matrix(a[1], f32, f32, &sx) ||
      !matrix(a[2], f8, u8, &w) || !matrix(a[3], f32, f32, &sw) || !matrix(a[4], bf16, bf16, &o) ||
      w.cols != x.cols || o.rows != x.rows || o.cols != w.rows || !scales_fit(&sx, x.rows, x.cols) ||
      !scales_fit(&sw, (w.rows + 127) / 128, w.cols) || !stream_of(a[5], &st) ||
      (a[6] != Py_None && !pointer(a[6], &status)))
    return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_matmul(x.ptr, x.ld, (const float*)sx.ptr, sx.ld, w.ptr, w.ld, (const float*)sw.ptr, sw.ld, o.ptr, o.ld,
                     (int32_t)x.rows, (int32_t)w.rows, (int32_t)x.cols, (uint32_t*)status, st);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* ------------------------------------------------------------ around the expert products of a training step */
typedef int (*sort_fn)(const void*, int32_t, int32_t, int32_t, void*, void*, void*, void*, size_t, void*);
typedef int (*permute_fn)(int32_t, const void*, int64_t, int32_t, int32_t, const void*, int32_t, void*, int64_t, int32_t,
                          void*, void*);
typedef int (*unpermute_fn)(int32_t, const void*, int64_t, int32_t, int32_t, const void*, const void*, int32_t, int32_t,
                            void*, int64_t, void*, void*);
typedef int (*unpermute_backward_fn)(int32_t, const void*, int64_t, const void*, int64_t, const void*, const void*, int32_t,
                                     int32_t, int32_t, void*, int64_t, int32_t, void*, void*, void*);
typedef int (*swiglu_save_fn)(int32_t, const void*, const void*, int64_t, int32_t, int32_t, const void*, void*, int64_t,
                              void*, void*, int64_t, void*, void*, int64_t, void*);
typedef int (*swiglu_backward_fn)(int32_t, const void*, int64_t, const void*, const void*, int64_t, const void*, const void*,
                                  int64_t, int32_t, int32_t, const void*, void*, void*, int64_t, void*, int64_t, void*);
typedef int (*dequantize_fn)(int32_t, const void*, int64_t, const void*, int64_t, int32_t, int32_t, const void*, int32_t,
                             void*, int64_t, int32_t, void*, void*);
static sort_fn call_sort;
static permute_fn call_permute;
static unpermute_fn call_unpermute;
static unpermute_backward_fn call_unpermute_backward;
static swiglu_save_fn call_swiglu_save;
static swiglu_backward_fn call_swiglu_backward;
static dequantize_fn call_dequantize;
static PyObject *f16, *i32;
static PyObject* n_get_device;

/* The current device and the stream's raw handle. */
typedef struct {
  long device;
  void* stream;
} Where;

static int where(PyObject* stream, Where* w) {
  PyObject *v, *d = PyObject_CallNoArgs(current_device);
  if (!d) return 0;
  w->device = PyLong_AsLong(d);
  v = stream == Py_None ? PyObject_CallOneArg(current_stream, d) : PyObject_GetAttr(stream, n_cuda_stream);
  Py_DECREF(d);
  if (!v) return 0;
  w->stream = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

/* On the current device; its dtype (borrowed: compared by identity only). */
static PyObject* here(PyObject* t, const Where* w) {
  long device;
  PyObject *d, *v = PyObject_CallMethodNoArgs(t, n_get_device);
  if (!v) return NULL;
  device = PyLong_AsLong(v);
  Py_DECREF(v);
  if (device != w->device || PyErr_Occurred()) return NULL;
  d = PyObject_GetAttr(t, n_dtype);
  Py_XDECREF(d);
  return d;
}

/* A 2-D tensor there with contiguous columns, neither extent empty nor over
 * 2^30; returns its dtype.  (A single row's stride as in matrix.) */
static PyObject* rows_of(PyObject* t, const Where* w, Mat* m) {
  long long s0, s1;
  PyObject* d = here(t, w);
  if (!d || !two(PyObject_GetAttr(t, n_shape), &m->rows, &m->cols)) return NULL;
  if (m->rows < 1 || m->cols < 1 || m->rows > (1 << 30) || m->cols > (1 << 30)) return NULL;
  if (!two(PyObject_CallMethodNoArgs(t, n_stride), &s0, &s1)) return NULL;
  if (s1 != 1 && m->cols > 1) return NULL;
  m->ld = m->rows > 1 ? s0 : (m->cols + 15) / 16 * 16;
  return m->ld != 0 && pointer(t, &m->ptr) ? d : NULL;
}

/* The type's number, -1 for one that is none of bf16, fp16 and fp32. */
static int type_of(PyObject* d) { return d == NULL ? -1 : d == bf16 ? 0 : d == f16 ? 1 : d == f32 ? 2 : -1; }

/* A contiguous [rows, cols] tensor of dtype d (rows 0: any, written to m). */
static int dense(PyObject* t, const Where* w, PyObject* d, long long rows, long long cols, Mat* m) {
  return rows_of(t, w, m) == d && (rows == 0 || (m->rows == rows && m->cols == cols)) && (m->rows == 1 || m->ld == m->cols);
}
/* The same, or None. */
static int dense_or_none(PyObject* t, const Where* w, PyObject* d, long long rows, long long cols, Mat* m) {
  m->ptr = NULL;
  return t == Py_None || dense(t, w, d, rows, cols, m);
}
/* A contiguous tensor of one dimension (n 0: of any length, which is returned). */
static long long line(PyObject* t, const Where* w, PyObject* d, long long n, void** p) {
  PyObject *v, *dt = here(t, w);
  long long len = 0, stride = 0;
  if (!dt || (d && dt != d)) return 0;
  v = PyObject_GetAttr(t, n_shape);
  if (v && PyTuple_Check(v) && PyTuple_GET_SIZE(v) == 1) len = PyLong_AsLongLong(PyTuple_GET_ITEM(v, 0));
  Py_XDECREF(v);
  if (len < 1 || (n && len != n)) return 0;
  if (len > 1) {
    v = PyObject_CallMethodNoArgs(t, n_stride);
    if (v && PyTuple_Check(v) && PyTuple_GET_SIZE(v) == 1) stride = PyLong_AsLongLong(PyTuple_GET_ITEM(v, 0));
    Py_XDECREF(v);
    if (stride != 1) return 0;
  }
  return pointer(t, p) ? len : 0;
}
static int line_or_none(PyObject* t, const Where* w, PyObject* d, long long n, void** p) {
  *p = NULL;
  return t == Py_None || line(t, w, d, n, p) > 0;
}

/* sort(idx, n_experts, offsets, perm_dst, ws (bytes), perm_src, stream) */
static PyObject* sort(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Where w;
  Mat idx, perm;
  void *offsets, *src = NULL, *ws = NULL;
  long long bytes = 0;
  int code;
  long E;
  (void)self;
  if (n != 7 || !call_sort || !PyLong_Check(a[1]) || !where(a[6], &w) || !dense(a[0], &w, i32, 0, 0, &idx) ||
      !dense(a[3], &w, i32, idx.rows, idx.cols, &perm))
    return not_mine();
  E = PyLong_AsLong(a[1]);
  if (E < 1 || E > (1 << 30) || !line(a[2], &w, i32, E + 1, &offsets) ||
      !line_or_none(a[5], &w, i32, idx.rows * idx.cols, &src) ||
      (a[4] != Py_None && !(bytes = line(a[4], &w, u8, 0, &ws))))
    return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_sort(idx.ptr, (int32_t)idx.rows, (int32_t)idx.cols, (int32_t)E, offsets, perm.ptr, src, ws, (size_t)bytes,
                   w.stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* permute(x, perm_dst, x_perm, stream, status: None) */
static PyObject* permute(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Where w;
  Mat x, perm, y;
  PyObject* d;
  int code, type;
  (void)self;
  if (n != 5 || !call_permute || a[4] != Py_None || !where(a[3], &w) || !(d = rows_of(a[0], &w, &x)) ||
      !dense(a[1], &w, i32, 0, 0, &perm) || rows_of(a[2], &w, &y) != d || perm.rows != x.rows || y.cols != x.cols)
    return not_mine();
  type = d == f8 || d == u8 ? 3 : type_of(d);
  if (type < 0) return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_permute(type, x.ptr, x.ld, (int32_t)x.rows, (int32_t)x.cols, perm.ptr, (int32_t)perm.cols, y.ptr, y.ld,
                      (int32_t)y.rows, NULL, w.stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* unpermute(y_perm, w, perm_dst, out, stream, status: None) */
static PyObject* unpermute(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Where w;
  Mat y, wt, perm, out;
  PyObject* d;
  int code, type;
  (void)self;
  if (n != 6 || !call_unpermute || a[5] != Py_None || !where(a[4], &w) || !(d = rows_of(a[0], &w, &y)) ||
      (type = type_of(d)) < 0 || !dense(a[2], &w, i32, 0, 0, &perm) ||
      !dense_or_none(a[1], &w, f32, perm.rows, perm.cols, &wt) ||
      rows_of(a[3], &w, &out) != d || perm.rows != out.rows || y.cols != out.cols)
    return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_unpermute(type, y.ptr, y.ld, (int32_t)y.rows, (int32_t)y.cols, wt.ptr, perm.ptr, (int32_t)perm.rows,
                        (int32_t)perm.cols, out.ptr, out.ld, NULL, w.stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* unpermute_backward(d_out, y_perm, w, perm_dst, d_y_perm, d_w, stream, status: None); with all of its tensors but w */
static PyObject* unpermute_backward(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Where w;
  Mat g, y, wt, perm, dy, dw;
  PyObject* d;
  int code, type;
  (void)self;
  if (n != 8 || !call_unpermute_backward || a[7] != Py_None || !where(a[6], &w) || !(d = rows_of(a[0], &w, &g)) ||
      (type = type_of(d)) < 0 || rows_of(a[1], &w, &y) != d || !dense(a[3], &w, i32, 0, 0, &perm) ||
      !dense_or_none(a[2], &w, f32, perm.rows, perm.cols, &wt) || rows_of(a[4], &w, &dy) != d ||
      !dense(a[5], &w, f32, perm.rows, perm.cols, &dw) || perm.rows != g.rows || y.cols != g.cols || dy.cols != g.cols ||
      dy.rows != y.rows)
    return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_unpermute_backward(type, g.ptr, g.ld, y.ptr, y.ld, wt.ptr, perm.ptr, (int32_t)perm.rows, (int32_t)perm.cols,
                                 (int32_t)g.cols, dy.ptr, dy.ld, (int32_t)y.rows, dw.ptr, NULL, w.stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* Kept values and scales of gate and up: four tensors from a on, for rows x cols. */
static int kept(PyObject* const* a, const Where* w, long long rows, long long cols, Mat* q) {
  int i;
  for (i = 0; i < 4; ++i) {
    PyObject* d = rows_of(a[i], w, &q[i]);
    if (i & 1 ? d != f32 || !scales_fit(&q[i], rows, cols) : (d != f8 && d != u8) || q[i].rows != rows || q[i].cols != cols)
      return 0;
  }
  return q[0].ld == q[2].ld && q[1].ld == q[3].ld;
}
static int like(PyObject* t, const Where* w, PyObject* d, const Mat* of, Mat* m) {
  return rows_of(t, w, m) == d && m->rows == of->rows && m->cols == of->cols;
}

/* swiglu_save(gate, up, h, gate_q, gate_s, up_q, up_s, stream, n_rows) */
static PyObject* swiglu_save(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Where w;
  Mat g, u, h, q[4];
  void* rows;
  PyObject* d;
  int code, type;
  (void)self;
  if (n != 9 || !call_swiglu_save || !where(a[7], &w) || !(d = rows_of(a[0], &w, &g)) || (type = type_of(d)) < 0 ||
      !like(a[1], &w, d, &g, &u) || u.ld != g.ld || !like(a[2], &w, d, &g, &h) || !kept(a + 3, &w, g.rows, g.cols, q) ||
      !line_or_none(a[8], &w, i32, 1, &rows))
    return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_swiglu_save(type, g.ptr, u.ptr, g.ld, (int32_t)g.rows, (int32_t)g.cols, rows, h.ptr, h.ld, q[0].ptr, q[2].ptr,
                          q[0].ld, q[1].ptr, q[3].ptr, q[1].ld, w.stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* swiglu_backward(d_h, gate_q, gate_s, up_q, up_s, d_gate, d_up, h, stream, n_rows) */
static PyObject* swiglu_backward(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Where w;
  Mat g, dg, du, h, q[4];
  void* rows;
  PyObject* d;
  int code, type;
  (void)self;
  h.ptr = NULL;
  h.ld = 0;
  if (n != 10 || !call_swiglu_backward || !where(a[8], &w) || !(d = rows_of(a[0], &w, &g)) || (type = type_of(d)) < 0 ||
      !kept(a + 1, &w, g.rows, g.cols, q) || !like(a[5], &w, d, &g, &dg) || !like(a[6], &w, d, &g, &du) || dg.ld != du.ld ||
      (a[7] != Py_None && !like(a[7], &w, d, &g, &h)) || !line_or_none(a[9], &w, i32, 1, &rows))
    return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_swiglu_backward(type, g.ptr, g.ld, q[0].ptr, q[2].ptr, q[0].ld, q[1].ptr, q[3].ptr, q[1].ld, (int32_t)g.rows,
                              (int32_t)g.cols, rows, dg.ptr, du.ptr, dg.ld, h.ptr, h.ld, w.stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

/* dequantize(q, scales, x, perm_dst, stream, status: None) */
static PyObject* dequantize(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Where w;
  Mat q, s, x, perm;
  PyObject* d;
  int code, type;
  (void)self;
  if (n != 6 || !call_dequantize || a[5] != Py_None || !where(a[4], &w) || !(d = rows_of(a[0], &w, &q)) ||
      (d != f8 && d != u8) || rows_of(a[1], &w, &s) != f32 || !scales_fit(&s, q.rows, q.cols) ||
      (type = type_of(rows_of(a[2], &w, &x))) < 0 || x.cols != q.cols)
    return not_mine();
  perm.ptr = NULL;
  perm.cols = 1;
  if (a[3] == Py_None ? x.rows != q.rows : !dense(a[3], &w, i32, 0, 0, &perm) || perm.rows != q.rows) return not_mine();
  Py_BEGIN_ALLOW_THREADS;
  code = call_dequantize(type, q.ptr, q.ld, s.ptr, s.ld, (int32_t)q.rows, (int32_t)q.cols, perm.ptr, (int32_t)perm.cols, x.ptr,
                         x.ld, (int32_t)x.rows, NULL, w.stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

static void keep(PyObject** to, PyObject* v) {
  Py_INCREF(v);
  Py_XSETREF(*to, v);
}

/* bind(quantize, swiglu, matmul: addresses; bfloat16, float32, float8_e4m3fn, uint8; current_device, current_stream) */
static PyObject* bind(PyObject* self, PyObject* args) {
  PyObject *q, *s, *m, *o[6];
  (void)self;
  if (!PyArg_ParseTuple(args, "OOOOOOOOO", &q, &s, &m, &o[0], &o[1], &o[2], &o[3], &o[4], &o[5])) return NULL;
  call_quantize = (quantize_fn)(uintptr_t)PyLong_AsVoidPtr(q);
  call_swiglu = (swiglu_fn)(uintptr_t)PyLong_AsVoidPtr(s);
  call_matmul = (matmul_fn)(uintptr_t)PyLong_AsVoidPtr(m);
  if (PyErr_Occurred()) return NULL;
  keep(&bf16, o[0]);
  keep(&f32, o[1]);
  keep(&f8, o[2]);
  keep(&u8, o[3]);
  keep(&current_device, o[4]);
  keep(&current_stream, o[5]);
  Py_RETURN_NONE;
}

/* bind_rows(sort, permute, unpermute, unpermute_backward, swiglu_save, swiglu_backward, dequantize: addresses; float16,
 * int32), after bind */
static PyObject* bind_rows(PyObject* self, PyObject* args) {
  PyObject *p[7], *o[2];
  void* at[7];
  int i;
  (void)self;
  if (!PyArg_ParseTuple(args, "OOOOOOOOO", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &o[0], &o[1])) return NULL;
  for (i = 0; i < 7; ++i) at[i] = PyLong_AsVoidPtr(p[i]);
  if (PyErr_Occurred()) return NULL;
  call_sort = (sort_fn)(uintptr_t)at[0];
  call_permute = (permute_fn)(uintptr_t)at[1];
  call_unpermute = (unpermute_fn)(uintptr_t)at[2];
  call_unpermute_backward = (unpermute_backward_fn)(uintptr_t)at[3];
  call_swiglu_save = (swiglu_save_fn)(uintptr_t)at[4];
  call_swiglu_backward = (swiglu_backward_fn)(uintptr_t)at[5];
  call_dequantize = (dequantize_fn)(uintptr_t)at[6];
  keep(&f16, o[0]);
  keep(&i32, o[1]);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind_rows", bind_rows, METH_VARARGS, "The entry points around a training step's expert products."},
    {"sort", (PyCFunction)(void (*)(void))sort, METH_FASTCALL, "asap_moe_sort: its code, or None."},
    {"permute", (PyCFunction)(void (*)(void))permute, METH_FASTCALL, "asap_moe_permute: its code, or None."},
    {"unpermute", (PyCFunction)(void (*)(void))unpermute, METH_FASTCALL, "asap_moe_unpermute: its code, or None."},
    {"unpermute_backward", (PyCFunction)(void (*)(void))unpermute_backward, METH_FASTCALL,
     "asap_moe_unpermute_backward: its code, or None."},
    {"swiglu_save", (PyCFunction)(void (*)(void))swiglu_save, METH_FASTCALL, "asap_moe_swiglu_save: its code, or None."},
    {"swiglu_backward", (PyCFunction)(void (*)(void))swiglu_backward, METH_FASTCALL,
     "asap_moe_swiglu_backward: its code, or None."},
    {"dequantize", (PyCFunction)(void (*)(void))dequantize, METH_FASTCALL, "asap_moe_fp8_dequantize: its code, or None."},
    {"bind", bind, METH_VARARGS, "The library's entry points, the dtypes and the stream's getters."},
    {"quantize", (PyCFunction)(void (*)(void))quantize, METH_FASTCALL, "asap_moe_fp8_quantize: its code, or None."},
    {"swiglu_quantize", (PyCFunction)(void (*)(void))swiglu_quantize, METH_FASTCALL,
     "asap_moe_fp8_swiglu_quantize: its code, or None."},
    {"matmul", (PyCFunction)(void (*)(void))matmul, METH_FASTCALL, "asap_moe_fp8_matmul: its code, or None."},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the short calls.", -1,
                                    methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
  n_shape = PyUnicode_InternFromString("shape");
  n_dtype = PyUnicode_InternFromString("dtype");
  n_is_cuda = PyUnicode_InternFromString("is_cuda");
  n_stride = PyUnicode_InternFromString("stride");
  n_data_ptr = PyUnicode_InternFromString("data_ptr");
  n_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  n_get_device = PyUnicode_InternFromString("get_device");
  if (!n_get_device || !n_shape || !n_dtype || !n_is_cuda || !n_stride || !n_data_ptr || !n_cuda_stream) return NULL;
  return PyModule_Create(&module);
}
