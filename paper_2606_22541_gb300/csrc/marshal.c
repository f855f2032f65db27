/* Argument marshalling of the calls that are short enough for it to count: the
 * e4m3 operators on plain tensors.  A Python wrapper spends 2.5 to 4 us on
 * attributes, checks and ctypes conversions, more than the launch itself (2.5
 * us); this takes about 1.
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

static PyMethodDef methods[] = {
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
  if (!n_shape || !n_dtype || !n_is_cuda || !n_stride || !n_data_ptr || !n_cuda_stream) return NULL;
  return PyModule_Create(&module);
}
