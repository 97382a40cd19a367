/* Python face of the calls whose cost is the call: quantisation, its inverse and
 * the product of 4-bit operands, which for a single token run 2 to 5 us on the GPU.
 * Through ctypes such a call costs the host 4.1 us, half of it marshalling; here
 * about 2.7, the rest being the launch. Argument marshalling only, like the ctypes
 * binding beside it: every argument is checked here or by the library. Where the
 * buffers lie is checked here, because only here it is known: the library launches
 * on the current device and takes addresses at their word. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/ps_b200.h"

/* An operand's description; the Python class MxTensor derives from it and owns the buffers. */
typedef struct {
  PyObject_HEAD
  ps_mx mx;
  int device;                                                  /* of both buffers; -1: not on a GPU */
} Operand;

static PyTypeObject OperandType;
/* (of the CUDA runtime that the library is linked to; through torch the lookup takes a quarter of a microsecond) */
extern int cudaGetDevice(int* device);

static PyObject *g_f32, *g_bf16, *g_fail;                      /* torch dtypes; what raises PsError */
static PyObject *s_shape, *s_stride, *s_get_device, *s_data_ptr, *s_dtype, *s_cuda_stream;

static int operand_init(PyObject* self, PyObject* args, PyObject* kw) {
  static char* names[] = {"codes", "scales", "rows", "cols", "device", NULL};
  unsigned long long codes, scales;
  long long rows, cols;
  int device;
  if (!PyArg_ParseTupleAndKeywords(args, kw, "KKLLi", names, &codes, &scales, &rows, &cols, &device)) return -1;
  ps_mx* m = &((Operand*)self)->mx;
  m->codes = (void*)(size_t)codes;
  m->scales = (void*)(size_t)scales;
  m->rows = rows;
  m->cols = cols;
  ((Operand*)self)->device = device;
  return 0;
}

static PyObject* operand_rows(PyObject* self, void* unused) {
  (void)unused;
  return PyLong_FromLongLong(((Operand*)self)->mx.rows);
}
static PyObject* operand_cols(PyObject* self, void* unused) {
  (void)unused;
  return PyLong_FromLongLong(((Operand*)self)->mx.cols);
}
static PyObject* operand_ref(PyObject* self, void* unused) {
  (void)unused;
  return PyLong_FromVoidPtr(&((Operand*)self)->mx);
}

static PyGetSetDef operand_fields[] = {
    {"rows", operand_rows, NULL, "elements along the operand's first dimension", NULL},
    {"cols", operand_cols, NULL, "elements along its second, the one that blocks and products run along", NULL},
    {"ref", operand_ref, NULL, "address of the ps_mx", NULL},
    {NULL, NULL, NULL, NULL, NULL}};

static PyTypeObject OperandType = {
    PyVarObject_HEAD_INIT(NULL, 0).tp_name = "paper_2204_03211_b200._ops.Operand",
    .tp_basicsize = sizeof(Operand),
    .tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE,
    .tp_doc = "A ps_mx: addresses of codes and scales, rows, cols; and the device that both lie on (-1: none).",
    .tp_new = PyType_GenericNew,
    .tp_init = operand_init,
    .tp_getset = operand_fields,
};

/* Raises PsError through the binding; always returns NULL. */
static PyObject* fail(int status, const char* where, const char* detail) {
  PyObject* r = PyObject_CallFunction(g_fail, "isz", status, where, detail);
  if (r) {                                                     /* (it raises) */
    Py_DECREF(r);
    PyErr_SetString(PyExc_RuntimeError, where);
  }
  return NULL;
}

typedef struct {
  void* ptr;
  int dtype, device;
  long long rows, cols, ld;
} Matrix;

/* A 2-d CUDA tensor with contiguous rows.  0, or -1 with an exception set. */
static int matrix(PyObject* t, Matrix* m, const char* where) {
  PyObject *shape = NULL, *stride = NULL, *device = NULL, *ptr = NULL, *dtype = NULL;
  long long s0, s1;
  int ok = -1;
  shape = PyObject_GetAttr(t, s_shape);
  if (!shape) goto out;
  stride = PyObject_CallMethodNoArgs(t, s_stride);
  device = stride ? PyObject_CallMethodNoArgs(t, s_get_device) : NULL;
  ptr = device ? PyObject_CallMethodNoArgs(t, s_data_ptr) : NULL;
  dtype = ptr ? PyObject_GetAttr(t, s_dtype) : NULL;
  if (!dtype) goto out;
  m->device = (int)PyLong_AsLong(device);                      /* -1 for a tensor that is not on a GPU */
  if (PyErr_Occurred()) goto out;
  if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != 2 || !PyTuple_Check(stride) || m->device < 0) {
    fail(PS_ERR_BAD_ARG, where, "a 2-d CUDA tensor with contiguous rows is wanted");
    goto out;
  }
  m->rows = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0));
  m->cols = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 1));
  s0 = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 0));
  s1 = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 1));
  m->ptr = PyLong_AsVoidPtr(ptr);
  if (PyErr_Occurred()) goto out;
  if (s1 != 1 && m->cols > 1) {
    fail(PS_ERR_BAD_ARG, where, "a 2-d CUDA tensor with contiguous rows is wanted");
    goto out;
  }
  m->ld = m->rows > 1 ? s0 : m->cols;
  if (dtype == g_f32) {
    m->dtype = PS_F32;
  } else if (dtype == g_bf16) {
    m->dtype = PS_BF16;
  } else {
    fail(PS_ERR_BAD_ARG, where, "a float32 or bfloat16 tensor is wanted");
    goto out;
  }
  ok = 0;
out:
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  Py_XDECREF(device);
  Py_XDECREF(ptr);
  Py_XDECREF(dtype);
  return ok;
}

/* None (the legacy default stream), an address, or an object with a cuda_stream. */
static int stream_of(PyObject* o, void** out) {
  *out = NULL;
  if (!o || o == Py_None) return 0;
  if (PyLong_Check(o)) {
    *out = PyLong_AsVoidPtr(o);
  } else {
    PyObject* v = PyObject_GetAttr(o, s_cuda_stream);
    if (!v) return -1;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
  }
  return PyErr_Occurred() ? -1 : 0;
}

/* Sorts positional and keyword arguments into slots by name; missing ones stay NULL. */
static int arguments(const char* where, PyObject* const* args, Py_ssize_t n, PyObject* kwnames, const char* const* names,
                     int count, int required, PyObject** out) {
  if (n > count) {
    PyErr_Format(PyExc_TypeError, "%s takes at most %d arguments", where, count);
    return -1;
  }
  for (int i = 0; i < count; ++i) out[i] = i < n ? args[i] : NULL;
  const Py_ssize_t nk = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
  for (Py_ssize_t k = 0; k < nk; ++k) {
    PyObject* key = PyTuple_GET_ITEM(kwnames, k);
    int i = 0;
    while (i < count && PyUnicode_CompareWithASCIIString(key, names[i]) != 0) ++i;
    if (i == count || out[i]) {
      PyErr_Format(PyExc_TypeError, "%s: unexpected or repeated argument %R", where, key);
      return -1;
    }
    out[i] = args[n + k];
  }
  for (int i = 0; i < required; ++i)
    if (!out[i]) {
      PyErr_Format(PyExc_TypeError, "%s: argument '%s' is missing", where, names[i]);
      return -1;
    }
  return 0;
}

/* 0 if the matrix and the operands (NULL: none) lie on the current device, where the library launches; else -1 with an
 * exception set. */
static int placed(const Matrix* m, PyObject* a, PyObject* b, const char* where) {
  PyObject* const ops[] = {a, b};
  for (int i = 0; i < 2; ++i)
    if (ops[i] && ops[i] != Py_None && ((Operand*)ops[i])->device != m->device) {
      fail(PS_ERR_BAD_ARG, where, "the tensor and the operands are not all on one GPU");
      return -1;
    }
  int current = -1;
  if (cudaGetDevice(&current) || current != m->device) {
    fail(PS_ERR_BAD_ARG, where, "the tensor and the operands are not on the current device");
    return -1;
  }
  return 0;
}

/* NULL for None or a missing argument; sets *bad for what is no operand. */
static const ps_mx* operand(PyObject* o, int* bad, const char* where) {
  if (!o || o == Py_None) return NULL;
  if (!PyObject_TypeCheck(o, &OperandType)) {
    PyErr_Format(PyExc_TypeError, "%s: an MxTensor is wanted, not %R", where, (PyObject*)Py_TYPE(o));
    *bad = 1;
    return NULL;
  }
  return &((Operand*)o)->mx;
}

static PyObject* py_quantize(PyObject* self, PyObject* const* args, Py_ssize_t n, PyObject* kwnames) {
  static const char* const names[] = {"x", "q", "qt", "stream"};
  static const char where[] = "ps_mx_quantize";
  PyObject* a[4];
  Matrix x;
  void* stream;
  int bad = 0, rc;
  (void)self;
  if (arguments(where, args, n, kwnames, names, 4, 1, a)) return NULL;
  const ps_mx* q = operand(a[1], &bad, where);
  const ps_mx* qt = bad ? NULL : operand(a[2], &bad, where);
  if (bad || matrix(a[0], &x, where) || stream_of(a[3], &stream) || placed(&x, a[1], a[2], where)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = ps_mx_quantize(x.ptr, x.dtype, x.rows, x.cols, x.ld, q, qt, stream);
  Py_END_ALLOW_THREADS
  if (rc) return fail(rc, where, NULL);
  Py_RETURN_NONE;
}

static PyObject* py_dequantize(PyObject* self, PyObject* const* args, Py_ssize_t n, PyObject* kwnames) {
  static const char* const names[] = {"q", "out", "stream"};
  static const char where[] = "ps_mx_dequantize";
  PyObject* a[3];
  Matrix o;
  void* stream;
  int bad = 0, rc;
  (void)self;
  if (arguments(where, args, n, kwnames, names, 3, 2, a)) return NULL;
  const ps_mx* q = operand(a[0], &bad, where);
  if (bad || matrix(a[1], &o, where) || stream_of(a[2], &stream)) return NULL;
  if (!q || o.rows != q->rows || o.cols != q->cols) return fail(PS_ERR_BAD_ARG, where, "out and the operand differ in shape");
  if (placed(&o, a[0], NULL, where)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = ps_mx_dequantize(q, o.dtype, o.ptr, o.ld, stream);
  Py_END_ALLOW_THREADS
  if (rc) return fail(rc, where, NULL);
  Py_INCREF(a[1]);
  return a[1];
}

static PyObject* py_matmul(PyObject* self, PyObject* const* args, Py_ssize_t n, PyObject* kwnames) {
  static const char* const names[] = {"a", "b", "out", "stream"};
  static const char where[] = "ps_mx_matmul";
  PyObject* v[4];
  Matrix o;
  void* stream;
  int bad = 0, rc;
  (void)self;
  if (arguments(where, args, n, kwnames, names, 4, 3, v)) return NULL;
  const ps_mx* a = operand(v[0], &bad, where);
  const ps_mx* b = bad ? NULL : operand(v[1], &bad, where);
  if (bad || matrix(v[2], &o, where) || stream_of(v[3], &stream)) return NULL;
  if (!a || !b || o.rows != a->rows || o.cols != b->rows)
    return fail(PS_ERR_BAD_ARG, where, "out is not of the product's shape");
  if (placed(&o, v[0], v[1], where)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = ps_mx_matmul(a, b, o.dtype, o.ptr, o.ld, stream);
  Py_END_ALLOW_THREADS
  if (rc) return fail(rc, where, NULL);
  Py_INCREF(v[2]);
  return v[2];
}

/* setup(float32, bfloat16, raiser): the objects that the calls compare with and report through. */
static PyObject* py_setup(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "setup(float32, bfloat16, raiser)");
    return NULL;
  }
  Py_XSETREF(g_f32, Py_NewRef(args[0]));
  Py_XSETREF(g_bf16, Py_NewRef(args[1]));
  Py_XSETREF(g_fail, Py_NewRef(args[2]));
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"ps_mx_quantize", (PyCFunction)(void (*)(void))py_quantize, METH_FASTCALL | METH_KEYWORDS,
     "ps_mx_quantize(x, q=None, qt=None, stream=None)\n\nQuantises the device matrix x (float32 or bfloat16, any row stride)\n"
     "along its rows into q and / or along its columns into qt (the operand of x's transpose)."},
    {"ps_mx_dequantize", (PyCFunction)(void (*)(void))py_dequantize, METH_FASTCALL | METH_KEYWORDS,
     "ps_mx_dequantize(q, out, stream=None)\n\nWrites the values q stands for to the device matrix out, which it returns."},
    {"ps_mx_matmul", (PyCFunction)(void (*)(void))py_matmul, METH_FASTCALL | METH_KEYWORDS,
     "ps_mx_matmul(a, b, out, stream=None)\n\nout[m][n] = sum over k of a[m][k] * b[n][k]; returns out (float32 or\n"
     "bfloat16, any row stride)."},
    {"setup", (PyCFunction)(void (*)(void))py_setup, METH_FASTCALL, "setup(float32, bfloat16, raiser)"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops", "Calls on 4-bit operands.", -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__ops(void) {
  static const char* const texts[] = {"shape", "stride", "get_device", "data_ptr", "dtype", "cuda_stream"};
  PyObject** const slots[] = {&s_shape, &s_stride, &s_get_device, &s_data_ptr, &s_dtype, &s_cuda_stream};
  for (int i = 0; i < 6; ++i)
    if (!(*slots[i] = PyUnicode_InternFromString(texts[i]))) return NULL;
  if (PyType_Ready(&OperandType) < 0) return NULL;
  PyObject* m = PyModule_Create(&module);
  if (!m) return NULL;
  Py_INCREF(&OperandType);
  if (PyModule_AddObject(m, "Operand", (PyObject*)&OperandType) < 0) {
    Py_DECREF(&OperandType);
    Py_DECREF(m);
    return NULL;
  }
  return m;
}
