/* Python entry of the calls that are made many times per step: mfet_grad_clip, mfet_rows_write, mfet_rows_read,
 * mfet_mx4_quantize, mfet_mx4_matmul, mfet_mx4_linear, mfet_layer_norm, mfet_layer_norm_backward, mfet_gated_linear,
 * mfet_gated_linear_backward and mfet_orthogonalize, argument for argument as in mfet.h, without the per-argument
 * cost of ctypes (17 arguments: 3.0 us there, 0.5 us here; the kernels of a small call take as long). Marshalling only: an argument that
 * is an address may be a tensor (its data_ptr() is taken), an int or None. The addresses of the functions come from the library that the
 * binding has loaded. A status other than MFET_OK goes to the binding's error function, which raises. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/mfet.h"

typedef int (*grad_clip_fn)(const mfet_grad_t*, int32_t, float, float*, void*, uint64_t, mfet_stream_t);
typedef int (*rows_fn)(const mfet_table_desc_t*, const int64_t*, int64_t, const int64_t*, void*, uint32_t, int64_t, uint32_t*,
                       mfet_stream_t);
typedef int (*quantize_fn)(const void*, uint32_t, int64_t, int64_t, int64_t, void*, void*, mfet_stream_t);
typedef int (*matmul_fn)(const void*, const void*, int64_t, const void*, const void*, int64_t, int64_t, const float*, uint32_t, void*,
                         uint32_t, int64_t, uint32_t*, mfet_stream_t);
typedef int (*linear_fn)(const void*, uint32_t, int64_t, int64_t, const void*, const void*, int64_t, int64_t, const float*, uint32_t,
                         void*, uint32_t, int64_t, void*, uint64_t, uint32_t*, mfet_stream_t);

typedef int (*norm_fn)(const void*, uint32_t, int64_t, int64_t, int64_t, const float*, const float*, float, void*, uint32_t, int64_t,
                       mfet_stream_t);
typedef int (*norm_back_fn)(const void*, uint32_t, int64_t, int64_t, int64_t, const float*, float, const void*, uint32_t, int64_t, void*,
                            int64_t, float*, float*, void*, uint64_t, mfet_stream_t);
typedef int (*gated_fn)(const void*, uint32_t, int64_t, int64_t, const void*, int64_t, const void*, int64_t, int64_t, int64_t, uint32_t,
                        void*, int64_t, void*, uint64_t, uint32_t*, mfet_stream_t);
typedef int (*gated_back_fn)(const void*, uint32_t, int64_t, int64_t, const void*, int64_t, const void*, int64_t, int64_t, int64_t,
                             uint32_t, const void*, int64_t, void*, int64_t, void*, int64_t, void*, int64_t, void*, uint64_t, uint32_t*,
                             mfet_stream_t);
typedef int (*orthogonalize_fn)(const void*, uint32_t, int64_t, int64_t, int64_t, const float*, int32_t, float, void*, uint32_t, int64_t,
                                void*, uint64_t, uint32_t*, mfet_stream_t);

static struct {
  grad_clip_fn grad_clip;
  rows_fn rows_write, rows_read;
  quantize_fn quantize;
  matmul_fn matmul;
  linear_fn linear;
  norm_fn norm;
  norm_back_fn norm_back;
  gated_fn gated;
  gated_back_fn gated_back;
  orthogonalize_fn orthogonalize;
} lib;
static PyObject *fail, *data_ptr;

/* The n arguments of `name`, of which the last may be left out down to `least`: kinds p = address, i = integer (u: of 32 bits
 * without a sign, d: with one, z: not negative; another value is MFET_ERR_INVALID_ARG), f = float, b = an object that lends its memory
 * (a ctypes structure or array; `bytes` is its length), o = any object. */
typedef struct {
  union {
    long long i;
    void* p;
    double f;
  };
  Py_ssize_t bytes;
} arg_t;

static int address(PyObject* o, void** p) {
  if (o == Py_None) {
    *p = NULL;
    return 1;
  }
  PyObject* v = o;
  if (!PyLong_Check(o)) {
    v = PyObject_CallMethodNoArgs(o, data_ptr);
    if (!v) return 0;
  }
  *p = (void*)(uintptr_t)PyLong_AsUnsignedLongLong(v);
  const int ok = !PyErr_Occurred();
  if (v != o) Py_DECREF(v);
  return ok;
}

static PyObject* done(int status, const char* name) {
  if (status == MFET_OK) Py_RETURN_NONE;
  PyObject* r = PyObject_CallFunction(fail, "is", status, name);
  if (r) {
    Py_DECREF(r);
    PyErr_Format(PyExc_RuntimeError, "%s: status %d", name, status);
  }
  return NULL;
}

static int parse(const char* name, const char* kinds, Py_ssize_t least, PyObject* const* args, Py_ssize_t n, arg_t* a) {
  const Py_ssize_t most = (Py_ssize_t)strlen(kinds);
  if (n < least || n > most) {
    PyErr_Format(PyExc_TypeError, "%s takes %zd to %zd arguments (%zd given)", name, least, most, n);
    return 0;
  }
  memset(a, 0, sizeof(arg_t) * (size_t)most);
  for (Py_ssize_t k = 0; k < n; ++k) {
    switch (kinds[k]) {
      case 'p':
        if (!address(args[k], &a[k].p)) return 0;
        break;
      case 'f':
        a[k].f = PyFloat_AsDouble(args[k]);
        if (a[k].f == -1.0 && PyErr_Occurred()) return 0;
        break;
      case 'b':
        if (args[k] == Py_None) {
          a[k].p = NULL;
        } else {
          Py_buffer view; /* the caller's reference keeps the memory for the length of the call */
          if (PyObject_GetBuffer(args[k], &view, PyBUF_SIMPLE) != 0) return 0;
          a[k].p = view.buf;
          a[k].bytes = view.len;
          PyBuffer_Release(&view);
        }
        break;
      case 'o': /* looked at by the caller */
        break;
      default:
        a[k].i = PyLong_AsLongLong(args[k]);
        if (a[k].i == -1 && PyErr_Occurred()) return 0;
        if ((kinds[k] == 'u' && (a[k].i < 0 || a[k].i > (long long)UINT32_MAX)) ||
            (kinds[k] == 'd' && (a[k].i < INT32_MIN || a[k].i > INT32_MAX)) || (kinds[k] == 'z' && a[k].i < 0)) {
          done(MFET_ERR_INVALID_ARG, name);
          return 0;
        }
    }
  }
  return 1;
}

#define RUN(call)          \
  int status;              \
  Py_BEGIN_ALLOW_THREADS;  \
  status = (call);         \
  Py_END_ALLOW_THREADS

static PyObject* py_grad_clip(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_grad_clip";
  arg_t a[6];
  if (!parse(name, "ofppzp", 5, args, n, a)) return NULL;
  PyObject* list = args[0];
  arg_t g[2];
  if (!PyTuple_Check(list) || !parse(name, "bd", 2, &PyTuple_GET_ITEM(list, 0), PyTuple_GET_SIZE(list), g)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "mfet_grad_clip: what make_grads gave is wanted");
    return NULL;
  }
  /* a list that is shorter than it says */
  if (g[0].p && g[1].i > g[0].bytes / (Py_ssize_t)sizeof(mfet_grad_t)) return done(MFET_ERR_INVALID_ARG, name);
  RUN(lib.grad_clip((const mfet_grad_t*)g[0].p, (int32_t)g[1].i, (float)a[1].f, (float*)a[2].p, a[3].p, (uint64_t)a[4].i, a[5].p));
  return done(status, name);
}

static PyObject* rows(rows_fn f, const char* name, PyObject* const* args, Py_ssize_t n) {
  arg_t a[9];
  if (!parse(name, "bpippuipp", 7, args, n, a)) return NULL;
  if (a[0].p && a[0].bytes < (Py_ssize_t)sizeof(mfet_table_desc_t)) return done(MFET_ERR_INVALID_ARG, name);
  RUN(f((const mfet_table_desc_t*)a[0].p, (const int64_t*)a[1].p, a[2].i, (const int64_t*)a[3].p, a[4].p, (uint32_t)a[5].i, a[6].i,
        (uint32_t*)a[7].p, a[8].p));
  return done(status, name);
}
static PyObject* py_rows_write(PyObject* self, PyObject* const* args, Py_ssize_t n) { return rows(lib.rows_write, "mfet_rows_write", args, n); }
static PyObject* py_rows_read(PyObject* self, PyObject* const* args, Py_ssize_t n) { return rows(lib.rows_read, "mfet_rows_read", args, n); }

static PyObject* py_quantize(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_mx4_quantize";
  arg_t a[8];
  if (!parse(name, "puiiippp", 7, args, n, a)) return NULL;
  RUN(lib.quantize(a[0].p, (uint32_t)a[1].i, a[2].i, a[3].i, a[4].i, a[5].p, a[6].p, a[7].p));
  return done(status, name);
}

static PyObject* py_matmul(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_mx4_matmul";
  arg_t a[14];
  if (!parse(name, "ppippiipupuipp", 12, args, n, a)) return NULL;
  RUN(lib.matmul(a[0].p, a[1].p, a[2].i, a[3].p, a[4].p, a[5].i, a[6].i, (const float*)a[7].p, (uint32_t)a[8].i, a[9].p,
                 (uint32_t)a[10].i, a[11].i, (uint32_t*)a[12].p, a[13].p));
  return done(status, name);
}

static PyObject* py_linear(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_mx4_linear";
  arg_t a[17];
  if (!parse(name, "puiippiipupuipzpp", 15, args, n, a)) return NULL;
  RUN(lib.linear(a[0].p, (uint32_t)a[1].i, a[2].i, a[3].i, a[4].p, a[5].p, a[6].i, a[7].i, (const float*)a[8].p, (uint32_t)a[9].i,
                 a[10].p, (uint32_t)a[11].i, a[12].i, a[13].p, (uint64_t)a[14].i, (uint32_t*)a[15].p, a[16].p));
  return done(status, name);
}

static PyObject* py_norm(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_layer_norm";
  arg_t a[12];
  if (!parse(name, "puiiippfpuip", 11, args, n, a)) return NULL;
  RUN(lib.norm(a[0].p, (uint32_t)a[1].i, a[2].i, a[3].i, a[4].i, (const float*)a[5].p, (const float*)a[6].p, (float)a[7].f, a[8].p,
               (uint32_t)a[9].i, a[10].i, a[11].p));
  return done(status, name);
}

static PyObject* py_norm_back(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_layer_norm_backward";
  arg_t a[17];
  if (!parse(name, "puiiipfpuipipppzp", 16, args, n, a)) return NULL;
  RUN(lib.norm_back(a[0].p, (uint32_t)a[1].i, a[2].i, a[3].i, a[4].i, (const float*)a[5].p, (float)a[6].f, a[7].p, (uint32_t)a[8].i,
                    a[9].i, a[10].p, a[11].i, (float*)a[12].p, (float*)a[13].p, a[14].p, (uint64_t)a[15].i, a[16].p));
  return done(status, name);
}

static PyObject* py_gated(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_gated_linear";
  arg_t a[17];
  if (!parse(name, "puiipipiiiupipzpp", 15, args, n, a)) return NULL;
  RUN(lib.gated(a[0].p, (uint32_t)a[1].i, a[2].i, a[3].i, a[4].p, a[5].i, a[6].p, a[7].i, a[8].i, a[9].i, (uint32_t)a[10].i, a[11].p,
                a[12].i, a[13].p, (uint64_t)a[14].i, (uint32_t*)a[15].p, a[16].p));
  return done(status, name);
}

static PyObject* py_gated_back(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_gated_linear_backward";
  arg_t a[23];
  if (!parse(name, "puiipipiiiupipipipipzpp", 21, args, n, a)) return NULL;
  RUN(lib.gated_back(a[0].p, (uint32_t)a[1].i, a[2].i, a[3].i, a[4].p, a[5].i, a[6].p, a[7].i, a[8].i, a[9].i, (uint32_t)a[10].i, a[11].p,
                     a[12].i, a[13].p, a[14].i, a[15].p, a[16].i, a[17].p, a[18].i, a[19].p, (uint64_t)a[20].i, (uint32_t*)a[21].p,
                     a[22].p));
  return done(status, name);
}

static PyObject* py_orthogonalize(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  static const char name[] = "mfet_orthogonalize";
  arg_t a[15];
  if (!parse(name, "puiiipdfpuipzpp", 13, args, n, a)) return NULL;
  RUN(lib.orthogonalize(a[0].p, (uint32_t)a[1].i, a[2].i, a[3].i, a[4].i, (const float*)a[5].p, (int32_t)a[6].i, (float)a[7].f, a[8].p,
                        (uint32_t)a[9].i, a[10].i, a[11].p, (uint64_t)a[12].i, (uint32_t*)a[13].p, a[14].p));
  return done(status, name);
}

/* bind(fail, grad_clip, rows_write, ..., orthogonalize): the error function and the library's addresses, in the order of `lib` */
static PyObject* py_bind(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  if (n != 12) {
    PyErr_SetString(PyExc_TypeError, "bind takes 12 arguments");
    return NULL;
  }
  void* p[11];
  for (int k = 0; k < 11; ++k)
    if (!address(args[k + 1], &p[k])) return NULL;
  lib.grad_clip = (grad_clip_fn)p[0];
  lib.rows_write = (rows_fn)p[1];
  lib.rows_read = (rows_fn)p[2];
  lib.quantize = (quantize_fn)p[3];
  lib.matmul = (matmul_fn)p[4];
  lib.linear = (linear_fn)p[5];
  lib.norm = (norm_fn)p[6];
  lib.norm_back = (norm_back_fn)p[7];
  lib.gated = (gated_fn)p[8];
  lib.gated_back = (gated_back_fn)p[9];
  lib.orthogonalize = (orthogonalize_fn)p[10];
  Py_INCREF(args[0]);
  Py_XSETREF(fail, args[0]);
  Py_RETURN_NONE;
}

#define METHOD(name, f, doc) {name, (PyCFunction)(void (*)(void))f, METH_FASTCALL, doc}
static PyMethodDef methods[] = {
    METHOD("bind", py_bind, NULL),
    METHOD("mfet_grad_clip", py_grad_clip,
           "mfet_grad_clip(grads, max_norm, norm, scratch, scratch_bytes, stream=None)\n\ngrads: what make_grads gave."),
    METHOD("mfet_rows_write", py_rows_write,
           "mfet_rows_write(table, rows, n, n_dev, values, dtype, ld, status=None, stream=None)\n\ntable: a TableDesc."),
    METHOD("mfet_rows_read", py_rows_read,
           "mfet_rows_read(table, rows, n, n_dev, values, dtype, ld, status=None, stream=None)\n\ntable: a TableDesc."),
    METHOD("mfet_mx4_quantize", py_quantize, "mfet_mx4_quantize(x, dtype, ld, rows, k, codes, scales, stream=None)"),
    METHOD("mfet_mx4_matmul", py_matmul,
           "mfet_mx4_matmul(a_codes, a_scales, m, w_codes, w_scales, n, k, bias, act, y, y_dtype, y_ld, status=None, stream=None)"),
    METHOD("mfet_mx4_linear", py_linear,
           "mfet_mx4_linear(x, x_dtype, x_ld, m, w_codes, w_scales, n, k, bias, act, y, y_dtype, y_ld, scratch, scratch_bytes,\n"
           "                status=None, stream=None)"),
    METHOD("mfet_layer_norm", py_norm, "mfet_layer_norm(x, x_dtype, x_ld, rows, cols, weight, bias, eps, y, y_dtype, y_ld, stream=None)"),
    METHOD("mfet_layer_norm_backward", py_norm_back,
           "mfet_layer_norm_backward(x, x_dtype, x_ld, rows, cols, weight, eps, dy, dy_dtype, dy_ld, dx, dx_ld, dweight, dbias, scratch,\n"
           "                         scratch_bytes, stream=None)"),
    METHOD("mfet_gated_linear", py_gated,
           "mfet_gated_linear(x, dtype, x_ld, m, w_gate, wg_ld, w_up, wu_ld, n, k, act, h, h_ld, scratch, scratch_bytes,\n"
           "                  status=None, stream=None)"),
    METHOD("mfet_gated_linear_backward", py_gated_back,
           "mfet_gated_linear_backward(x, dtype, x_ld, m, w_gate, wg_ld, w_up, wu_ld, n, k, act, dh, dh_ld, dx, dx_ld, dw_gate, dwg_ld,\n"
           "                           dw_up, dwu_ld, scratch, scratch_bytes, status=None, stream=None)"),
    METHOD("mfet_orthogonalize", py_orthogonalize,
           "mfet_orthogonalize(g, dtype, ld, rows, cols, coefficients, steps, scale, out, out_dtype, out_ld, scratch, scratch_bytes,\n"
           "                   status=None, stream=None)\n\ncoefficients: an address, or None."),
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fastcall(void) {
  data_ptr = PyUnicode_InternFromString("data_ptr");
  return data_ptr ? PyModule_Create(&module) : NULL;
}
