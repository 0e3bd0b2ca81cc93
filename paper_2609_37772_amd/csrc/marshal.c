/* Argument checks of the calls that a decoding step makes once per token and layer, in
 * C: the same as _binding.py's, for the usual case only (dense tensors of the expected
 * type, size and device).  Anything else, an error included, is answered with None, and
 * the caller takes the long way, which names what is wrong.  A call's checks took 1.9
 * of its 5.5 us in Python and half of a microsecond here.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

static PyObject *tensor_type, *f32, *bf16, *i32;
static PyObject *s_dtype, *s_shape, *s_is_contiguous, *s_get_device, *s_data_ptr;

typedef struct {
  PyObject *kind; /* dtype; only ever compared */
  int64_t size[3];
  void *data;
} Tensor;

/* Whether t is a dense tensor of `dims` dimensions on `device`. */
static int look(PyObject *t, int dims, long device, Tensor *out) {
  if ((PyObject *)Py_TYPE(t) != tensor_type) return 0;
  PyObject *o = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  if (!o) return 0;
  int ok = o == Py_True;
  Py_DECREF(o);
  if (!ok || !(o = PyObject_CallMethodNoArgs(t, s_get_device))) return 0;
  ok = PyLong_Check(o) && PyLong_AsLong(o) == device;
  Py_DECREF(o);
  if (!ok || !(o = PyObject_GetAttr(t, s_dtype))) return 0;
  out->kind = o;
  Py_DECREF(o); /* torch keeps its dtypes */
  if (!(o = PyObject_GetAttr(t, s_shape))) return 0;
  ok = PyTuple_Check(o) && PyTuple_GET_SIZE(o) == dims;
  for (int i = 0; ok && i < dims; ++i) {
    out->size[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
    ok = out->size[i] >= 0 && out->size[i] <= INT32_MAX;
  }
  Py_DECREF(o);
  if (!ok || !(o = PyObject_CallMethodNoArgs(t, s_data_ptr))) return 0;
  out->data = PyLong_AsVoidPtr(o);
  Py_DECREF(o);
  return !PyErr_Occurred();
}

/* An optional int32 tensor of n entries. */
static int look_ints(PyObject *t, int64_t n, long device, void **data) {
  Tensor x;
  *data = NULL;
  if (t == Py_None) return 1;
  if (!look(t, 1, device, &x) || x.kind != i32 || x.size[0] != n) return 0;
  *data = x.data;
  return 1;
}

/* What both calls look at alike: two tensors of rows, page table, lengths, positions. */
typedef struct {
  void *fn, *kv, *lens, *positions;
  Tensor a, b, table;
  long layer, heads, dim, device;
  int dtype; /* as in uad.h */
} Call;

static int look_call(PyObject *fn, PyObject *kv, PyObject *layer, PyObject *a, PyObject *b, PyObject *table, PyObject *lens,
                     PyObject *positions, PyObject *heads, PyObject *dim, PyObject *device, Call *c) {
  if (!PyLong_Check(fn) || !PyLong_Check(kv) || !PyLong_Check(layer)) return 0;
  c->fn = PyLong_AsVoidPtr(fn);
  c->kv = PyLong_AsVoidPtr(kv);
  c->layer = PyLong_AsLong(layer);
  c->heads = PyLong_AsLong(heads);
  c->dim = PyLong_AsLong(dim);
  c->device = PyLong_AsLong(device);
  if (PyErr_Occurred() || !c->fn || !c->kv || c->layer < INT32_MIN || c->layer > INT32_MAX) return 0;
  if (!look(a, 3, c->device, &c->a) || !look(b, 3, c->device, &c->b) || !look(table, 2, c->device, &c->table)) return 0;
  if (c->a.kind != c->b.kind || (c->a.kind != f32 && c->a.kind != bf16) || c->table.kind != i32) return 0;
  c->dtype = c->a.kind == bf16;
  for (int i = 0; i < 3; ++i)
    if (c->a.size[i] != c->b.size[i]) return 0;
  if (c->a.size[1] != c->heads || c->a.size[2] != c->dim) return 0;
  return lens != Py_None && look_ints(lens, c->table.size[0], c->device, &c->lens) &&
         look_ints(positions, c->a.size[0], c->device, &c->positions);
}

static PyObject *long_way(void) {
  PyErr_Clear();
  Py_RETURN_NONE;
}

typedef int32_t (*append_fn)(void *, int32_t, const void *, const void *, int32_t, int64_t, int64_t, int32_t, const void *,
                             const void *, const void *, const void *, int32_t, int32_t);
typedef int32_t (*attend_fn)(void *, int32_t, const void *, void *, int32_t, int64_t, int64_t, const void *, const void *,
                             const void *, int32_t, int32_t, float);

/* append(uad_kv_append, kv, layer, k, v, page_table, lens, row_start, positions, heads, dim, device) */
static PyObject *append(PyObject *self, PyObject *const *x, Py_ssize_t n) {
  Call c;
  void *row_start;
  int32_t st;
  (void)self;
  if (n != 12 || !look_call(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[8], x[9], x[10], x[11], &c) ||
      !look_ints(x[7], c.table.size[0] + 1, c.device, &row_start))
    return long_way();
  const int64_t row = (int64_t)c.heads * c.dim;
  Py_BEGIN_ALLOW_THREADS
  st = ((append_fn)c.fn)(c.kv, (int32_t)c.layer, c.a.data, c.b.data, c.dtype, row, row, (int32_t)c.a.size[0], row_start, c.lens,
                         c.positions, c.table.data, (int32_t)c.table.size[1], (int32_t)c.table.size[0]);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* attend(uad_kv_attend, kv, layer, q, out, page_table, lens, positions, scale, heads, dim, device) */
static PyObject *attend(PyObject *self, PyObject *const *x, Py_ssize_t n) {
  Call c;
  int32_t st;
  (void)self;
  if (n != 12 || !look_call(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7], x[9], x[10], x[11], &c) ||
      c.a.size[0] != c.table.size[0] || !PyFloat_Check(x[8]))
    return long_way();
  const float scale = (float)PyFloat_AS_DOUBLE(x[8]);
  const int64_t row = (int64_t)c.heads * c.dim;
  Py_BEGIN_ALLOW_THREADS
  st = ((attend_fn)c.fn)(c.kv, (int32_t)c.layer, c.a.data, c.b.data, c.dtype, row, row, c.lens, c.positions, c.table.data,
                         (int32_t)c.table.size[1], (int32_t)c.table.size[0], scale);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* setup(torch.Tensor, torch.float32, torch.bfloat16, torch.int32): kept for good */
static PyObject *setup(PyObject *self, PyObject *const *x, Py_ssize_t n) {
  (void)self;
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "setup(Tensor, float32, bfloat16, int32)");
    return NULL;
  }
  PyObject **keep[4] = {&tensor_type, &f32, &bf16, &i32};
  for (int i = 0; i < 4; ++i) {
    Py_INCREF(x[i]);
    Py_XSETREF(*keep[i], x[i]);
  }
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, NULL},
                                {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, NULL},
                                {"setup", (PyCFunction)(void (*)(void))setup, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
  struct {
    PyObject **to;
    const char *text;
  } names[] = {{&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_is_contiguous, "is_contiguous"}, {&s_get_device, "get_device"},
               {&s_data_ptr, "data_ptr"}};
  for (size_t i = 0; i < sizeof names / sizeof *names; ++i)
    if (!*names[i].to && !(*names[i].to = PyUnicode_InternFromString(names[i].text))) return NULL;
  return PyModule_Create(&module);
}
