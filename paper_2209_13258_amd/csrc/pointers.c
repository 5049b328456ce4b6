/* Looks at tensors and their addresses, many in one go, and whole calls, for binding.py.
 *
 * What makes a tensor safe to hand on is its length, type, device and that it is contiguous.  Asked from Python, each question to each tensor costs
 * 50 ns, which makes a call with 8 shards 2 us longer and one with 64 12 us, more than the kernels of a small call take.  PyTorch's tensors offer all
 * of it at once by DLPack's exchange from C (version 1: the structures below, and the type's attribute that holds them); a list that holds anything
 * else, or anything that does not fit, is left to Python, which says what is wrong with it. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "osdp.h"

typedef struct {
  void *data;
  int32_t device_type, device;
  int32_t dims;
  uint8_t code, bits; /* of an element's type */
  uint16_t lanes;
  int64_t *shape, *strides;
  uint64_t offset;
} View;

typedef struct {
  uint32_t major, minor;
  void *before;                         /* an older version */
  void *allocate, *from_py, *to_py;     /* (not used here) */
  int (*view)(void *tensor, View *out); /* of memory that the tensor keeps */
  void *stream;
} Exchange;

enum { kCuda = 2, kRocm = 10 };

/* The exchange of a tensor's type, or NULL. */
static const Exchange *exchange_of(PyObject *t) {
  PyObject *capsule = PyObject_GetAttrString((PyObject *)Py_TYPE(t), "__dlpack_c_exchange_api__");
  if (!capsule) return NULL;
  const Exchange *x = PyCapsule_GetPointer(capsule, "dlpack_exchange_api"); /* (outlives the capsule) */
  Py_DECREF(capsule);
  return x && x->major == 1 && x->view ? x : NULL;
}

/* Whether the tensor is as asked for; its address. */
static int look(const Exchange *x, PyObject *t, int64_t bytes, const uint8_t *kinds, Py_ssize_t kinds_bytes, int64_t device, uint64_t *address) {
  View v;
  if (x->view(t, &v) != 0) return 0;
  if ((v.device_type != kCuda && v.device_type != kRocm) || v.device != device || v.lanes != 1) return 0;
  Py_ssize_t k = 0;
  while (k + 1 < kinds_bytes && (kinds[k] != v.code || kinds[k + 1] != v.bits)) k += 2;
  if (k + 1 >= kinds_bytes) return 0;
  int64_t n = 1;
  for (int32_t d = v.dims - 1; d >= 0; --d) {
    if (v.shape[d] != 1 && v.strides && v.strides[d] != n) return 0;
    n *= v.shape[d];
  }
  *address = (uint64_t)(uintptr_t)v.data + v.offset;
  return n * (v.bits / 8) >= bytes;
}

static PyObject *pointers(PyObject *self, PyObject *const *args, Py_ssize_t count) {
  (void)self;
  if (count != 4 || !PyBytes_Check(args[2])) {
    PyErr_SetString(PyExc_TypeError, "pointers(tensors, bytes, kinds, device)");
    return NULL;
  }
  const long long bytes = PyLong_AsLongLong(args[1]);
  const long long device = PyErr_Occurred() ? 0 : PyLong_AsLongLong(args[3]);
  if (PyErr_Occurred()) return NULL;
  PyObject *tensors = PySequence_Tuple(args[0]); /* (whatever the looks run, these stay) */
  if (!tensors) return NULL;
  const Py_ssize_t n = PyTuple_GET_SIZE(tensors);
  PyObject *out = PyBytes_FromStringAndSize(NULL, n * (Py_ssize_t)sizeof(uint64_t));
  if (!out) {
    Py_DECREF(tensors);
    return NULL;
  }
  uint64_t *address = (uint64_t *)PyBytes_AS_STRING(out);
  const Exchange *x = NULL;
  PyTypeObject *type = NULL;
  int fits = 1;
  for (Py_ssize_t i = 0; i < n && fits; ++i) {
    PyObject *t = PyTuple_GET_ITEM(tensors, i);
    if (Py_TYPE(t) != type) {
      type = Py_TYPE(t);
      x = exchange_of(t);
    }
    fits = x && look(x, t, bytes, (const uint8_t *)PyBytes_AS_STRING(args[2]), PyBytes_GET_SIZE(args[2]), device, address + i);
  }
  PyErr_Clear(); /* (of a tensor that has no view: Python says what it is) */
  Py_DECREF(tensors);
  if (fits) return out;
  Py_DECREF(out);
  Py_RETURN_NONE;
}

/* ---- whole calls ------------------------------------------------------------------------------------------------------
 * The calls of the operator with an epilogue and of the norms of queries and keys have a dozen tensors each; looked at from Python they take
 * 10 us, twice what the kernels of a small call do.  Here the tensors are looked at and the library called in one go.  The answer is
 * the library's status, or None where an argument is anything but the common one: then nothing has been done, and binding.py does all of
 * it again, saying what is wrong if something is. */
static struct {
  int (*device)(int *);
  int (*qk_fwd)(const osdp_qk *, const osdp_heads *, const osdp_heads *, const osdp_heads *, const osdp_heads *, void *);
  int (*qk_bwd)(const osdp_qk *, const osdp_heads *, const osdp_heads *, const osdp_heads *, const osdp_heads *, const osdp_heads *,
                const osdp_heads *, void *, void *, void *, size_t, void *);
  int (*fwd)(const osdp_shape *, const osdp_plan *, int32_t, const osdp_epilogue *, const void *, int64_t, const void *const *,
             const void *const *, int64_t, void *, int64_t, void *, size_t, void *, void *);
  int (*bwd)(const osdp_shape *, const osdp_plan *, int32_t, const osdp_epilogue_grad *, const void *, int64_t, const void *, int64_t,
             const void *const *, const void *const *, int64_t, void *, int64_t, void *const *, void *const *, void *, size_t, void *,
             void *);
} lib;

static PyObject *connect(PyObject *self, PyObject *const *args, Py_ssize_t count) {
  (void)self;
  void *p[5];
  if (count != 5) {
    PyErr_SetString(PyExc_TypeError, "connect(hipGetDevice, qk forward, qk backward, forward, backward)");
    return NULL;
  }
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(args[i]);
    if (!p[i]) return NULL;
  }
  lib.device = (int (*)(int *))p[0];
  *(void **)&lib.qk_fwd = p[1];
  *(void **)&lib.qk_bwd = p[2];
  *(void **)&lib.fwd = p[3];
  *(void **)&lib.bwd = p[4];
  Py_RETURN_NONE;
}

/* What a call's tensors are looked at by: the exchange of the type that the last one had, and the GPU that all must be on. */
typedef struct {
  PyTypeObject *type;
  const Exchange *exchange;
  int device;
} Looker;

enum { kBf16 = 0, kF32 = 1, kI64 = 2, kF64 = 3, kU8 = 4, kOther = -1 };
static int kind_of(const View *v) {
  if (v->lanes != 1) return kOther;
  if (v->code == 4 && v->bits == 16) return kBf16;
  if (v->code == 2 && v->bits == 32) return kF32;
  if (v->code == 0 && v->bits == 64) return kI64;
  if (v->code == 2 && v->bits == 64) return kF64;
  if (v->code == 1 && v->bits == 8) return kU8;
  return kOther;
}

static int view(Looker *l, PyObject *t, View *v, void **data) {
  if (Py_TYPE(t) != l->type) {
    l->type = Py_TYPE(t);
    l->exchange = exchange_of(t);
  }
  if (!l->exchange || l->exchange->view(t, v) != 0) return 0;
  *data = (char *)v->data + v->offset;
  return (v->device_type == kCuda || v->device_type == kRocm) && v->device == l->device && v->shape && v->strides;
}

static int contiguous(const View *v, int64_t *elements) {
  int64_t n = 1;
  for (int32_t d = v->dims - 1; d >= 0; --d) {
    if (v->shape[d] != 1 && v->strides[d] != n) return 0;
    n *= v->shape[d];
  }
  *elements = n;
  return 1;
}

/* A contiguous tensor of so many elements (fewer than 0: any number, which is written there) of one kind; None is NULL. */
static int array(Looker *l, PyObject *t, int kind, int64_t *elements, void **data) {
  *data = NULL;
  if (t == Py_None) return 1;
  View v;
  int64_t n;
  if (!view(l, t, &v, data) || kind_of(&v) != kind || !contiguous(&v, &n)) return 0;
  if (*elements >= 0 && n != *elements) return 0;
  *elements = n;
  return 1;
}

/* A vector of n bf16 or fp32, all of a call's alike (*type: -1 before the first). */
static int vector(Looker *l, PyObject *t, int64_t n, int32_t *type, void **data) {
  *data = NULL;
  if (t == Py_None) return 1;
  View v;
  int64_t have;
  if (!view(l, t, &v, data) || !contiguous(&v, &have) || have != n) return 0;
  const int kind = kind_of(&v);
  if ((kind != kBf16 && kind != kF32) || (*type >= 0 && *type != kind)) return 0;
  *type = kind;
  return 1;
}

/* A bf16 matrix; rows and cols fewer than 0 are written.  None is NULL. */
static int matrix(Looker *l, PyObject *t, int64_t *rows, int64_t *cols, void **data, int64_t *ld) {
  *data = NULL;
  *ld = 0;
  if (t == Py_None) return 1;
  View v;
  if (!view(l, t, &v, data) || kind_of(&v) != kBf16 || v.dims != 2) return 0;
  if (*rows < 0) *rows = v.shape[0];
  if (*cols < 0) *cols = v.shape[1];
  if (v.shape[0] != *rows || v.shape[1] != *cols || (v.strides[1] != 1 && *cols > 1)) return 0;
  *ld = *rows > 1 ? v.strides[0] : *cols;
  return 1;
}

static int heads(Looker *l, PyObject *t, int64_t *T, int64_t *H, int64_t *D, osdp_heads *out) {
  View v;
  if (!view(l, t, &v, &out->p) || kind_of(&v) != kBf16 || v.dims != 3) return 0;
  if (*T < 0) *T = v.shape[0];
  if (*H < 0) *H = v.shape[1];
  if (*D < 0) *D = v.shape[2];
  if (v.shape[0] != *T || v.shape[1] != *H || v.shape[2] != *D || v.strides[2] != 1) return 0;
  out->ld = v.strides[0];
  out->head_stride = v.strides[1];
  return 1;
}

/* The tensors of a list of shards: contiguous bf16 of at least n elements each. */
static int shards(Looker *l, PyObject *list, int64_t I, int64_t O, int N, void **out) {
  const int64_t n = (I * O + N - 1) / N;
  for (int i = 0; i < N; ++i) {
    View v;
    int64_t have;
    if (!view(l, PyTuple_GET_ITEM(list, i), &v, &out[i]) || kind_of(&v) != kBf16 || !contiguous(&v, &have) || have < n) return 0;
  }
  return 1;
}

static int number(PyObject *o, int64_t *out) {
  if (!PyLong_CheckExact(o)) return 0;
  *out = PyLong_AsLongLong(o);
  return !(*out == -1 && PyErr_Occurred());
}
static int stream(PyObject *o, void **out) {
  *out = NULL;
  if (o == Py_None) return 1;
  if (!PyLong_CheckExact(o)) return 0;
  *out = PyLong_AsVoidPtr(o);
  return !(*out == NULL && PyErr_Occurred());
}

static int begin(Looker *l) {
  l->type = NULL;
  l->exchange = NULL;
  l->device = -1;
  return lib.device && lib.device(&l->device) == 0;
}

static PyObject *none(void) {
  PyErr_Clear();
  Py_RETURN_NONE;
}

/* qk(heads, positions, freqs, q weight, k weight, dq weight, dk weight, workspace, eps, norm, interleaved, stream): heads are q, k, q_out,
 * k_out, or q, k, dq_out, dk_out, dq, dk. */
static PyObject *qk(PyObject *self, PyObject *const *a, Py_ssize_t count) {
  (void)self;
  Looker l;
  if (count != 12 || !PyTuple_CheckExact(a[0]) || !PyFloat_CheckExact(a[8]) || !PyBool_Check(a[9]) || !PyBool_Check(a[10]) || !begin(&l)) return none();
  const Py_ssize_t n = PyTuple_GET_SIZE(a[0]);
  if (n != 4 && n != 6) return none();
  int64_t T = -1, H[2] = {-1, -1}, D = -1, pairs = -1, bytes = -1;
  osdp_heads h[6];
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!heads(&l, PyTuple_GET_ITEM(a[0], i), &T, &H[i & 1], &D, &h[i])) return none();
  if (H[0] > 65535 || H[1] > 65535 || D > 65535) return none();
  osdp_qk q = {0};
  void *p[7], *s;
  q.weight_type = -1;
  if (!array(&l, a[1], kI64, &T, &p[0]) || !array(&l, a[2], kF64, &pairs, &p[1]) || !vector(&l, a[3], D, &q.weight_type, &p[2]) ||
      !vector(&l, a[4], D, &q.weight_type, &p[3]) || !vector(&l, a[5], D, &q.weight_type, &p[4]) || !vector(&l, a[6], D, &q.weight_type, &p[5]) ||
      !array(&l, a[7], kU8, &bytes, &p[6]) || !stream(a[11], &s) || pairs > 65535)
    return none();
  q.T = T; q.q_heads = (int32_t)H[0]; q.k_heads = (int32_t)H[1]; q.D = (int32_t)D;
  q.rotary = a[2] == Py_None ? 0 : (int32_t)(2 * pairs);
  q.interleaved = a[10] == Py_True; q.norm = a[9] == Py_True;
  if (q.weight_type < 0) q.weight_type = OSDP_BF16;
  q.eps = PyFloat_AS_DOUBLE(a[8]);
  q.positions = p[0]; q.freqs = p[1]; q.q_weight = p[2]; q.k_weight = p[3];
  int status;
  Py_BEGIN_ALLOW_THREADS;
  status = n == 4 ? lib.qk_fwd(&q, &h[0], &h[1], &h[2], &h[3], s)
                  : lib.qk_bwd(&q, &h[0], &h[1], &h[2], &h[3], &h[4], &h[5], p[4], p[5], p[6], p[6] ? (size_t)bytes : 0, s);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(status);
}

/* A plan's arrays, of up to 64 operators. */
typedef struct {
  osdp_plan plan;
  int32_t k[64], staging[64];
  uint64_t mask[64];
  uint8_t dim[64];
} Plan;

static int sequence(PyObject *plan, const char *name, Py_ssize_t n, uint64_t most, uint64_t *out, int *there) {
  PyObject *list = PyObject_GetAttrString(plan, name);
  if (!list) return 0;
  int fits = 1;
  *there = list != Py_None;
  if (*there) {
    fits = (PyList_CheckExact(list) || PyTuple_CheckExact(list)) && PySequence_Fast_GET_SIZE(list) == n;
    for (Py_ssize_t i = 0; fits && i < n; ++i) {
      PyObject *o = PySequence_Fast_GET_ITEM(list, i);
      fits = PyLong_CheckExact(o);
      if (fits) out[i] = PyLong_AsUnsignedLongLong(o);
      fits = fits && !PyErr_Occurred() && out[i] <= most;
    }
  }
  Py_DECREF(list);
  return fits;
}

static int plan_of(PyObject *o, Plan *p) {
  PyObject *ks = PyObject_GetAttrString(o, "k_per_op"), *staging;
  if (!ks) return 0;
  const Py_ssize_t n = PyList_CheckExact(ks) || PyTuple_CheckExact(ks) ? PySequence_Fast_GET_SIZE(ks) : -1;
  Py_DECREF(ks);
  if (n < 1 || n > 64 || !(staging = PyObject_GetAttrString(o, "staging"))) return 0;
  int64_t mode;
  const int fits = number(staging, &mode) && mode >= 0 && mode <= INT32_MAX;
  Py_DECREF(staging);
  uint64_t v[64];
  int there;
  if (!fits || !sequence(o, "k_per_op", n, INT32_MAX, v, &there)) return 0;
  p->plan = (osdp_plan){.n_ops = (int32_t)n, .k_per_op = p->k, .staging = (int32_t)mode};
  for (Py_ssize_t i = 0; i < n; ++i) p->k[i] = (int32_t)v[i];
  if (!sequence(o, "zdp_mask", n, UINT64_MAX, p->mask, &there)) return 0;
  p->plan.zdp_mask = there ? p->mask : NULL;
  if (!sequence(o, "split_dim_per_op", n, 255, v, &there)) return 0;
  for (Py_ssize_t i = 0; there && i < n; ++i) p->dim[i] = (uint8_t)v[i];
  p->plan.split_dim_per_op = there ? p->dim : NULL;
  if (!sequence(o, "staging_per_op", n, INT32_MAX, v, &there)) return 0;
  for (Py_ssize_t i = 0; there && i < n; ++i) p->staging[i] = (int32_t)v[i];
  p->plan.staging_per_op = there ? p->staging : NULL;
  return 1;
}

static PyObject *linear_of(PyObject *const *a, PyObject *w_shards, PyObject *dw_shards);

/* linear(X, w_shards, Y or dY, k, workspace, plan, operator, stream, copy stream, activation, z, bias, residual) forward;
 * .. bias's gradient, dz, dX, dw_shards) backward.  No slices in DP mode. */
static PyObject *linear(PyObject *self, PyObject *const *a, Py_ssize_t count) {
  (void)self;
  if ((count != 13 && count != 15) || !PyList_CheckExact(a[1]) || (count == 15 && !PyList_CheckExact(a[14]))) return none();
  PyObject *w = PyList_AsTuple(a[1]), *dw = count == 15 ? PyList_AsTuple(a[14]) : NULL, *answer = NULL; /* (whatever the looks run, these stay) */
  if (w && (dw || count == 13)) answer = linear_of(a, w, dw);
  Py_XDECREF(w);
  Py_XDECREF(dw);
  return answer;
}

static PyObject *linear_of(PyObject *const *a, PyObject *w_shards, PyObject *dw_shards) {
  Looker l;
  const int forward = dw_shards == NULL;
  if (!begin(&l)) return none();
  const Py_ssize_t N = PyTuple_GET_SIZE(w_shards);
  int64_t T = -1, I = -1, O = -1, k, op, act, bytes = -1, ld[5];
  void *x, *y, *z, *bias, *other, *dx = NULL, *ws, *sc, *sp, *w[OSDP_MAX_SHARDS], *dw[OSDP_MAX_SHARDS];
  int32_t type = -1;
  Plan plan;
  if (N < 1 || N > OSDP_MAX_SHARDS || a[0] == Py_None || a[2] == Py_None || a[4] == Py_None || !number(a[3], &k) || !number(a[6], &op) ||
      !number(a[9], &act) || k < 0 || k > INT32_MAX || op < 0 || op > 63 || act < 0 || act > INT32_MAX || !stream(a[7], &sc) || !stream(a[8], &sp) ||
      !matrix(&l, a[0], &T, &I, &x, &ld[0]) || !matrix(&l, a[2], &T, &O, &y, &ld[1]) || !matrix(&l, a[10], &T, &O, &z, &ld[2]) ||
      !vector(&l, a[11], O, &type, &bias) || !matrix(&l, a[12], &T, &O, &other, &ld[3]) || !array(&l, a[4], kU8, &bytes, &ws) || I < 1 || O < 1 ||
      I > INT32_MAX || O > INT32_MAX || !shards(&l, w_shards, I, O, (int)N, w) || (a[5] != Py_None && !plan_of(a[5], &plan)))
    return none();
  if (!forward && (a[13] == Py_None || PyTuple_GET_SIZE(dw_shards) != N || !matrix(&l, a[13], &T, &I, &dx, &ld[4]) ||
                   !shards(&l, dw_shards, I, O, (int)N, dw)))
    return none();
  const osdp_shape shape = {T, I, O, (int32_t)N, (int32_t)k};
  const osdp_plan *use = a[5] != Py_None ? &plan.plan : NULL;
  if (type < 0) type = OSDP_BF16;
  int status;
  Py_BEGIN_ALLOW_THREADS;
  if (forward) {
    const osdp_epilogue e = {bias, other, ld[3], z, ld[2], (int32_t)act, type};
    status = lib.fwd(&shape, use, (int32_t)op, &e, x, ld[0], (const void *const *)w, NULL, 0, y, ld[1], ws, (size_t)bytes, sc, sp);
  } else {
    const osdp_epilogue_grad e = {z, ld[2], other, ld[3], bias, (int32_t)act, type};
    status = lib.bwd(&shape, use, (int32_t)op, &e, x, ld[0], y, ld[1], (const void *const *)w, NULL, 0, dx, ld[4], dw, NULL, ws, (size_t)bytes,
                     sc, sp);
  }
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(status);
}

static PyMethodDef methods[] = {
    {"connect", (PyCFunction)(void (*)(void))connect, METH_FASTCALL, "connect(addresses of hipGetDevice and the library's entry points)"},
    {"qk", (PyCFunction)(void (*)(void))qk, METH_FASTCALL, "norms and rotation of queries and keys, or the pass back: the library's status, or None"},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, "the operator with an epilogue, or its pass back: the library's status, or None"},
    {"pointers", (PyCFunction)(void (*)(void))pointers, METH_FASTCALL,
     "pointers(tensors, bytes, kinds, device): addresses, as an array of 64-bit numbers in bytes, of tensors that are contiguous, on that GPU, of one\n"
     "of the kinds (two bytes each: DLPack's type code and bits) and of at least so many bytes; None if one is not, or cannot be looked at."},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pointers", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pointers(void) { return PyModule_Create(&module); }
