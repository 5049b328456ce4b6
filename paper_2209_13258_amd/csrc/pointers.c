/* A look at a list of shards and their addresses, in one go, for binding.py.
 *
 * What makes a tensor safe to hand on is its length, type, device and that it is contiguous.  Asked from Python, each question to each tensor costs
 * 50 ns, which makes a call with 8 shards 2 us longer and one with 64 12 us, more than the kernels of a small call take.  PyTorch's tensors offer all
 * of it at once by DLPack's exchange from C (version 1: the structures below, and the type's attribute that holds them); a list that holds anything
 * else, or anything that does not fit, is left to Python, which says what is wrong with it. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

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

static PyMethodDef methods[] = {
    {"pointers", (PyCFunction)(void (*)(void))pointers, METH_FASTCALL,
     "pointers(tensors, bytes, kinds, device): addresses, as an array of 64-bit numbers in bytes, of tensors that are contiguous, on that GPU, of one\n"
     "of the kinds (two bytes each: DLPack's type code and bits) and of at least so many bytes; None if one is not, or cannot be looked at."},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pointers", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pointers(void) { return PyModule_Create(&module); }
