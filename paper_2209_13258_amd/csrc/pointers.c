/* A look at a list of shards and their addresses, in one go, for binding.py.
 *
 * What makes a tensor safe to hand on (its bytes, type, device and that it is contiguous) is four questions to each besides its address.  Asked
 * from Python they make a call with 8 shards 2 us longer and one with 64 12 us, more than the kernels of a small call take; from here 0.8 and 6.5. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

static PyObject *name_nbytes, *name_dtype, *name_get_device, *name_is_contiguous, *name_data_ptr;

static PyObject *ask(PyObject *t, PyObject *method) {
  return PyObject_VectorcallMethod(method, &t, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, NULL);
}

/* *out = what `x` holds, which is let go; -1: it is no whole number. */
static int whole(PyObject *x, long long *out) {
  if (!x) return -1;
  *out = PyLong_AsLongLong(x);
  Py_DECREF(x);
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

/* 1: the tensor is as asked for, and *address where it lies; 0: it is not; -1: an exception. */
static int look(PyObject *t, long long bytes, PyObject *kinds, long long device, uint64_t *address) {
  long long n;
  PyObject *x;
  if (whole(PyObject_GetAttr(t, name_nbytes), &n) < 0) return -1;
  if (n < bytes) return 0;
  if (!(x = PyObject_GetAttr(t, name_dtype))) return -1;
  PyObject *allowed = PyDict_GetItemWithError(kinds, x);
  Py_DECREF(x);
  if (!allowed && PyErr_Occurred()) return -1;
  if (allowed != Py_True) return 0;
  if (whole(ask(t, name_get_device), &n) < 0) return -1;
  if (n != device) return 0;
  if (!(x = ask(t, name_is_contiguous))) return -1;
  Py_DECREF(x); /* (True and False outlive this) */
  if (x != Py_True) return 0;
  if (!(x = ask(t, name_data_ptr))) return -1;
  *address = PyLong_AsUnsignedLongLong(x);
  Py_DECREF(x);
  return PyErr_Occurred() ? -1 : 1;
}

static PyObject *pointers(PyObject *self, PyObject *const *args, Py_ssize_t count) {
  (void)self;
  if (count != 4 || !PyDict_Check(args[2])) {
    PyErr_SetString(PyExc_TypeError, "pointers(tensors, bytes, {dtype: True}, device)");
    return NULL;
  }
  const long long bytes = PyLong_AsLongLong(args[1]);
  const long long device = PyErr_Occurred() ? 0 : PyLong_AsLongLong(args[3]);
  if (PyErr_Occurred()) return NULL;
  PyObject *tensors = PySequence_Tuple(args[0]); /* (whatever the questions run, these stay) */
  if (!tensors) return NULL;
  const Py_ssize_t n = PyTuple_GET_SIZE(tensors);
  PyObject *out = PyBytes_FromStringAndSize(NULL, n * (Py_ssize_t)sizeof(uint64_t));
  int ok = out ? 1 : -1;
  for (Py_ssize_t i = 0; i < n && ok > 0; ++i)
    ok = look(PyTuple_GET_ITEM(tensors, i), bytes, args[2], device, (uint64_t *)PyBytes_AS_STRING(out) + i);
  Py_DECREF(tensors);
  if (ok > 0) return out;
  Py_XDECREF(out);
  if (ok < 0) return NULL;
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"pointers", (PyCFunction)(void (*)(void))pointers, METH_FASTCALL,
     "Addresses, as an array of 64-bit numbers in bytes, of tensors that are contiguous, on that device, of a type that maps to True and of at\n"
     "least so many bytes; None if one is not."},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pointers", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pointers(void) {
  if (!(name_nbytes = PyUnicode_InternFromString("nbytes")) || !(name_dtype = PyUnicode_InternFromString("dtype")) ||
      !(name_get_device = PyUnicode_InternFromString("get_device")) || !(name_is_contiguous = PyUnicode_InternFromString("is_contiguous")) ||
      !(name_data_ptr = PyUnicode_InternFromString("data_ptr")))
    return NULL;
  return PyModule_Create(&module);
}
