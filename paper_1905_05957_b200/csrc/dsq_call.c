/* Calls of the C ABI from Python for the paths where the call itself is what counts (a product for one token takes a few
 * microseconds on the device; ctypes spends about as long on seventeen arguments).
 *
 * call(address, a, b, ...) -> int: calls a function of the ABI whose arguments are all pointers or integers.  Every argument is
 * passed as 64 bits, which the x86-64 and AArch64 calling conventions pass in the same places as narrower integers; None is
 * NULL.  The caller vouches for the address and the number of arguments.
 *
 * call_struct(address, stream, a, b, ...) -> int: calls a function of the ABI that takes a structure whose members are all 64 bits
 * wide, given one by one (a Python float becomes a double), and a stream.  size_struct(address, a, b, ...) -> int: one that takes such a
 * structure alone and returns a size of 64 bits; members that are not given are 0.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#define MOST 18
typedef uint64_t u;

static PyObject* call(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  u a[MOST] = {0};
  (void)self;
  if (n < 1 || n > MOST + 1) {
    PyErr_SetString(PyExc_TypeError, "an address and at most 18 arguments expected");
    return NULL;
  }
  const u f = (u)PyLong_AsUnsignedLongLong(args[0]);
  if (PyErr_Occurred()) return NULL;
  for (Py_ssize_t i = 1; i < n; ++i) {
    if (args[i] == Py_None) continue;
    a[i - 1] = (u)PyLong_AsUnsignedLongLongMask(args[i]);
    if (a[i - 1] == (u)-1 && PyErr_Occurred()) return NULL;
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = ((int (*)(u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u))f)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10],
                                                                        a[11], a[12], a[13], a[14], a[15], a[16], a[17]);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

#define MOST_MEMBERS 64

static int members(u* to, PyObject* const* args, Py_ssize_t n) {
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (args[i] == Py_None) continue;
    if (PyFloat_CheckExact(args[i])) {
      const double v = PyFloat_AS_DOUBLE(args[i]);
      memcpy(to + i, &v, sizeof v);
      continue;
    }
    to[i] = (u)PyLong_AsUnsignedLongLongMask(args[i]);
    if (to[i] == (u)-1 && PyErr_Occurred()) return 0;
  }
  return 1;
}

static PyObject* call_struct(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  u a[MOST_MEMBERS] = {0}, head[2] = {0};
  (void)self;
  if (n < 3 || n > MOST_MEMBERS + 2) {
    PyErr_SetString(PyExc_TypeError, "an address, a stream and 1 to 64 members expected");
    return NULL;
  }
  if (!members(head, args, 2) || !members(a, args + 2, n - 2)) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = ((int (*)(const u*, u))head[0])(a, head[1]);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyObject* size_struct(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  u a[MOST_MEMBERS] = {0}, f = 0;
  (void)self;
  if (n < 2 || n > MOST_MEMBERS + 1) {
    PyErr_SetString(PyExc_TypeError, "an address and 1 to 64 members expected");
    return NULL;
  }
  if (!members(&f, args, 1) || !members(a, args + 1, n - 1)) return NULL;
  return PyLong_FromUnsignedLongLong(((u (*)(const u*))f)(a));
}

static PyMethodDef methods[] = {{"call", (PyCFunction)(void*)call, METH_FASTCALL, "call(address, *integers) -> int"},
                                {"call_struct", (PyCFunction)(void*)call_struct, METH_FASTCALL, "call_struct(address, stream, *members) -> int"},
                                {"size_struct", (PyCFunction)(void*)size_struct, METH_FASTCALL, "size_struct(address, *members) -> int"},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "dsq_call", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit_dsq_call(void) { return PyModule_Create(&module); }
