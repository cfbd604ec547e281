/* Calls of the C ABI from Python for the paths where the call itself is what counts (a product for one token takes a few
 * microseconds on the device; ctypes spends about as long on seventeen arguments).
 *
 * call(address, a, b, ...) -> int: calls a function of the ABI whose arguments are all pointers or integers.  Every argument is
 * passed as 64 bits, which the x86-64 and AArch64 calling conventions pass in the same places as narrower integers; None is
 * NULL.  The caller vouches for the address and the number of arguments.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

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

static PyMethodDef methods[] = {{"call", (PyCFunction)(void*)call, METH_FASTCALL, "call(address, *integers) -> int"}, {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "dsq_call", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit_dsq_call(void) { return PyModule_Create(&module); }
