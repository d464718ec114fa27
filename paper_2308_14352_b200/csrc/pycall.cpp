// CPython callables of C entry points.  The training operators' smallest calls run for 2 to 6 us on the GPU, and turning a dozen arguments through
// ctypes takes as long as one of their launches (us per call of twelve arguments without the call itself: ctypes 1.7, this 0.2).
// bind(address, kinds, types, owner) gives a callable of one entry point: kinds is one letter per argument, 'p' an address (an int or None), 'i' a
// 32-bit integer, 's' a description (an object of the next of `types`, whose buffer it is, or None); the result is its int status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stddef.h>
#include <stdint.h>

namespace {

constexpr int MOST = 18;

struct Call {
  PyObject_HEAD
  vectorcallfunc vectorcall;
  void* entry;
  PyObject* owner;  // whose code `entry` is
  Py_ssize_t n;
  char kinds[MOST];
  PyTypeObject* types[MOST];
};

// Every argument is of the integer class: on this ABI (x86-64 System V) it travels as one 64-bit word, of which an int parameter reads the lower half.
using W = uint64_t;
int call_entry(void* entry, Py_ssize_t n, const W* a) {
  switch (n) {
    case 9: return reinterpret_cast<int (*)(W, W, W, W, W, W, W, W, W)>(entry)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8]);
    case 8: return reinterpret_cast<int (*)(W, W, W, W, W, W, W, W)>(entry)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
    case 10: return reinterpret_cast<int (*)(W, W, W, W, W, W, W, W, W, W)>(entry)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9]);
    case 12:
      return reinterpret_cast<int (*)(W, W, W, W, W, W, W, W, W, W, W, W)>(entry)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11]);
    case 13:
      return reinterpret_cast<int (*)(W, W, W, W, W, W, W, W, W, W, W, W, W)>(entry)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10],
                                                                                     a[11], a[12]);
    default:
      return reinterpret_cast<int (*)(W, W, W, W, W, W, W, W, W, W, W, W, W, W, W, W)>(entry)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9],
                                                                                              a[10], a[11], a[12], a[13], a[14], a[15]);
  }
}
bool takes(Py_ssize_t n) { return n == 8 || n == 9 || n == 10 || n == 12 || n == 13 || n == 16; }

PyObject* call(PyObject* self, PyObject* const* args, size_t nargsf, PyObject* names) {
  Call* c = reinterpret_cast<Call*>(self);
  const Py_ssize_t n = PyVectorcall_NARGS(nargsf);
  if (n != c->n || (names && PyTuple_GET_SIZE(names) > 0))
    return PyErr_Format(PyExc_TypeError, "expected %zd positional arguments, got %zd", c->n, n + (names ? PyTuple_GET_SIZE(names) : 0));
  W words[MOST] = {};
  Py_buffer views[MOST];
  int held = 0;
  bool ok = true;
  for (Py_ssize_t i = 0; i < n && ok; ++i) {
    if (c->kinds[i] == 'i') {
      const long v = PyLong_AsLong(args[i]);
      if (v == -1 && PyErr_Occurred()) ok = false;
      else if (v < INT32_MIN || v > INT32_MAX) {
        PyErr_Format(PyExc_OverflowError, "argument %zd is no 32-bit integer", i);
        ok = false;
      }
      words[i] = static_cast<W>(v);
    } else if (args[i] == Py_None) {
      words[i] = 0;
    } else if (c->kinds[i] == 'p') {
      if (!PyLong_Check(args[i])) {
        PyErr_Format(PyExc_TypeError, "argument %zd is an address: an int or None", i);
        ok = false;
        break;
      }
      words[i] = reinterpret_cast<W>(PyLong_AsVoidPtr(args[i]));
      ok = words[i] != 0 || !PyErr_Occurred();
    } else {
      if (!PyObject_TypeCheck(args[i], c->types[i])) {
        PyErr_Format(PyExc_TypeError, "argument %zd is a description of type %s", i, c->types[i]->tp_name);
        ok = false;
        break;
      }
      ok = PyObject_GetBuffer(args[i], &views[held], PyBUF_SIMPLE) == 0;
      if (ok) words[i] = reinterpret_cast<W>(views[held++].buf);
    }
  }
  int status = 0;
  if (ok) {
    Py_BEGIN_ALLOW_THREADS  // a launch may wait for room in its queue
    status = call_entry(c->entry, n, words);
    Py_END_ALLOW_THREADS
  }
  while (held > 0) PyBuffer_Release(&views[--held]);
  return ok ? PyLong_FromLong(status) : nullptr;
}

void release(PyObject* self) {
  Call* c = reinterpret_cast<Call*>(self);
  for (PyTypeObject* t : c->types) Py_XDECREF(t);
  Py_XDECREF(c->owner);
  Py_TYPE(self)->tp_free(self);
}

PyTypeObject call_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyObject* bind(PyObject*, PyObject* args) {
  PyObject *address, *types, *owner;
  const char* kinds;
  Py_ssize_t n;
  if (!PyArg_ParseTuple(args, "O!s#O!O", &PyLong_Type, &address, &kinds, &n, &PyTuple_Type, &types, &owner)) return nullptr;
  if (!takes(n)) return PyErr_Format(PyExc_ValueError, "no entry point has %zd arguments", n);
  Call* c = PyObject_New(Call, &call_type);
  if (!c) return nullptr;
  c->vectorcall = call;
  c->owner = nullptr;
  c->n = n;
  c->entry = PyLong_AsVoidPtr(address);
  for (PyTypeObject*& t : c->types) t = nullptr;
  Py_ssize_t next = 0;
  bool ok = c->entry != nullptr;
  for (Py_ssize_t i = 0; i < n && ok; ++i) {
    c->kinds[i] = kinds[i];
    if (kinds[i] == 's') {
      PyObject* t = next < PyTuple_GET_SIZE(types) ? PyTuple_GET_ITEM(types, next++) : nullptr;
      ok = t && PyType_Check(t);
      if (ok) {
        Py_INCREF(t);
        c->types[i] = reinterpret_cast<PyTypeObject*>(t);
      }
    } else {
      ok = kinds[i] == 'p' || kinds[i] == 'i';
    }
  }
  if (!ok || next != PyTuple_GET_SIZE(types)) {
    Py_DECREF(c);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address, one letter (p, i, s) per argument and a type per s");
    return nullptr;
  }
  Py_INCREF(owner);
  c->owner = owner;
  return reinterpret_cast<PyObject*>(c);
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, "bind(address, kinds, types, owner): a callable of one C entry point"}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", "Callables of C entry points", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pycall() {
  call_type.tp_name = "_pycall.Call";
  call_type.tp_basicsize = sizeof(Call);
  call_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL;
  call_type.tp_vectorcall_offset = offsetof(Call, vectorcall);
  call_type.tp_call = PyVectorcall_Call;
  call_type.tp_dealloc = release;
  call_type.tp_free = PyObject_Free;
  if (PyType_Ready(&call_type) < 0) return nullptr;
  return PyModule_Create(&module);
}
