/* The calls of a generated token (lrsa_cache_append, lrsa_attn_decode, lrsa_store_append, lrsa_store_decode) and the short ones
 * around them as a Python module over plain integers: they are host-bound for one sequence, and a foreign-function call with
 * ten arguments takes 1.1 us where this takes 0.2.  Every other entry point goes through ctypes. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/lrsa.h"

/* args[i] as an address, a size or a count; None is a null pointer */
static unsigned long long arg(PyObject* const* args, int i) {
  return args[i] == Py_None ? 0ull : PyLong_AsUnsignedLongLong(args[i]);
}
#define PTR(i) ((void*)(uintptr_t)arg(args, i))

/* (params, cache, cache_bytes, k_new, v_new, n_prev, n_new, workspace, workspace_bytes, stream) -> status */
static PyObject* cache_append(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != 10) return PyErr_Format(PyExc_TypeError, "cache_append takes 10 arguments");
  const lrsa_params_t* p = (const lrsa_params_t*)PTR(0);
  void *cache = PTR(1), *k = PTR(3), *v = PTR(4), *ws = PTR(7), *st = PTR(9);
  const size_t bytes = (size_t)arg(args, 2), ws_bytes = (size_t)arg(args, 8);
  const int32_t n_prev = (int32_t)PyLong_AsLong(args[5]), n_new = (int32_t)PyLong_AsLong(args[6]);
  if (PyErr_Occurred()) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = lrsa_cache_append(p, cache, bytes, k, v, n_prev, n_new, ws, ws_bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* (params, cache, cache_bytes, q, n_tokens, o, lse, workspace, workspace_bytes, stream) -> status */
static PyObject* attn_decode(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != 10) return PyErr_Format(PyExc_TypeError, "attn_decode takes 10 arguments");
  const lrsa_params_t* p = (const lrsa_params_t*)PTR(0);
  void *cache = PTR(1), *q = PTR(3), *o = PTR(5), *lse = PTR(6), *ws = PTR(7), *st = PTR(9);
  const size_t bytes = (size_t)arg(args, 2), ws_bytes = (size_t)arg(args, 8);
  const int32_t n_tokens = (int32_t)PyLong_AsLong(args[4]);
  if (PyErr_Occurred()) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = lrsa_attn_decode(p, cache, bytes, q, n_tokens, o, (float*)lse, ws, ws_bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* (params, q, k, lse, weight, workspace, workspace_bytes, stream) -> status */
static PyObject* attn_weights(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != 8) return PyErr_Format(PyExc_TypeError, "attn_weights takes 8 arguments");
  const lrsa_params_t* p = (const lrsa_params_t*)PTR(0);
  void *q = PTR(1), *k = PTR(2), *lse = PTR(3), *w = PTR(4), *ws = PTR(5), *st = PTR(7);
  const size_t ws_bytes = (size_t)arg(args, 6);
  if (PyErr_Occurred()) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = lrsa_attn_weights(p, q, k, (const float*)lse, (float*)w, ws, ws_bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* (params, weight, idx, stream) -> status */
static PyObject* weight_select(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != 4) return PyErr_Format(PyExc_TypeError, "weight_select takes 4 arguments");
  const lrsa_params_t* p = (const lrsa_params_t*)PTR(0);
  void *w = PTR(1), *idx = PTR(2), *st = PTR(3);
  if (PyErr_Occurred()) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = lrsa_weight_select(p, (const float*)w, (int32_t*)idx, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* args[1 .. 11]: list type, block, keep, then the eight pointers of lrsa_store_t */
#define STORE_ARGS 11
static lrsa_store_t store_of(PyObject* const* args) {
  lrsa_store_t s;
  s.list_type = (int32_t)PyLong_AsLong(args[1]);
  s.block = (int32_t)PyLong_AsLong(args[2]);
  s.keep = (int32_t)PyLong_AsLong(args[3]);
  s.reserved = 0;
  s.k_list = PTR(4); s.v_list = PTR(5); s.k_scale = (float*)PTR(6); s.v_scale = (float*)PTR(7);
  s.k_recent = PTR(8); s.v_recent = PTR(9); s.weight = (float*)PTR(10); s.idx = (int32_t*)PTR(11);
  return s;
}

/* (params, store ..., k_new, v_new, w_new, n_prev, n_new, workspace, workspace_bytes, stream) -> status */
static PyObject* store_append(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != 9 + STORE_ARGS) return PyErr_Format(PyExc_TypeError, "store_append takes 20 arguments");
  const lrsa_params_t* p = (const lrsa_params_t*)PTR(0);
  const lrsa_store_t s = store_of(args);
  void *k = PTR(12), *v = PTR(13), *w = PTR(14), *ws = PTR(17), *st = PTR(19);
  const int32_t n_prev = (int32_t)PyLong_AsLong(args[15]), n_new = (int32_t)PyLong_AsLong(args[16]);
  const size_t ws_bytes = (size_t)arg(args, 18);
  if (PyErr_Occurred()) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = lrsa_store_append(p, &s, k, v, (const float*)w, n_prev, n_new, ws, ws_bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* (params, store ..., q, n_tokens, o, lse, workspace, workspace_bytes, stream) -> status */
static PyObject* store_decode(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != 8 + STORE_ARGS) return PyErr_Format(PyExc_TypeError, "store_decode takes 19 arguments");
  const lrsa_params_t* p = (const lrsa_params_t*)PTR(0);
  const lrsa_store_t s = store_of(args);
  void *q = PTR(12), *o = PTR(14), *lse = PTR(15), *ws = PTR(16), *st = PTR(18);
  const int32_t n_tokens = (int32_t)PyLong_AsLong(args[13]);
  const size_t ws_bytes = (size_t)arg(args, 17);
  if (PyErr_Occurred()) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = lrsa_store_decode(p, &s, q, n_tokens, o, (float*)lse, ws, ws_bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* (params, store ..., n_windows, k, v, stream) -> status */
static PyObject* store_rows(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != 5 + STORE_ARGS) return PyErr_Format(PyExc_TypeError, "store_rows takes 16 arguments");
  const lrsa_params_t* p = (const lrsa_params_t*)PTR(0);
  const lrsa_store_t s = store_of(args);
  const int32_t n_windows = (int32_t)PyLong_AsLong(args[12]);
  void *k = PTR(13), *v = PTR(14), *st = PTR(15);
  if (PyErr_Occurred()) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = lrsa_store_rows(p, &s, n_windows, (float*)k, (float*)v, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyMethodDef methods[] = {
    {"cache_append", (PyCFunction)(void (*)(void))cache_append, METH_FASTCALL, NULL},
    {"attn_decode", (PyCFunction)(void (*)(void))attn_decode, METH_FASTCALL, NULL},
    {"attn_weights", (PyCFunction)(void (*)(void))attn_weights, METH_FASTCALL, NULL},
    {"weight_select", (PyCFunction)(void (*)(void))weight_select, METH_FASTCALL, NULL},
    {"store_append", (PyCFunction)(void (*)(void))store_append, METH_FASTCALL, NULL},
    {"store_decode", (PyCFunction)(void (*)(void))store_decode, METH_FASTCALL, NULL},
    {"store_rows", (PyCFunction)(void (*)(void))store_rows, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lrsa_call", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__lrsa_call(void) { return PyModule_Create(&module); }
