// The calls that are made once per layer and step, for the Python binding without ctypes in between:
// ck_decode_step and the four on caches in pages.
//
// ck_decode_step is made once per layer and generated token, and at small batches its marshalling (fifteen tensors, two method
// calls and two ctypes conversions each) took longer than the kernel: 9.9 us from call to call
// for 2 head-problems, B = 256, where the kernel needs 7.1.  The host now needs 5.9 us.
//
// decode_step(entry, shape, 15 tensors, 9 numbers) takes what ck_decode_step takes, `entry` being
// its address.  It returns the status code, or None if any argument is not of the plain
// kind (a contiguous tensor, a number): nothing has been called then, and the caller goes the
// general way, which accepts or refuses the arguments in its own words.  The others do the same;
// they also look at the tensors' types, shapes and strides, as the general way does.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "clusterkv.h"

namespace {

using Entry = decltype(&ck_decode_step);

PyObject *s_is_contiguous, *s_data_ptr, *s_dtype, *s_size, *s_stride, *s_hkv, *s_d, *s_address, *s_device,
    *s_get_device;
PyObject* s_shape[7];
PyObject* types[4];                                     // torch's bfloat16 and float32 (CK_BF16, CK_F32), int32, uint8
enum { INT32 = 2, UINT8 = 3 };

bool as_int(PyObject* o, int64_t* v) {
  if (!o || !PyLong_Check(o)) return false;
  int overflow = 0;
  *v = PyLong_AsLongLongAndOverflow(o, &overflow);
  return overflow == 0;
}
bool as_i32(PyObject* o, int32_t* v) {
  int64_t w;
  if (!as_int(o, &w) || w < INT32_MIN || w > INT32_MAX) return false;
  *v = (int32_t)w;
  return true;
}

bool as_pointer(PyObject* t, void** p) {
  if (t == Py_None || PyLong_Check(t)) return false;
  PyObject* c = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  const bool plain = c == Py_True;
  Py_XDECREF(c);
  if (!plain) return false;
  PyObject* a = PyObject_CallMethodNoArgs(t, s_data_ptr);
  int64_t v = 0;
  const bool ok = as_int(a, &v);
  Py_XDECREF(a);
  *p = reinterpret_cast<void*>(static_cast<uintptr_t>(v));
  return ok;
}

bool as_shape(PyObject* o, ck_shape* sh) {
  int32_t* f[7] = {&sh->S, &sh->Hq, &sh->Hkv, &sh->d, nullptr, &sh->C_cap, &sh->dtype};
  for (int i = 0; i < 7; ++i) {
    PyObject* a = PyObject_GetAttr(o, s_shape[i]);
    const bool ok = a && (f[i] ? as_i32(a, f[i]) : as_int(a, &sh->N_cap));
    Py_XDECREF(a);
    if (!ok) return false;
  }
  return true;
}

enum { TENSORS = 15, NUMBERS = 9, ARGS = 2 + TENSORS + NUMBERS };

PyObject* decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != ARGS) {
    PyErr_SetString(PyExc_TypeError, "decode_step: wrong number of arguments");
    return nullptr;
  }
  int64_t entry;
  ck_shape sh;
  void* p[TENSORS];
  int64_t sink, rb, re, ws_bytes, stream;
  int32_t n_clusters, budget, flags, stride;
  bool ok = as_int(args[0], &entry) && entry != 0 && as_shape(args[1], &sh);
  for (int i = 0; ok && i < TENSORS; ++i) ok = as_pointer(args[2 + i], &p[i]);
  PyObject* const* a = args + 2 + TENSORS;
  ok = ok && as_i32(a[0], &n_clusters) && as_i32(a[1], &budget) && as_i32(a[2], &flags) &&
       as_int(a[3], &sink) && as_int(a[4], &rb) && as_int(a[5], &re) && PyFloat_Check(a[6]) &&
       as_i32(a[7], &stride) && as_int(a[8], &stream);
  if (ok) {
    PyObject* b = PyObject_CallMethod(args[2 + TENSORS - 1], "numel", nullptr);
    ok = as_int(b, &ws_bytes) && ws_bytes >= 0;         // the workspace holds bytes
    Py_XDECREF(b);
  }
  if (!ok) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  const float scale = (float)PyFloat_AS_DOUBLE(a[6]);
  const Entry fn = reinterpret_cast<Entry>(static_cast<uintptr_t>(entry));
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(&sh, p[0], p[1], p[2], p[3], (const int32_t*)p[4], (const int32_t*)p[5],
          (const int32_t*)p[6], n_clusters, budget, (uint32_t)flags, sink, rb, re, scale,
          (float*)p[7], (int32_t*)p[8], (int32_t*)p[9], (int32_t*)p[10], (int32_t*)p[11], stride,
          (int32_t*)p[12], p[13], p[14], (size_t)ws_bytes,
          reinterpret_cast<void*>(static_cast<uintptr_t>(stream)));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// ---- tensors of a given type, shape and layout ----
bool has_type(PyObject* t, PyObject* type) {
  PyObject* a = PyObject_GetAttr(t, s_dtype);
  const bool ok = a && a == type;
  Py_XDECREF(a);
  return ok;
}
// attribute or result of a method: a tuple of n numbers at most 4
bool as_tuple(PyObject* tuple, int n, int64_t* v) {
  bool ok = tuple && PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == n;
  for (int i = 0; ok && i < n; ++i) ok = as_int(PyTuple_GET_ITEM(tuple, i), &v[i]);
  Py_XDECREF(tuple);
  return ok;
}
bool has_shape(PyObject* t, int n, const int64_t* shape) {
  int64_t v[4];
  if (!as_tuple(PyObject_GetAttr(t, s_size), n, v)) return false;
  for (int i = 0; i < n; ++i)
    if (v[i] != shape[i]) return false;
  return true;
}
// index of its device; -1 for the host
bool as_device(PyObject* t, int64_t* device) {
  PyObject* a = PyObject_CallMethodNoArgs(t, s_get_device);
  const bool ok = as_int(a, device);
  Py_XDECREF(a);
  return ok;
}
// what the tensors of a call have in common
struct Common {
  int64_t entry, device;
  ck_shape sh;
  const ck_paged_kv* kv;
  PyObject* type;
  bool here(PyObject* t) const {
    int64_t d;
    return as_device(t, &d) && d == device;
  }
};
// contiguous, of a type and shape; None is a null pointer where it may be
bool as_dense(const Common& c, PyObject* t, PyObject* type, int n, const int64_t* shape, void** p, bool may_be_none = false) {
  if (t == Py_None) {
    *p = nullptr;
    return may_be_none;
  }
  return !PyLong_Check(t) && has_type(t, type) && has_shape(t, n, shape) && c.here(t) && as_pointer(t, p);
}
// token rows [n, heads, d] that may lie apart
bool as_rows(const Common& c, PyObject* t, const int64_t (&shape)[3], void** p, int64_t* row_stride) {
  if (t == Py_None || PyLong_Check(t) || !has_type(t, c.type) || !has_shape(t, 3, shape) || !c.here(t)) return false;
  int64_t st[3];
  if (!as_tuple(PyObject_CallMethodNoArgs(t, s_stride), 3, st)) return false;
  if (st[2] != 1 || (st[1] != shape[2] && shape[1] > 1)) return false;
  *row_stride = shape[0] > 1 ? st[0] : shape[1] * shape[2];
  PyObject* a = PyObject_CallMethodNoArgs(t, s_data_ptr);
  int64_t v = 0;
  const bool ok = as_int(a, &v);
  Py_XDECREF(a);
  *p = reinterpret_cast<void*>(static_cast<uintptr_t>(v));
  return ok;
}
// a cache in pages whose heads, type and device are the call's
bool as_paged(const Common& c, PyObject* kv, const ck_paged_kv** p) {
  PyObject* const names[4] = {s_address, s_hkv, s_d, s_device};
  int64_t v[4];
  for (int i = 0; i < 4; ++i) {
    PyObject* a = PyObject_GetAttr(kv, names[i]);
    const bool ok = as_int(a, &v[i]);
    Py_XDECREF(a);
    if (!ok) return false;
  }
  *p = reinterpret_cast<const ck_paged_kv*>(static_cast<uintptr_t>(v[0]));
  return *p && v[1] == c.sh.Hkv && v[2] == c.sh.d && v[3] == c.device && has_type(kv, c.type);
}
// Arguments entry, shape and cache, and a tensor that says which device.
bool as_call(PyObject* const* args, PyObject* tensor, Common* c) {
  if (!types[0] || !as_int(args[0], &c->entry) || c->entry == 0 || !as_shape(args[1], &c->sh)) return false;
  if (c->sh.dtype != CK_BF16 && c->sh.dtype != CK_F32) return false;
  c->type = types[c->sh.dtype];
  if (tensor == Py_None || PyLong_Check(tensor) || !as_device(tensor, &c->device)) return false;
  return as_paged(*c, args[2], &c->kv);
}
bool as_float(PyObject* o, double* v) {
  if (!PyFloat_Check(o)) return false;
  *v = PyFloat_AS_DOUBLE(o);
  return true;
}
PyObject* not_plain() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// set_types(bfloat16, float32, int32, uint8): torch's
PyObject* set_types(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "set_types: wrong number of arguments");
    return nullptr;
  }
  for (int i = 0; i < 4; ++i) {
    Py_INCREF(args[i]);
    Py_XSETREF(types[i], args[i]);
  }
  Py_RETURN_NONE;
}

// rope_append(entry, shape, cache, q, k, v, q_out, lengths, freqs, q_starts, positions, factor, flags, stream)
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 14) {
    PyErr_SetString(PyExc_TypeError, "rope_append: wrong number of arguments");
    return nullptr;
  }
  Common c;
  int64_t stream, flags, size[3], n_freqs, s_q, s_k, s_v;
  void *q = nullptr, *k, *v, *q_out, *lengths, *freqs, *starts, *positions;
  double factor;
  if (!as_call(a, a[4], &c) || !as_tuple(PyObject_GetAttr(a[4], s_size), 3, size) ||
      !as_tuple(PyObject_GetAttr(a[8], s_size), 1, &n_freqs) || n_freqs > INT32_MAX / 2)
    return not_plain();
  const ck_shape& sh = c.sh;
  const int64_t n = size[0], rows_q[3] = {n, sh.Hq, sh.d}, rows_k[3] = {n, sh.Hkv, sh.d}, per_seq[1] = {sh.S};
  const int64_t n_starts[1] = {(int64_t)sh.S + 1}, per_row[1] = {n}, rates[1] = {n_freqs};
  const bool queries = a[3] != Py_None;
  s_q = (int64_t)sh.Hq * sh.d;
  const bool ok = (!queries || as_rows(c, a[3], rows_q, &q, &s_q)) && as_rows(c, a[4], rows_k, &k, &s_k) &&
                  as_rows(c, a[5], rows_k, &v, &s_v) && as_dense(c, a[6], c.type, 3, rows_q, &q_out, !queries) &&
                  as_dense(c, a[7], types[INT32], 1, per_seq, &lengths) &&
                  as_dense(c, a[8], types[CK_F32], 1, rates, &freqs) &&
                  as_dense(c, a[9], types[INT32], 1, n_starts, &starts, true) &&
                  as_dense(c, a[10], types[INT32], 1, per_row, &positions, true) && as_float(a[11], &factor) &&
                  as_int(a[12], &flags) && as_int(a[13], &stream);
  if (!ok) return not_plain();
  const auto fn = reinterpret_cast<decltype(&ck_rope_append)>(static_cast<uintptr_t>(c.entry));
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(&sh, q, k, v, s_q, s_k, s_v, n, (const int32_t*)starts, (const int32_t*)lengths, (const int32_t*)positions,
          (const float*)freqs, (int32_t)(2 * n_freqs), (float)factor, (uint32_t)flags, q_out, c.kv,
          reinterpret_cast<void*>(static_cast<uintptr_t>(stream)));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// paged_decode_attn(entry, shape, cache, q, lengths, out, token_idx, n_tokens, workspace, n_sink, window, max_tokens,
//                   scale, stream); max_tokens may be None: the lists' width
PyObject* paged_decode_attn(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 14) {
    PyErr_SetString(PyExc_TypeError, "paged_decode_attn: wrong number of arguments");
    return nullptr;
  }
  Common c;
  int64_t stream, sink, window, size[3] = {0, 0, 0}, ws_bytes;
  int32_t most;
  void *q, *lengths, *out, *list, *counts, *ws;
  double scale;
  if (!as_call(a, a[3], &c) || (a[6] != Py_None && !as_tuple(PyObject_GetAttr(a[6], s_size), 3, size)) ||
      !as_tuple(PyObject_GetAttr(a[8], s_size), 1, &ws_bytes))
    return not_plain();
  const ck_shape& sh = c.sh;
  const int64_t width = size[2], rows[3] = {sh.S, sh.Hq, sh.d}, per_seq[1] = {sh.S}, heads[2] = {sh.S, sh.Hkv};
  const int64_t lists[3] = {sh.S, sh.Hkv, width};
  most = (int32_t)width;
  const bool ok = as_dense(c, a[3], c.type, 3, rows, &q) && as_dense(c, a[4], types[INT32], 1, per_seq, &lengths) &&
                  as_dense(c, a[5], c.type, 3, rows, &out) && as_dense(c, a[6], types[INT32], 3, lists, &list, true) &&
                  as_dense(c, a[7], types[INT32], 2, heads, &counts, true) &&
                  as_dense(c, a[8], types[UINT8], 1, &ws_bytes, &ws) && as_int(a[9], &sink) &&
                  as_int(a[10], &window) && (a[11] == Py_None || as_i32(a[11], &most)) && as_float(a[12], &scale) &&
                  as_int(a[13], &stream) && width <= INT32_MAX;
  if (!ok) return not_plain();
  const auto fn = reinterpret_cast<decltype(&ck_paged_decode_attn)>(static_cast<uintptr_t>(c.entry));
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(&sh, q, c.kv, (const int32_t*)lengths, sink, window, (const int32_t*)list, (const int32_t*)counts,
          (int32_t)width, most, (float)scale, out, ws, (size_t)ws_bytes,
          reinterpret_cast<void*>(static_cast<uintptr_t>(stream)));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// prompt_attn(entry, shape, cache, q, q_starts, lengths, out, workspace, n_sink, window, scale, stream)
PyObject* prompt_attn(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 12) {
    PyErr_SetString(PyExc_TypeError, "prompt_attn: wrong number of arguments");
    return nullptr;
  }
  Common c;
  int64_t stream, sink, window, size[3], ws_bytes;
  void *q, *starts, *lengths, *out, *ws;
  double scale;
  if (!as_call(a, a[3], &c) || !as_tuple(PyObject_GetAttr(a[3], s_size), 3, size) ||
      !as_tuple(PyObject_GetAttr(a[7], s_size), 1, &ws_bytes))
    return not_plain();
  const ck_shape& sh = c.sh;
  const int64_t rows[3] = {size[0], sh.Hq, sh.d}, n_starts[1] = {(int64_t)sh.S + 1}, per_seq[1] = {sh.S};
  const bool ok = as_dense(c, a[3], c.type, 3, rows, &q) && as_dense(c, a[4], types[INT32], 1, n_starts, &starts) &&
                  as_dense(c, a[5], types[INT32], 1, per_seq, &lengths) && as_dense(c, a[6], c.type, 3, rows, &out) &&
                  as_dense(c, a[7], types[UINT8], 1, &ws_bytes, &ws) && as_int(a[8], &sink) && as_int(a[9], &window) &&
                  as_float(a[10], &scale) && as_int(a[11], &stream);
  if (!ok) return not_plain();
  const auto fn = reinterpret_cast<decltype(&ck_prompt_attn)>(static_cast<uintptr_t>(c.entry));
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(&sh, q, size[0], (const int32_t*)starts, c.kv, (const int32_t*)lengths, sink, window, (float)scale, out, ws,
          (size_t)ws_bytes, reinterpret_cast<void*>(static_cast<uintptr_t>(stream)));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// copy_rows(entry, shape, source, destination, n_copy, max_rows, row_idx, begin, src_seq, stream)
PyObject* copy_rows(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 10) {
    PyErr_SetString(PyExc_TypeError, "copy_rows: wrong number of arguments");
    return nullptr;
  }
  Common c;
  const ck_paged_kv* dst;
  int64_t stream, size[3] = {0, 0, 0};
  int32_t most;
  void *counts, *list, *begin, *src_seq;
  if (!as_call(a, a[4], &c) || !as_paged(c, a[3], &dst) || !as_i32(a[5], &most) ||
      (a[6] != Py_None && !as_tuple(PyObject_GetAttr(a[6], s_size), 3, size)))
    return not_plain();
  const ck_shape& sh = c.sh;
  const int64_t per_seq[1] = {sh.S}, lists[3] = {sh.S, sh.Hkv, size[2]};
  const bool ok = as_dense(c, a[4], types[INT32], 1, per_seq, &counts) &&
                  as_dense(c, a[6], types[INT32], 3, lists, &list, true) &&
                  as_dense(c, a[7], types[INT32], 1, per_seq, &begin, true) &&
                  as_dense(c, a[8], types[INT32], 1, per_seq, &src_seq, true) && as_int(a[9], &stream) &&
                  size[2] <= INT32_MAX;
  if (!ok) return not_plain();
  const auto fn = reinterpret_cast<decltype(&ck_copy_rows)>(static_cast<uintptr_t>(c.entry));
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(&sh, c.kv, dst, (const int32_t*)counts, most, (const int32_t*)list, list ? (int32_t)size[2] : most,
          (const int32_t*)begin, (const int32_t*)src_seq, reinterpret_cast<void*>(static_cast<uintptr_t>(stream)));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

#define CK_METHOD(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL
PyMethodDef methods[] = {
    {"decode_step", CK_METHOD(decode_step), "ck_decode_step on plain tensors; None if an argument is of another kind"},
    {"rope_append", CK_METHOD(rope_append), "ck_rope_append, likewise"},
    {"paged_decode_attn", CK_METHOD(paged_decode_attn), "ck_paged_decode_attn, likewise"},
    {"prompt_attn", CK_METHOD(prompt_attn), "ck_prompt_attn, likewise"},
    {"copy_rows", CK_METHOD(copy_rows), "ck_copy_rows, likewise"},
    {"set_types", CK_METHOD(set_types), "torch's bfloat16, float32, int32 and uint8"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ckhost", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ckhost(void) {
  static const char* const names[7] = {"S", "Hq", "Hkv", "d", "N_cap", "C_cap", "dtype"};
  for (int i = 0; i < 7; ++i)
    if (!(s_shape[i] = PyUnicode_InternFromString(names[i]))) return nullptr;
  const struct { PyObject** to; const char* name; } more[] = {
      {&s_is_contiguous, "is_contiguous"}, {&s_data_ptr, "data_ptr"}, {&s_dtype, "dtype"}, {&s_size, "shape"},
      {&s_stride, "stride"}, {&s_hkv, "Hkv"}, {&s_d, "_d"}, {&s_address, "_address"},
      {&s_device, "_device"}, {&s_get_device, "get_device"}};
  for (const auto& m : more)
    if (!(*m.to = PyUnicode_InternFromString(m.name))) return nullptr;
  return PyModule_Create(&module);
}
