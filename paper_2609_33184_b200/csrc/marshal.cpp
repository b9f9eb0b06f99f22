// Argument marshalling of the calls that a program makes once or twice per layer and step: checks a call's tensors
// and passes their addresses and strides to the C entry point.  (Without the launch a call of four tensors takes 0.5 us of
// the host; with ctypes, checks in Python and structures built one by one it was 7.5 us, more than its kernel takes of
// the GPU.  Called one by one, 64 new tokens were appended in 9.5 us, now in 3.5.)  Functions return the entry point's status; tensors that do not fit raise AssertionError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "specstream.h"

namespace {

// What the checks need of a context, and of a cache (bits: 16 or 8; desc: its description, which the caller keeps).
struct Ctx {
  ss_ctx* handle;
  int64_t dev, H_q, H_kv, d;
};
struct Cache {
  const void* desc;
  int64_t bits, H_kv, d, requests, dev;
};

template <typename S>
void drop(PyObject* cap) {
  delete static_cast<S*>(PyCapsule_GetPointer(cap, nullptr));
}

bool fail(const char* what) {
  PyErr_SetString(PyExc_AssertionError, what);
  return false;
}
const Ctx* ctx_of(PyObject* o) {
  if (!PyCapsule_CheckExact(o)) {
    fail("closed context");
    return nullptr;
  }
  return static_cast<const Ctx*>(PyCapsule_GetPointer(o, nullptr));
}
bool int_of(PyObject* o, int64_t* out) {
  *out = PyLong_AsLongLong(o);
  return !(*out == -1 && PyErr_Occurred());
}
bool int32_of(PyObject* o, int32_t* out) {
  int64_t v;
  if (!int_of(o, &v)) return false;
  if (v < INT32_MIN || v > INT32_MAX) {
    PyErr_SetString(PyExc_OverflowError, "not an int32");
    return false;
  }
  *out = (int32_t)v;
  return true;
}
bool float_of(PyObject* o, float* out) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) return false;
  *out = (float)v;
  return true;
}
template <typename T>
bool address_of(PyObject* o, T* out) {
  *out = o == Py_None ? nullptr : reinterpret_cast<T>(PyLong_AsVoidPtr(o));
  return !PyErr_Occurred();
}

// A [B, H, T, d] bf16 tensor, d contiguous.
bool rows(const Ctx* c, PyObject* o, int64_t B, int64_t H, int64_t T, ss_tensor* out) {
  if (!THPVariable_Check(o)) return fail("tensor expected");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.dim() != 4 || t.scalar_type() != at::kBFloat16 || t.get_device() != c->dev || t.size(0) != B || t.size(1) != H ||
      t.size(2) != T || t.size(3) != c->d || t.stride(3) != 1)
    return fail("bf16 tensor [B, H, T, d] of the call's shape on the context's device expected, d contiguous");
  *out = {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
  return true;
}
// B and T of the call, from its first tensor.
bool sizes(PyObject* o, int64_t* B, int64_t* T) {
  if (!THPVariable_Check(o)) return fail("tensor expected");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.dim() != 4) return fail("tensor [B, H, T, d] expected");
  *B = t.size(0);
  *T = t.size(2);
  return (*B <= INT32_MAX && *T <= INT32_MAX) || fail("too many rows");
}
// Rows in and rows out, or neither.
bool pair(const Ctx* c, PyObject* x, PyObject* out, int64_t B, int64_t H, int64_t T, ss_tensor* a, ss_tensor* b) {
  *a = *b = {nullptr, 0, 0, 0};
  if (x == Py_None) return out == Py_None || fail("rows out without rows in");
  return rows(c, x, B, H, T, a) && rows(c, out, B, H, T, b);
}
// n contiguous int32, or None.
bool ints(const Ctx* c, PyObject* o, int64_t n, const int32_t** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) return fail("tensor expected");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != at::kInt || t.numel() != n || t.get_device() != c->dev || !t.is_contiguous())
    return fail("contiguous int32 tensor of the call's size on the context's device expected");
  *out = static_cast<const int32_t*>(t.data_ptr());
  return true;
}
// A contiguous output.
bool output(const Ctx* c, PyObject* o, at::ScalarType type, int64_t B, int64_t T, bool row, void** out) {
  if (!THPVariable_Check(o)) return fail("tensor expected");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != type || t.get_device() != c->dev || !t.is_contiguous() || t.dim() != (row ? 4 : 3) ||
      t.size(0) != B || t.size(1) != c->H_q || t.size(2) != T || (row && t.size(3) != c->d))
    return fail("contiguous O (bf16, of Q's shape) and LSE (fp32 [B, H_q, T_q]) on the context's device expected");
  *out = t.data_ptr();
  return true;
}
const Cache* cache_of(const Ctx* c, PyObject* o, int64_t bits, int64_t B) {
  if (!PyCapsule_CheckExact(o)) {
    fail("cache expected");
    return nullptr;
  }
  const Cache* k = static_cast<const Cache*>(PyCapsule_GetPointer(o, nullptr));
  if (!k || k->bits != bits || k->H_kv != c->H_kv || k->d != c->d || k->requests < B || k->dev != c->dev) {
    fail("cache of another kind, shape or device");
    return nullptr;
  }
  return k;
}
bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return false;
}
using Args = PyObject* const*;

// The entry point's status.  It runs without the interpreter's lock, as a launch may wait for room in the device's queue
// (the caller keeps tensors, context and cache alive).
template <typename F>
PyObject* status_of(F call) {
  ss_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = call();
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

// context(handle, dev, H_q, H_kv, d)
PyObject* context(PyObject*, Args a, Py_ssize_t n) {
  Ctx c;
  if (!count(n, 5) || !address_of(a[0], &c.handle) || !int_of(a[1], &c.dev) || !int_of(a[2], &c.H_q) ||
      !int_of(a[3], &c.H_kv) || !int_of(a[4], &c.d))
    return nullptr;
  return PyCapsule_New(new Ctx(c), nullptr, drop<Ctx>);
}
// cache(description, bits, H_kv, d, requests, dev)
PyObject* cache(PyObject*, Args a, Py_ssize_t n) {
  Cache c;
  if (!count(n, 6) || !address_of(a[0], &c.desc) || !int_of(a[1], &c.bits) || !int_of(a[2], &c.H_kv) ||
      !int_of(a[3], &c.d) || !int_of(a[4], &c.requests) || !int_of(a[5], &c.dev))
    return nullptr;
  return PyCapsule_New(new Cache(c), nullptr, drop<Cache>);
}

// rope_rotate(context, rope, Q, K, Q_out, K_out, pos, pos_off, row_cnt, stream)
PyObject* rope_rotate(PyObject*, Args a, Py_ssize_t n) {
  const Ctx* c;
  const ss_rope* rope;
  int64_t B, T;
  ss_tensor q, qo, k, ko;
  const int32_t *pos, *off, *cnt;
  void* stream;
  if (!count(n, 10) || !(c = ctx_of(a[0])) || !address_of(a[1], &rope)) return nullptr;
  if (!sizes(a[3] == Py_None ? a[2] : a[3], &B, &T) || !pair(c, a[2], a[4], B, c->H_q, T, &q, &qo) ||
      !pair(c, a[3], a[5], B, c->H_kv, T, &k, &ko) || !ints(c, a[6], (rope ? rope->n_axes : 1) * B * T, &pos) ||
      !ints(c, a[7], B, &off) || !ints(c, a[8], B, &cnt) || !address_of(a[9], &stream))
    return nullptr;
  return status_of([&] { return ss_rope_rotate(c->handle, rope, q, k, (int32_t)B, (int32_t)T, pos, off, cnt, qo, ko, stream); });
}

// kv_append / kv8_append(context, cache, K, V, rope, pos, Q, Q_out, dst_off, row_cnt, row_idx, stream)
template <int BITS>
PyObject* append(PyObject*, Args a, Py_ssize_t n) {
  const Ctx* c;
  const Cache* cache;
  const ss_rope* rope;
  int64_t B, T;
  ss_tensor k, v, q, qo;
  const int32_t *pos, *off, *cnt, *idx;
  void* stream;
  if (!count(n, 12) || !(c = ctx_of(a[0])) || !sizes(a[2], &B, &T) || !(cache = cache_of(c, a[1], BITS, B)) ||
      !rows(c, a[2], B, c->H_kv, T, &k) || !rows(c, a[3], B, c->H_kv, T, &v) || !address_of(a[4], &rope) ||
      !ints(c, a[5], (rope ? rope->n_axes : 1) * B * T, &pos) || !pair(c, a[6], a[7], B, c->H_q, T, &q, &qo) ||
      !ints(c, a[8], B, &off) || !ints(c, a[9], B, &cnt) || !ints(c, a[10], B * T, &idx) || !address_of(a[11], &stream))
    return nullptr;
  const int32_t b = (int32_t)B, t = (int32_t)T;
  return status_of([&] {
    return BITS == 8 ? ss_kv8_append(c->handle, static_cast<const ss_cache8*>(cache->desc), k, v, b, t, rope, pos, idx, cnt, off, q, qo, stream)
                     : ss_kv_append(c->handle, static_cast<const ss_cache16*>(cache->desc), k, v, b, t, rope, pos, idx, cnt, off, q, qo, stream);
  });
}

// decode_window / decode8_window(context, Q, scale, cache, window, sinks, valid_len, O, LSE, stream)
template <int BITS>
PyObject* decode_window(PyObject*, Args a, Py_ssize_t n) {
  const Ctx* c;
  const Cache* cache;
  int64_t B, T;
  float scale;
  int32_t window, sinks;
  ss_tensor q;
  const int32_t* len;
  void *o, *lse = nullptr, *stream;
  if (!count(n, 10) || !(c = ctx_of(a[0])) || !sizes(a[1], &B, &T) || !rows(c, a[1], B, c->H_q, T, &q) ||
      !float_of(a[2], &scale) || !(cache = cache_of(c, a[3], BITS, B)) || !int32_of(a[4], &window) ||
      !int32_of(a[5], &sinks) || !ints(c, a[6], B, &len) || !output(c, a[7], at::kBFloat16, B, T, true, &o) ||
      (a[8] != Py_None && !output(c, a[8], at::kFloat, B, T, false, &lse)) || !address_of(a[9], &stream))
    return nullptr;
  const int32_t b = (int32_t)B, t = (int32_t)T;
  return status_of([&] {
    return BITS == 8 ? ss_decode8_window(c->handle, q, b, t, scale, static_cast<const ss_cache8*>(cache->desc), window, sinks, len, o,
                                         static_cast<float*>(lse), stream)
                     : ss_decode_window(c->handle, q, b, t, scale, static_cast<const ss_cache16*>(cache->desc), window, sinks, len, o,
                                        static_cast<float*>(lse), stream);
  });
}

// verify_chunk_window / verify_chunk8_window(context, cache, window, sinks, valid_len, depth, B, T_q, stream)
template <int BITS>
PyObject* chunk_window(PyObject*, Args a, Py_ssize_t n) {
  const Ctx* c;
  const Cache* cache;
  int64_t B, T;
  int32_t window, sinks;
  const int32_t *len, *depth;
  void* stream;
  if (!count(n, 9) || !(c = ctx_of(a[0])) || !int_of(a[6], &B) || !int_of(a[7], &T) || !(cache = cache_of(c, a[1], BITS, B)) ||
      !int32_of(a[2], &window) || !int32_of(a[3], &sinks) || !ints(c, a[4], B, &len) || !ints(c, a[5], B * T, &depth) ||
      !address_of(a[8], &stream))
    return nullptr;
  return status_of([&] {
    return BITS == 8 ? ss_verify_chunk8_window(c->handle, static_cast<const ss_cache8*>(cache->desc), window, sinks, len, depth, stream)
                     : ss_verify_chunk_window(c->handle, static_cast<const ss_cache16*>(cache->desc), window, sinks, len, depth, stream);
  });
}

// A tensor without strides or storage (sparse, nested) throws when it is asked for them: no exception leaves a call.
template <PyObject* (*F)(PyObject*, Args, Py_ssize_t)>
PyObject* guarded(PyObject* self, Args a, Py_ssize_t n) {
  try {
    return F(self, a, n);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_AssertionError, e.what());
    return nullptr;
  }
}
#define SS_METHOD(name, ...) \
  {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<__VA_ARGS__>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SS_METHOD("context", context),
                         SS_METHOD("cache", cache),
                         SS_METHOD("rope_rotate", rope_rotate),
                         SS_METHOD("kv_append", append<16>),
                         SS_METHOD("kv8_append", append<8>),
                         SS_METHOD("decode_window", decode_window<16>),
                         SS_METHOD("decode8_window", decode_window<8>),
                         SS_METHOD("verify_chunk_window", chunk_window<16>),
                         SS_METHOD("verify_chunk8_window", chunk_window<8>),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
