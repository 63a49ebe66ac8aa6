// The calls of binding.py that a program makes per chunk, without ctypes: the arguments of an ordinary call are read from the
// tensors, checked as binding.py checks them, and handed to the C ABI.  Anything else (another type than torch.Tensor, a host
// tensor, an int that is none or does not fit, shapes or strides that do not match) returns None, and binding.py goes its own
// way, which accepts or refuses it.  Nothing is kept from one call to the next.
//
// One 256-token chunk of 4 layers decoded into pages took 8.2 us a call, 5 of them in Python and ctypes; the launch takes 2.4.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cmath>
#include <cstdint>

#include "../../include/kvh.h"

// The tensor-exchange interface of the DLPack specification, where torch brings its header and offers it: one call of a C function gives all
// fields of a tensor, in place of five attribute look-ups of 70 to 130 ns each.  The serving-cache calls, which take up to a dozen
// tensors, come this way or not at all (a call of kvh_attention for one token: 15.9 us through ctypes, 13 of them on the host).
#if __has_include(<ATen/dlpack.h>)
#include <ATen/dlpack.h>
#endif
#if defined(DLPACK_MAJOR_VERSION) && DLPACK_MAJOR_VERSION == 1 && DLPACK_MINOR_VERSION >= 3
#define KVH_EXCHANGE 1
#else
#define KVH_EXCHANGE 0
#endif

namespace {

// Looked up once, when the module is imported.
PyObject *tensor_type, *dtype_f16, *dtype_bf16, *dtype_i32;  // torch's
PyObject *s_is_cuda, *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_numel, *s_cuda_stream;

// The functions of one loaded library, and torch's queries for the current stream.
struct Calls {
  PyObject_HEAD
  decltype(&kvh_encode) encode;
  decltype(&kvh_encode_batch) encode_batch;
  decltype(&kvh_decode) decode;
  decltype(&kvh_decode_batch) decode_batch;
  decltype(&kvh_encode_kept) encode_kept;
  decltype(&kvh_decode_kept) decode_kept;
  decltype(&kvh_append) append;
  decltype(&kvh_attention) attention;
  PyObject *current_device, *raw_stream;
};

// What one call has read so far.  A failed step leaves ok false; an error raised on the way is dropped, because the slow path
// meets the same one, but not what is no error of the call (an interrupt, an exit).
struct Reader {
  bool ok = true;

  bool is_true(PyObject* t, PyObject* name) {
    PyObject* r = PyObject_GetAttr(t, name);
    const bool yes = r == Py_True;
    Py_XDECREF(r);
    return yes;
  }
  bool device_tensor(PyObject* t) { return Py_TYPE(t) == reinterpret_cast<PyTypeObject*>(tensor_type) && is_true(t, s_is_cuda); }
  bool has_dtype(PyObject* t, PyObject* dtype) {
    PyObject* r = PyObject_GetAttr(t, s_dtype);
    const bool same = r == dtype;
    Py_XDECREF(r);
    return same;
  }
  int64_t int_method(PyObject* t, PyObject* name) {
    PyObject* r = PyObject_CallMethodNoArgs(t, name);
    int64_t v = 0;
    if (r == nullptr || !PyLong_CheckExact(r)) ok = false; else v = PyLong_AsLongLong(r);
    Py_XDECREF(r);
    if (PyErr_Occurred()) ok = false;
    return v;
  }
  void* pointer(PyObject* t) {
    PyObject* r = PyObject_CallMethodNoArgs(t, s_data_ptr);
    void* p = nullptr;
    if (r == nullptr || !PyLong_CheckExact(r)) ok = false; else p = PyLong_AsVoidPtr(r);
    Py_XDECREF(r);
    if (PyErr_Occurred()) ok = false;
    return p;
  }
  // A device tensor of any type.
  void* device(PyObject* t) {
    if (ok && !device_tensor(t)) ok = false;
    return ok ? pointer(t) : nullptr;
  }
  // None, or a device tensor of int32 with at least `least` elements.
  int32_t* words(PyObject* t, int64_t least) {
    if (!ok || t == Py_None) return nullptr;
    if (!device_tensor(t) || !has_dtype(t, dtype_i32) || (least > 0 && int_method(t, s_numel) < least)) ok = false;
    return ok ? static_cast<int32_t*>(pointer(t)) : nullptr;
  }
  int64_t wide(PyObject* o) {
    if (!PyLong_CheckExact(o)) {
      ok = false;
      return 0;
    }
    int overflow = 0;
    const int64_t v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow != 0) ok = false;
    return v;
  }
  int narrow(PyObject* o) {
    const int64_t v = wide(o);
    if (v < INT32_MIN || v > INT32_MAX) ok = false;
    return (int)v;
  }
  int dims(PyObject* tuple, int64_t (&out)[4]) {
    if (tuple == nullptr || !PyTuple_Check(tuple) || PyTuple_GET_SIZE(tuple) > 4) {
      ok = false;
      return 0;
    }
    const int n = (int)PyTuple_GET_SIZE(tuple);
    for (int i = 0; i < n; ++i) out[i] = wide(PyTuple_GET_ITEM(tuple, i));
    return n;
  }
};

// K and V: device tensors [l][tokens][c], or [l][blocks][block][c] when paged, of one 16-bit type, equal in shape and strides.
struct View {
  kvh_kv_view v;
  kvh_dtype dt;
  int l, tokens, c;
};

View read_view(Reader& r, PyObject* k, PyObject* v, bool paged) {
  View out{};
  if (!r.ok || !r.device_tensor(k) || !r.device_tensor(v)) {
    r.ok = false;
    return out;
  }
  PyObject* dt = PyObject_GetAttr(k, s_dtype);
  Py_XDECREF(dt);  // torch keeps its types
  if ((dt != dtype_f16 && dt != dtype_bf16) || !r.has_dtype(v, dt)) {
    r.ok = false;
    return out;
  }
  int64_t size[2][4], stride[2][4];
  int n[2];
  PyObject* t[2] = {k, v};
  for (int i = 0; i < 2; ++i) {
    PyObject* sizes = PyObject_GetAttr(t[i], s_shape);
    n[i] = r.dims(sizes, size[i]);
    Py_XDECREF(sizes);
    PyObject* strides = PyObject_CallMethodNoArgs(t[i], s_stride);
    if (r.dims(strides, stride[i]) != n[i]) r.ok = false;
    Py_XDECREF(strides);
  }
  const int want = paged ? 4 : 3;
  if (!r.ok || n[0] != want || n[1] != want) {
    r.ok = false;
    return out;
  }
  for (int i = 0; i < want; ++i)
    if (size[0][i] != size[1][i] || stride[0][i] != stride[1][i] || size[0][i] > INT32_MAX) r.ok = false;
  if (stride[0][want - 1] != 1 || (paged && stride[0][1] != stride[0][2] * size[0][2])) r.ok = false;
  out.dt = dt == dtype_f16 ? KVH_F16 : KVH_BF16;
  out.l = (int)size[0][0];
  out.tokens = (int)size[0][1];
  out.c = (int)size[0][want - 1];
  out.v.layer_stride = stride[0][0];
  out.v.token_stride = stride[0][want - 2];
  if (r.ok) {
    out.v.k = r.pointer(k);
    out.v.v = r.pointer(v);
  }
  return out;
}

void* read_stream(Reader& r, Calls* self, PyObject* stream) {
  if (!r.ok) return nullptr;
  PyObject* p = nullptr;
  if (stream != Py_None) {
    p = PyObject_GetAttr(stream, s_cuda_stream);
  } else if (PyObject* dev = PyObject_CallNoArgs(self->current_device)) {
    p = PyObject_CallOneArg(self->raw_stream, dev);
    Py_DECREF(dev);
  }
  void* out = nullptr;
  if (p == nullptr || !PyLong_CheckExact(p)) r.ok = false; else out = PyLong_AsVoidPtr(p);
  Py_XDECREF(p);
  if (PyErr_Occurred()) r.ok = false;
  return out;
}

// The status of `call()`, made without the interpreter's lock as ctypes makes it, or None for binding.py to take over.
template <typename F>
PyObject* finish(const Reader& r, F&& call) {
  if (!r.ok) {
    if (PyErr_Occurred() != nullptr && !PyErr_ExceptionMatches(PyExc_Exception)) return nullptr;
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

#define KVH_ARGS(N)                                                      \
  Calls* self = reinterpret_cast<Calls*>(self_);                         \
  if (n_args != (N)) {                                                   \
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");       \
    return nullptr;                                                      \
  }                                                                      \
  Reader r

// encode(k, v, level, blob, n_tokens or None, stream)
PyObject* encode(PyObject* self_, PyObject* const* a, Py_ssize_t n_args) {
  KVH_ARGS(6);
  const View kv = read_view(r, a[0], a[1], false);
  const int level = r.narrow(a[2]), n = a[4] == Py_None ? kv.tokens : r.narrow(a[4]);
  void* blob = r.device(a[3]);
  const int64_t cap = r.ok ? r.int_method(a[3], s_numel) : 0;
  void* stream = read_stream(r, self, a[5]);
  return finish(r, [&] { return self->encode(&kv.v, kv.dt, kv.l, n, kv.c, level, blob, (size_t)cap, stream); });
}

// encode_batch(items, n_items, max_tokens_per_item, k, v, stream)
PyObject* encode_batch(PyObject* self_, PyObject* const* a, Py_ssize_t n_args) {
  KVH_ARGS(6);
  const View kv = read_view(r, a[3], a[4], false);
  const void* items = r.device(a[0]);
  const int n = r.narrow(a[1]), most = r.narrow(a[2]);
  void* stream = read_stream(r, self, a[5]);
  return finish(r, [&] {
    return self->encode_batch(static_cast<const kvh_enc_item*>(items), n, most, kv.dt, kv.l, kv.c, &kv.v, stream);
  });
}

// decode(blob, level, n_tokens, k, v, dst_token0, page_table or None, block_tokens, status or None, stream)
PyObject* decode(PyObject* self_, PyObject* const* a, Py_ssize_t n_args) {
  KVH_ARGS(10);
  const View kv = read_view(r, a[3], a[4], a[6] != Py_None);
  const void* blob = r.device(a[0]);
  const int level = r.narrow(a[1]), n = r.narrow(a[2]), block = r.narrow(a[7]);
  const int64_t at = r.wide(a[5]);
  const int32_t* table = r.words(a[6], 0);
  int32_t* status = r.words(a[8], 0);
  void* stream = read_stream(r, self, a[9]);
  return finish(r, [&] { return self->decode(blob, kv.dt, kv.l, n, kv.c, level, &kv.v, at, table, block, status, stream); });
}

// decode_batch(items, n_items, max_tokens_per_item, k, v, paged, block_tokens, status or None, stream)
PyObject* decode_batch(PyObject* self_, PyObject* const* a, Py_ssize_t n_args) {
  KVH_ARGS(9);
  if (a[5] != Py_True && a[5] != Py_False) r.ok = false;
  const View kv = read_view(r, a[3], a[4], a[5] == Py_True);
  const void* items = r.device(a[0]);
  const int n = r.narrow(a[1]), most = r.narrow(a[2]), block = r.narrow(a[6]);
  int32_t* status = r.words(a[7], n);
  void* stream = read_stream(r, self, a[8]);
  return finish(r, [&] {
    return self->decode_batch(static_cast<const kvh_item*>(items), n, most, kv.dt, kv.l, kv.c, &kv.v, block, status, stream);
  });
}

// encode_kept(k, v, sink, window, level, blob, stream)
PyObject* encode_kept(PyObject* self_, PyObject* const* a, Py_ssize_t n_args) {
  KVH_ARGS(7);
  const View kv = read_view(r, a[0], a[1], false);
  const int sink = r.narrow(a[2]), window = r.narrow(a[3]), level = r.narrow(a[4]);
  void* blob = r.device(a[5]);
  const int64_t cap = r.ok ? r.int_method(a[5], s_numel) : 0;
  void* stream = read_stream(r, self, a[6]);
  return finish(r, [&] {
    return self->encode_kept(&kv.v, kv.dt, kv.l, kv.tokens, kv.c, sink, window, level, blob, (size_t)cap, stream);
  });
}

// decode_kept(blob, level, N, sink, window, k, v, dst_token0, compact, page_table or None, block_tokens, status or None, stream)
PyObject* decode_kept(PyObject* self_, PyObject* const* a, Py_ssize_t n_args) {
  KVH_ARGS(13);
  if (a[8] != Py_True && a[8] != Py_False) r.ok = false;
  const View kv = read_view(r, a[5], a[6], a[9] != Py_None);
  const void* blob = r.device(a[0]);
  const int level = r.narrow(a[1]), n = r.narrow(a[2]), sink = r.narrow(a[3]), window = r.narrow(a[4]), block = r.narrow(a[10]);
  const int64_t at = r.wide(a[7]);
  const int32_t* table = r.words(a[9], 0);
  int32_t* status = r.words(a[11], 0);
  void* stream = read_stream(r, self, a[12]);
  return finish(r, [&] {
    return self->decode_kept(blob, kv.dt, kv.l, n, kv.c, sink, window, level, &kv.v, at, a[8] == Py_True, table, block, status, stream);
  });
}

#if KVH_EXCHANGE
int (*fields_of)(void*, DLTensor*);  // looked up when the module is imported; nullptr where torch does not offer it

enum class Type { kNone, kF16, kBF16, kF32, kI8, kE4M3, kI32, kU8 };

// A tensor's fields.  Strides of dimensions of one entry are of no account.
struct Fields {
  void* p = nullptr;
  Type type = Type::kNone;
  int n = 0;
  int64_t size[4], stride[4];
  bool dense(int d) const { return size[d] <= 1 || stride[d] == 1; }
};

Type type_of(const DLDataType& t) {
  if (t.lanes != 1) return Type::kNone;
  if (t.code == kDLFloat && t.bits == 16) return Type::kF16;
  if (t.code == kDLFloat && t.bits == 32) return Type::kF32;
  if (t.code == kDLBfloat && t.bits == 16) return Type::kBF16;
  if (t.code == kDLInt && t.bits == 8) return Type::kI8;
  if (t.code == kDLInt && t.bits == 32) return Type::kI32;
  if (t.code == kDLUInt && t.bits == 8) return Type::kU8;
  if (t.code == kDLFloat8_e4m3fn && t.bits == 8) return Type::kE4M3;
  return Type::kNone;
}

// `dims` dimensions of a device tensor; None is nothing where that is allowed.
Fields read_fields(Reader& r, PyObject* t, int dims, bool optional = false) {
  Fields f;
  if (!r.ok || (optional && t == Py_None)) return f;
  DLTensor d;
  if (fields_of == nullptr || Py_TYPE(t) != reinterpret_cast<PyTypeObject*>(tensor_type) || fields_of(t, &d) != 0 || d.device.device_type != kDLROCM ||
      d.ndim != dims || d.strides == nullptr || d.data == nullptr) {
    r.ok = false;
    return f;
  }
  f.p = static_cast<char*>(d.data) + d.byte_offset;
  f.type = type_of(d.dtype);
  f.n = dims;
  for (int i = 0; i < dims; ++i) {
    f.size[i] = d.shape[i], f.stride[i] = d.strides[i];
    if (f.size[i] > INT32_MAX || f.size[i] < 1) r.ok = false;
  }
  return f;
}

void expect(Reader& r, bool fine) {
  if (!fine) r.ok = false;
}

// The cache of [l][P][block][c] tensors, as binding.py's _cache takes it.
kvh_cache read_cache(Reader& r, PyObject* kc, PyObject* vc, PyObject* ks, PyObject* vs, int head_dim, Type type) {
  kvh_cache c{};
  const Fields k = read_fields(r, kc, 4), v = read_fields(r, vc, 4), a = read_fields(r, ks, 3, true), b = read_fields(r, vs, 3, true);
  if (!r.ok) return c;
  expect(r, k.type == v.type && (k.type == type || k.type == Type::kI8 || k.type == Type::kE4M3) && head_dim > 0 && k.size[3] % head_dim == 0 && k.dense(3));
  for (int i = 0; i < 4; ++i) expect(r, k.size[i] == v.size[i] && (k.size[i] == 1 || k.stride[i] == v.stride[i]));
  if (!r.ok) return c;
  const int64_t pages = k.size[1], block = k.size[2];
  const int64_t row = block > 1 ? k.stride[2] : pages > 1 ? k.stride[1] : k.size[3];
  expect(r, pages == 1 || k.stride[1] == row * block);
  c.k = k.p, c.v = v.p;
  c.layer_stride = k.size[0] > 1 ? k.stride[0] : 0, c.token_stride = row;
  c.layers = (int32_t)k.size[0], c.pages = (int32_t)pages, c.block_tokens = (int32_t)block, c.heads = (int32_t)(k.size[3] / head_dim), c.head_dim = head_dim;
  c.kind = k.type == type ? KVH_CACHE_16 : k.type == Type::kI8 ? KVH_CACHE_I8 : KVH_CACHE_E4M3;
  if (c.kind == KVH_CACHE_16) {
    expect(r, a.p == nullptr && b.p == nullptr);
  } else {
    const Fields* both[2] = {&a, &b};
    for (const Fields* s : both) {
      expect(r, s->p != nullptr && s->type == Type::kF32);
      if (!r.ok) return c;
      expect(r, s->size[0] == c.layers && s->size[1] == pages && s->size[2] == c.heads && s->dense(2));
      for (int i = 0; i < 2; ++i) expect(r, a.size[i] == 1 || a.stride[i] == s->stride[i]);
    }
    c.k_scale = static_cast<float*>(a.p), c.v_scale = static_cast<float*>(b.p);
    c.scale_layer_stride = c.layers > 1 ? a.stride[0] : 0, c.scale_page_stride = pages > 1 ? a.stride[1] : c.heads;
  }
  return c;
}

int32_t* read_words(Reader& r, PyObject* t, int64_t least, bool optional = false) {
  const Fields f = read_fields(r, t, 1, optional);
  if (!r.ok || f.p == nullptr) return nullptr;
  expect(r, f.type == Type::kI32 && f.dense(0) && f.size[0] >= least);
  return static_cast<int32_t*>(f.p);
}

kvh_requests read_requests(Reader& r, PyObject* starts, PyObject* lens, PyObject* table, PyObject* max_new, int64_t n_tokens) {
  kvh_requests q{};
  const Fields l = read_fields(r, lens, 1), t = read_fields(r, table, 2);
  if (!r.ok) return q;
  expect(r, l.type == Type::kI32 && l.dense(0) && t.type == Type::kI32 && t.dense(1) && t.size[0] >= l.size[0] && n_tokens <= INT32_MAX);
  q.starts = read_words(r, starts, l.size[0] + 1);
  q.lens = static_cast<const int32_t*>(l.p), q.page_table = static_cast<const int32_t*>(t.p);
  q.table_stride = t.size[0] > 1 ? t.stride[0] : t.size[1], q.table_pages = (int32_t)t.size[1];
  q.n_requests = (int32_t)l.size[0], q.max_new = r.narrow(max_new), q.n_tokens = (int32_t)n_tokens;
  return q;
}

// [l][T][channels], or [T][channels] with l = 1.
kvh_rows rows_of(Reader& r, const Fields& f, Type type, int64_t layers, int64_t tokens, int64_t channels) {
  const int d = f.n - 2;
  expect(r, f.type == type && f.size[d] == tokens && f.size[d + 1] == channels && f.dense(d + 1) && (d == 0 || f.size[0] == layers));
  return kvh_rows{f.p, d == 1 && layers > 1 ? f.stride[0] : 0, tokens > 1 ? f.stride[d] : channels};
}

// append(k, v, k_cache, v_cache, starts, lens, page_table, max_new, head_dim, k_scale, v_scale, q, q_out, rotation, positions, pairs, status, stream)
PyObject* append(PyObject* self_, PyObject* const* a, Py_ssize_t n_args) {
  KVH_ARGS(18);
  if (self->append == nullptr) Py_RETURN_NONE;
  const Fields k = read_fields(r, a[0], 3), v = read_fields(r, a[1], 3), q = read_fields(r, a[11], 3, true), o = read_fields(r, a[12], 3, true),
               t = read_fields(r, a[13], 2, true);
  const int head_dim = r.narrow(a[8]);
  if (a[15] != Py_True && a[15] != Py_False) r.ok = false;
  expect(r, r.ok && (k.type == Type::kF16 || k.type == Type::kBF16) && (q.p == nullptr) == (o.p == nullptr));
  kvh_cache c{};
  kvh_requests req{};
  kvh_kv_view kv{};
  kvh_rows from{}, to{};
  kvh_rotation rot{};
  int q_heads = 0;
  if (r.ok) {
    c = read_cache(r, a[2], a[3], a[9], a[10], head_dim, k.type);
    req = read_requests(r, a[4], a[5], a[6], a[7], k.size[1]);
  }
  if (r.ok) {
    const kvh_rows kr = rows_of(r, k, k.type, c.layers, k.size[1], (int64_t)c.heads * head_dim), vr = rows_of(r, v, k.type, c.layers, k.size[1], k.size[2]);
    expect(r, kr.layer_stride == vr.layer_stride && kr.token_stride == vr.token_stride);
    kv = kvh_kv_view{kr.p, vr.p, kr.layer_stride, kr.token_stride};
    if (q.p != nullptr) {
      expect(r, q.size[2] % head_dim == 0);
      q_heads = (int)(q.size[2] / head_dim);
      from = rows_of(r, q, k.type, c.layers, k.size[1], q.size[2]);
      to = rows_of(r, o, k.type, c.layers, k.size[1], q.size[2]);
    }
    rot.positions = read_words(r, a[14], k.size[1], true);
    if (t.p != nullptr) {
      expect(r, t.type == Type::kF32 && t.dense(1));
      rot.table = static_cast<const float*>(t.p), rot.table_stride = t.size[0] > 1 ? t.stride[0] : t.size[1];
      rot.n_positions = (int32_t)t.size[0], rot.rot = (int32_t)t.size[1], rot.pairs = a[15] == Py_True;
    } else {
      expect(r, rot.positions == nullptr);
    }
  }
  int32_t* status = read_words(r, a[16], req.n_requests, true);
  void* stream = read_stream(r, self, a[17]);
  const kvh_dtype dt = k.type == Type::kF16 ? KVH_F16 : KVH_BF16;
  return finish(r, [&] {
    return self->append(&c, &req, dt, &kv, q.p != nullptr ? &from : nullptr, q.p != nullptr ? &to : nullptr, q_heads, t.p != nullptr ? &rot : nullptr, status,
                        stream);
  });
}

// attention(q, k_cache, v_cache, layer, starts, lens, page_table, max_new, head_dim, k_scale, v_scale, scale or None, causal, sink, window, out, lse,
// workspace, status, stream)
PyObject* attention(PyObject* self_, PyObject* const* a, Py_ssize_t n_args) {
  KVH_ARGS(20);
  if (self->attention == nullptr) Py_RETURN_NONE;
  const Fields q = read_fields(r, a[0], 2), o = read_fields(r, a[15], 2), lse = read_fields(r, a[16], 2, true), ws = read_fields(r, a[17], 1);
  const int layer = r.narrow(a[3]), head_dim = r.narrow(a[8]), sink = r.narrow(a[13]), window = r.narrow(a[14]);
  if ((a[12] != Py_True && a[12] != Py_False) || (a[11] != Py_None && !PyFloat_CheckExact(a[11]))) r.ok = false;
  expect(r, r.ok && (q.type == Type::kF16 || q.type == Type::kBF16) && ws.type == Type::kU8 && ws.dense(0) && head_dim > 0 && q.size[1] % head_dim == 0);
  kvh_cache c{};
  kvh_requests req{};
  kvh_rows from{}, to{};
  int q_heads = 0;
  if (r.ok) {
    c = read_cache(r, a[1], a[2], a[9], a[10], head_dim, q.type);
    req = read_requests(r, a[4], a[5], a[6], a[7], q.size[0]);
  }
  if (r.ok) {
    q_heads = (int)(q.size[1] / head_dim);
    from = rows_of(r, q, q.type, 1, q.size[0], q.size[1]);
    to = rows_of(r, o, q.type, 1, q.size[0], q.size[1]);
    if (lse.p != nullptr)
      expect(r, lse.type == Type::kF32 && lse.size[0] == q.size[0] && lse.size[1] == q_heads && lse.dense(1) && (lse.size[0] == 1 || lse.stride[0] == q_heads));
  }
  int32_t* status = read_words(r, a[18], req.n_requests, true);
  void* stream = read_stream(r, self, a[19]);
  const float scale = a[11] == Py_None ? (r.ok ? (float)std::pow((double)head_dim, -0.5) : 0.0f) : (float)PyFloat_AS_DOUBLE(a[11]);
  const kvh_dtype dt = q.type == Type::kF16 ? KVH_F16 : KVH_BF16;
  return finish(r, [&] {
    return self->attention(&c, layer, &req, dt, &from, &to, q_heads, static_cast<float*>(lse.p), scale, a[12] == Py_True, sink, window, ws.p, (size_t)ws.size[0],
                           status, stream);
  });
}

void find_exchange() {
  PyObject* capsule = PyObject_GetAttrString(tensor_type, "__dlpack_c_exchange_api__");
  if (capsule != nullptr && PyCapsule_IsValid(capsule, "dlpack_exchange_api")) {
    const auto* api = static_cast<const DLPackExchangeAPI*>(PyCapsule_GetPointer(capsule, "dlpack_exchange_api"));
    if (api != nullptr && api->header.version.major == DLPACK_MAJOR_VERSION) fields_of = api->dltensor_from_py_object_no_sync;
  }
  Py_XDECREF(capsule);
  PyErr_Clear();
}
#else
// Without the interface these calls are binding.py's.
PyObject* append(PyObject*, PyObject* const*, Py_ssize_t) { Py_RETURN_NONE; }
PyObject* attention(PyObject*, PyObject* const*, Py_ssize_t) { Py_RETURN_NONE; }
void find_exchange() {}
#endif

// Calls(current_device, raw_stream, addresses of the functions in the order of the struct; those of the serving cache may be left out, and its
// calls then go the ctypes way)
PyObject* calls_new(PyTypeObject* type, PyObject* args, PyObject*) {
  PyObject *dev, *raw;
  unsigned long long p[8] = {};
  if (!PyArg_ParseTuple(args, "OOKKKKKK|KK", &dev, &raw, &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7])) return nullptr;
  Calls* c = reinterpret_cast<Calls*>(type->tp_alloc(type, 0));
  if (c == nullptr) return nullptr;
  c->encode = reinterpret_cast<decltype(c->encode)>((uintptr_t)p[0]);
  c->encode_batch = reinterpret_cast<decltype(c->encode_batch)>((uintptr_t)p[1]);
  c->decode = reinterpret_cast<decltype(c->decode)>((uintptr_t)p[2]);
  c->decode_batch = reinterpret_cast<decltype(c->decode_batch)>((uintptr_t)p[3]);
  c->encode_kept = reinterpret_cast<decltype(c->encode_kept)>((uintptr_t)p[4]);
  c->decode_kept = reinterpret_cast<decltype(c->decode_kept)>((uintptr_t)p[5]);
  c->append = reinterpret_cast<decltype(c->append)>((uintptr_t)p[6]);
  c->attention = reinterpret_cast<decltype(c->attention)>((uintptr_t)p[7]);
  Py_INCREF(dev);
  Py_INCREF(raw);
  c->current_device = dev;
  c->raw_stream = raw;
  return reinterpret_cast<PyObject*>(c);
}

void calls_dealloc(PyObject* o) {
  Calls* c = reinterpret_cast<Calls*>(o);
  Py_XDECREF(c->current_device);
  Py_XDECREF(c->raw_stream);
  PyTypeObject* type = Py_TYPE(o);
  type->tp_free(o);
  Py_DECREF(type);
}

#define KVH_METHOD(F) {#F, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(F)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {KVH_METHOD(encode), KVH_METHOD(encode_batch), KVH_METHOD(decode), KVH_METHOD(decode_batch),
                         KVH_METHOD(encode_kept), KVH_METHOD(decode_kept), KVH_METHOD(append), KVH_METHOD(attention), {nullptr, nullptr, 0, nullptr}};
PyType_Slot slots[] = {{Py_tp_new, reinterpret_cast<void*>(calls_new)}, {Py_tp_dealloc, reinterpret_cast<void*>(calls_dealloc)},
                       {Py_tp_methods, methods}, {0, nullptr}};
PyType_Spec spec = {"kvh_fastcall.Calls", sizeof(Calls), 0, Py_TPFLAGS_DEFAULT, slots};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) {
  PyObject* torch = PyImport_ImportModule("torch");
  if (torch == nullptr) return nullptr;
  tensor_type = PyObject_GetAttrString(torch, "Tensor");
  dtype_f16 = PyObject_GetAttrString(torch, "float16");
  dtype_bf16 = PyObject_GetAttrString(torch, "bfloat16");
  dtype_i32 = PyObject_GetAttrString(torch, "int32");
  Py_DECREF(torch);
  if (tensor_type != nullptr) find_exchange();
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_numel = PyUnicode_InternFromString("numel");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  PyObject* m = PyModule_Create(&module);
  PyObject* type = m != nullptr ? PyType_FromSpec(&spec) : nullptr;
  if (PyErr_Occurred() || type == nullptr || PyModule_AddObject(m, "Calls", type) < 0) {
    Py_XDECREF(type);
    Py_XDECREF(m);
    return nullptr;
  }
  return m;
}
