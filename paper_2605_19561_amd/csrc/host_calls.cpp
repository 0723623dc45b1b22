// The calls of the binding that a program makes again and again, marshalled in C++ (module _host): torq_linear,
// torq_rotate_quantize (and _fmt), torq_block_gram (and _positions), torq_code_histogram, torq_block_tables, torq_cache_append,
// torq_paged_attention and torq_add_rms_norm.  The kernels of the smallest of
// them take 3 to 6 us, the interpreter 8 to 13 for the attribute look-ups, checks, allocations and a ctypes call.  One row
// through a 4096 x 4096 layer, a call among others: 10.2 us -> 5.6 or 6.4 from one process to the next (the kernel, replayed from a
// graph, 5.7).
//
// A function here takes a call only where everything about it is plain: exact tensors (no subclass), the shapes, types and
// layout that the library takes.  Anything else it leaves alone, returns None, and binding.py's own Python goes through the
// arguments one by one and raises what it always raised.  Same allocations, same C ABI, the status checked by the same
// function; no state but the addresses handed over in bind().
#include <Python.h>

#include <torch/csrc/Stream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>

#include <algorithm>
#include <cstdint>
#include <optional>

#include "../../include/torq.h"

namespace {

using at::Tensor;

// the library's entry points and the binding's two functions
int (*f_linear)(const void *, const void *, const void *, const void *, void *, int64_t, int64_t, void *, size_t, void *);
size_t (*f_linear_bytes)(int64_t, int64_t, int);
int (*f_rotate_quantize)(const void *, const void *, int64_t, void *, void *, void *);
int (*f_rotate_quantize_fmt)(const void *, const void *, int64_t, int, float, void *, void *, void *);
int (*f_gram)(const void *, int64_t, int, int, void *, void *, size_t, void *);
int (*f_gram_positions)(const void *, int64_t, int, int, void *, void *, size_t, void *);
size_t (*f_gram_bytes)(int);
int (*f_histogram)(const void *, int64_t, int, void *, void *, size_t, void *);
size_t (*f_histogram_bytes)();
decltype(&torq_block_tables) f_tables;
decltype(&torq_cache_append) f_append;
decltype(&torq_paged_attention) f_attention;
decltype(&torq_paged_attention_workspace_bytes) f_attention_bytes;
decltype(&torq_add_rms_norm) f_norm;
PyObject *py_stream, *py_check;
PyObject *s_handle, *s_kv_handle, *s_kv_device, *s_value, *s_d;

struct NotPlain {};

const Tensor &tensor(PyObject *o) {
  if (!THPVariable_CheckExact(o)) throw NotPlain{};
  return THPVariable_Unpack(o);
}
void *address(const Tensor &t, at::ScalarType type) {
  if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous()) throw NotPlain{};
  return t.data_ptr();
}
int64_t integer(PyObject *o) {
  if (!PyLong_CheckExact(o)) throw NotPlain{};
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw NotPlain{};
  return v;
}
int small_integer(PyObject *o) {
  const int64_t v = integer(o);
  if (v < 0 || v > 0x7FFFFFFF) throw NotPlain{};
  return (int)v;
}
struct Ref {
  PyObject *p;
  explicit Ref(PyObject *o) : p(o) {
    if (!p) throw NotPlain{};
  }
  ~Ref() { Py_DECREF(p); }
  Ref(const Ref &) = delete;
  Ref &operator=(const Ref &) = delete;
};
// an address held by a Python integer
void *pointer(PyObject *o) {
  if (!PyLong_Check(o)) throw NotPlain{};
  void *p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw NotPlain{};
  return p;
}
// an attribute that is a ctypes pointer: Rotation.handle (None once it is closed), KVCache.kv_handle
void *handle_of(PyObject *owner, PyObject *name) {
  Ref h(PyObject_GetAttr(owner, name));
  if (h.p == Py_None) throw NotPlain{};
  Ref v(PyObject_GetAttr(h.p, s_value));
  return pointer(v.p);
}
int64_t d_of(PyObject *rot) {
  Ref d(PyObject_GetAttr(rot, s_d));
  return integer(d.p);
}
void *stream_of(PyObject *stream) {
  Ref s(PyObject_CallOneArg(py_stream, stream));
  return pointer(s.p);
}

// The stream of a call that allocates its own workspace: that goes back to the allocator when the call returns, ahead of the
// kernels that use it, so a stream that is not the one it is allocated on has to be known there.
std::optional<c10::Stream> user_of(PyObject *stream, const Tensor *workspace) {
  if (workspace || stream == Py_None) return std::nullopt;
  if (!THPStream_Check(stream)) throw NotPlain{};
  const THPStream *s = reinterpret_cast<const THPStream *>(stream);
  return c10::Stream::unpack3(s->stream_id, (c10::DeviceIndex)s->device_index, (c10::DeviceType)s->device_type);
}

// allocations and launches without the interpreter's lock, as ctypes and torch's own functions do them
struct Unlocked {
  PyThreadState *state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

Tensor given_or_new(const Tensor *given, const Tensor &like, at::IntArrayRef sizes, at::ScalarType type) {
  return given ? *given : at::empty(sizes, like.options().dtype(type));
}
Tensor scratch(const Tensor *given, const Tensor &like, int64_t bytes, const std::optional<c10::Stream> &user) {
  if (given) return *given;
  Tensor t = like.new_empty({bytes}, like.options().dtype(at::kByte));
  if (user) t.record_stream(*user);
  return t;
}
const Tensor *optional(PyObject *o) { return o == Py_None ? nullptr : &tensor(o); }
PyObject *wrapped(PyObject *given, const Tensor &t) {
  if (given == Py_None) return THPVariable_Wrap(t);
  Py_INCREF(given);
  return given;
}
// None of the arguments has been used if this returns nullptr without an error set
bool ok(int status, const char *what) {
  if (status == 0) return true;
  PyObject *r = PyObject_CallFunction(py_check, "is", status, what);
  Py_XDECREF(r);
  return false;
}

template <class F>
PyObject *plain_or_none(F &&f) {
  try {
    return f();
  } catch (...) {
    // (an interrupt that arrived while the interpreter was asked for something says nothing about the arguments)
    if (PyErr_Occurred() && !PyErr_ExceptionMatches(PyExc_Exception)) return nullptr;
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// linear(rot, x, W_q, W_s, out, workspace, stream)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return plain_or_none([&]() -> PyObject * {
    if (n != 7) throw NotPlain{};
    const Tensor &x = tensor(a[1]), &W_q = tensor(a[2]), &W_s = tensor(a[3]);
    const Tensor *out_in = optional(a[4]), *ws_in = optional(a[5]);
    if (x.dim() != 2 || W_q.dim() != 2 || W_s.dim() != 2) throw NotPlain{};
    const int64_t M = x.size(0), d = x.size(1), N = W_q.size(0);
    if (d != d_of(a[0]) || W_q.size(1) != d / 2 || W_s.size(0) != N || W_s.size(1) != d / 32) throw NotPlain{};
    void *const handle = handle_of(a[0], s_handle), *const xp = address(x, at::kBFloat16), *const qp = address(W_q, at::kByte),
                *const sp = address(W_s, at::kByte), *const stream = stream_of(a[6]);
    const std::optional<c10::Stream> user = user_of(a[6], ws_in);
    Tensor out;
    int status;
    {
      Unlocked unlocked;
      const Tensor ws = scratch(ws_in, x, ws_in ? 1 : std::max<int64_t>((int64_t)f_linear_bytes(M, N, (int)d), 1), user);
      out = given_or_new(out_in, x, {M, N}, at::kBFloat16);
      status = f_linear(handle, xp, qp, sp, address(out, at::kBFloat16), M, N, address(ws, at::kByte), (size_t)ws.numel(), stream);
    }
    return ok(status, "torq_linear") ? wrapped(a[4], out) : nullptr;
  });
}

// rotate_quantize(rot, x, format or None, global_scale, codes, scales, stream)
PyObject *rotate_quantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return plain_or_none([&]() -> PyObject * {
    if (n != 7) throw NotPlain{};
    const Tensor &x = tensor(a[1]);
    const Tensor *codes_in = optional(a[4]), *scales_in = optional(a[5]);
    const bool with_format = a[2] != Py_None;
    const int format = with_format ? small_integer(a[2]) : 0;
    if (!PyFloat_CheckExact(a[3]) || x.dim() != 2) throw NotPlain{};
    const float global_scale = (float)PyFloat_AS_DOUBLE(a[3]);
    const int64_t M = x.size(0), d = x.size(1);
    if (d != d_of(a[0])) throw NotPlain{};
    void *const handle = handle_of(a[0], s_handle), *const xp = address(x, at::kBFloat16), *const stream = stream_of(a[6]);
    Tensor codes, scales;
    int status;
    {
      Unlocked unlocked;
      codes = given_or_new(codes_in, x, {M, d / 2}, at::kByte);
      scales = given_or_new(scales_in, x, {M, format == 2 ? d / 16 : d / 32}, at::kByte);
      void *const cp = address(codes, at::kByte), *const sp = address(scales, at::kByte);
      status = with_format ? f_rotate_quantize_fmt(handle, xp, M, format, global_scale, cp, sp, stream)
                           : f_rotate_quantize(handle, xp, M, cp, sp, stream);
    }
    if (!ok(status, with_format ? "torq_rotate_quantize_fmt" : "torq_rotate_quantize")) return nullptr;
    PyObject *c = wrapped(a[4], codes), *s = wrapped(a[5], scales), *pair = c && s ? PyTuple_Pack(2, c, s) : nullptr;
    Py_XDECREF(c);
    Py_XDECREF(s);
    return pair;
  });
}

// gram(x, G, positions, Sigma, workspace, stream)
PyObject *gram(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return plain_or_none([&]() -> PyObject * {
    if (n != 6) throw NotPlain{};
    const Tensor &x = tensor(a[0]);
    const Tensor *sigma_in = optional(a[3]), *ws_in = optional(a[4]);
    const int G = small_integer(a[1]);
    const bool positions = a[2] == Py_True;
    if (x.dim() != 2 || x.size(1) > 0x7FFFFFFF) throw NotPlain{};
    const int64_t M = x.size(0), d = x.size(1);
    void *const xp = address(x, at::kBFloat16), *const stream = stream_of(a[5]);
    const std::optional<c10::Stream> user = user_of(a[5], ws_in);
    Tensor sigma;
    int status;
    {
      Unlocked unlocked;
      const int64_t shape[3] = {32, G, G};
      sigma = given_or_new(sigma_in, x, positions ? at::IntArrayRef(shape, 3) : at::IntArrayRef(shape + 1, 2), at::kDouble);
      const Tensor ws = scratch(ws_in, x, ws_in ? 1 : std::max<int64_t>((int64_t)f_gram_bytes(G), 16), user);
      status = (positions ? f_gram_positions : f_gram)(xp, M, (int)d, G, address(sigma, at::kDouble), address(ws, at::kByte),
                                                       (size_t)ws.numel(), stream);
    }
    return ok(status, positions ? "torq_block_gram_positions" : "torq_block_gram") ? wrapped(a[3], sigma) : nullptr;
  });
}

// histogram(codes, d, counts, workspace, stream)
PyObject *histogram(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return plain_or_none([&]() -> PyObject * {
    if (n != 5) throw NotPlain{};
    const Tensor &codes = tensor(a[0]);
    const Tensor *counts_in = optional(a[2]), *ws_in = optional(a[3]);
    const int d = small_integer(a[1]);
    if (codes.dim() != 2 || codes.size(1) * 2 != d) throw NotPlain{};
    void *const cp = address(codes, at::kByte), *const stream = stream_of(a[4]);
    const std::optional<c10::Stream> user = user_of(a[4], ws_in);
    Tensor counts;
    int status;
    {
      Unlocked unlocked;
      counts = given_or_new(counts_in, codes, {32, 8}, at::kLong);
      const Tensor ws = scratch(ws_in, codes, ws_in ? 1 : (int64_t)f_histogram_bytes(), user);
      status = f_histogram(cp, codes.size(0), d, address(counts, at::kLong), address(ws, at::kByte), (size_t)ws.numel(), stream);
    }
    return ok(status, "torq_code_histogram") ? wrapped(a[2], counts) : nullptr;
  });
}

// a tensor of that type and number of dimensions, contiguous along the last
void *rows(const Tensor &t, at::ScalarType type, int64_t dims) {
  if (!t.is_cuda() || t.scalar_type() != type || t.dim() != dims || (t.numel() && t.size(dims - 1) > 1 && t.stride(dims - 1) != 1)) throw NotPlain{};
  return t.data_ptr();
}
void shape(const Tensor &t, at::IntArrayRef sizes) {
  if (t.sizes() != sizes) throw NotPlain{};
}
// a dimension of one entry has no stride to speak of
int64_t step(const Tensor &t, int64_t dim) { return t.size(dim) > 1 ? t.stride(dim) : 0; }
double number(PyObject *o) {
  if (!PyFloat_CheckExact(o)) throw NotPlain{};
  return PyFloat_AS_DOUBLE(o);
}
// a cache on the GPU of the tensor that it is used with (one on the host has no handle)
const torq_kv_cache_t *cache_of(PyObject *cache, const Tensor &with_it) {
  const torq_kv_cache_t *c = static_cast<const torq_kv_cache_t *>(handle_of(cache, s_kv_handle));
  Ref device(PyObject_GetAttr(cache, s_kv_device));
  if (!c || integer(device.p) != with_it.get_device()) throw NotPlain{};
  return c;
}
PyObject *packed(std::initializer_list<PyObject *> items) {
  PyObject *t = PyTuple_New((Py_ssize_t)items.size());
  Py_ssize_t i = 0;
  bool fine = t != nullptr;
  for (PyObject *o : items) {
    fine = fine && o;
    if (t && o) PyTuple_SET_ITEM(t, i++, o);
    else Py_XDECREF(o);
  }
  if (!fine) Py_CLEAR(t);
  return t;
}

// block_tables(held, lengths, free_pages, cursor, block_tables, page_size, tokens, slots, cursor_out, stream)
PyObject *block_tables(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return plain_or_none([&]() -> PyObject * {
    if (n != 10) throw NotPlain{};
    const Tensor &held = tensor(a[0]), &lengths = tensor(a[1]), &pages = tensor(a[2]), &cursor = tensor(a[3]), &tables = tensor(a[4]);
    const Tensor *slots_in = optional(a[7]), *cursor_in = optional(a[8]);
    const int page_size = small_integer(a[5]);
    const int64_t tokens = integer(a[6]);
    int32_t *const tp = static_cast<int32_t *>(rows(tables, at::kInt, 2));
    const int64_t B = tables.size(0), width = tables.size(1);
    shape(held, {B});
    shape(lengths, {B});
    shape(cursor, {1});
    if (pages.dim() != 1 || width > 0x7FFFFFFF || tokens < 0) throw NotPlain{};
    if (slots_in) shape(*slots_in, {tokens});
    if (cursor_in) shape(*cursor_in, {1});
    auto ints = [](const Tensor &t) { return static_cast<int32_t *>(address(t, at::kInt)); };
    const int32_t *const hp = ints(held), *const lp = ints(lengths), *const fp = ints(pages), *const cp = ints(cursor);
    void *const stream_p = stream_of(a[9]);
    Tensor slots, after;
    int status;
    {
      Unlocked unlocked;
      slots = given_or_new(slots_in, held, {tokens}, at::kLong);
      after = given_or_new(cursor_in, held, {1}, at::kInt);
      status = f_tables(hp, lp, B, fp, pages.numel(), cp, ints(after), tp, B > 1 ? tables.stride(0) : width, (int)width, page_size,
                        static_cast<int64_t *>(address(slots, at::kLong)), tokens, stream_p);
    }
    return ok(status, "torq_block_tables") ? packed({wrapped(a[7], slots), wrapped(a[8], after)}) : nullptr;
  });
}

// cache_append(cache, key, value, slots, stream): True
PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return plain_or_none([&]() -> PyObject * {
    if (n != 5) throw NotPlain{};
    const Tensor &key = tensor(a[1]), &value = tensor(a[2]), &slots = tensor(a[3]);
    const torq_kv_cache_t *const cache = cache_of(a[0], key);
    const void *const kp = rows(key, at::kBFloat16, 3), *const vp = rows(value, at::kBFloat16, 3);
    const int64_t *const sp = static_cast<const int64_t *>(address(slots, at::kLong)), T = slots.numel();
    shape(slots, {T});
    shape(key, {T, cache->heads, cache->head_dim});
    shape(value, key.sizes());
    void *const stream_p = stream_of(a[4]);
    int status;
    {
      Unlocked unlocked;
      status = f_append(cache, kp, step(key, 0), step(key, 1), vp, step(value, 0), step(value, 1), sp, T, stream_p);
    }
    if (!ok(status, "torq_cache_append")) return nullptr;
    Py_RETURN_TRUE;
  });
}

// paged_attention(q, cache, block_tables, lengths, scale, out, workspace, stream)
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return plain_or_none([&]() -> PyObject * {
    if (n != 8) throw NotPlain{};
    const Tensor &q = tensor(a[0]), &tables = tensor(a[2]), &lengths = tensor(a[3]);
    const torq_kv_cache_t *const cache = cache_of(a[1], q);
    const float scale = (float)number(a[4]);
    const Tensor *out_in = optional(a[5]), *ws_in = optional(a[6]);
    const void *const qp = rows(q, at::kBFloat16, 3);
    const int32_t *const tp = static_cast<const int32_t *>(rows(tables, at::kInt, 2)), *const lp = static_cast<const int32_t *>(address(lengths, at::kInt));
    const int64_t B = q.size(0), heads = q.size(1), width = tables.size(1);
    shape(lengths, {B});
    shape(q, {B, heads, cache->head_dim});
    if (tables.size(0) != B || heads > 0x7FFFFFFF || width > 0x7FFFFFFF) throw NotPlain{};
    if (out_in) shape(*out_in, q.sizes());
    void *const stream_p = stream_of(a[7]);
    const std::optional<c10::Stream> user = user_of(a[7], ws_in);
    Tensor out;
    int status;
    {
      Unlocked unlocked;
      const Tensor ws = scratch(ws_in, q, ws_in ? 1 : std::max<int64_t>((int64_t)f_attention_bytes(cache, (int)heads, B, (int)width), 16), user);
      out = given_or_new(out_in, q, q.sizes(), at::kBFloat16);
      status = f_attention(cache, qp, step(q, 0), step(q, 1), (int)heads, tp, B > 1 ? tables.stride(0) : width, (int)width, lp, B, scale,
                           address(out, at::kBFloat16), address(ws, at::kByte), (size_t)ws.numel(), stream_p);
    }
    return ok(status, "torq_paged_attention") ? wrapped(a[5], out) : nullptr;
  });
}

// add_rms_norm(x, residual, weight, eps, format, residual_out, out, scales, stream)
PyObject *add_rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return plain_or_none([&]() -> PyObject * {
    if (n != 9) throw NotPlain{};
    const Tensor &x = tensor(a[0]), &weight = tensor(a[2]);
    const Tensor *residual = optional(a[1]), *sum_in = optional(a[5]), *out_in = optional(a[6]), *scales_in = optional(a[7]);
    const float eps = (float)number(a[3]);
    const int format = small_integer(a[4]);
    const bool mx = format == TORQ_FMT_MXFP8;
    if (x.dim() != 2 || x.size(1) > 0x7FFFFFFF || (sum_in && !residual) || (scales_in && !mx)) throw NotPlain{};
    const int64_t M = x.size(0), d = x.size(1);
    shape(weight, {d});
    if (residual) shape(*residual, {M, d});
    if (sum_in) shape(*sum_in, {M, d});
    if (out_in) shape(*out_in, {M, d});
    if (scales_in) shape(*scales_in, {M, d / 32});
    const void *const xp = address(x, at::kBFloat16), *const wp = address(weight, at::kBFloat16);
    const void *const rp = residual ? address(*residual, at::kBFloat16) : nullptr;
    void *const stream_p = stream_of(a[8]);
    Tensor sum, out, scales;
    int status;
    {
      Unlocked unlocked;
      if (residual) sum = given_or_new(sum_in, x, {M, d}, at::kBFloat16);
      out = given_or_new(out_in, x, {M, d}, mx ? at::kFloat8_e4m3fn : at::kBFloat16);
      if (mx) scales = given_or_new(scales_in, x, {M, d / 32}, at::kFloat8_e8m0fnu);
      status = f_norm(xp, rp, wp, M, (int)d, eps, format, residual ? address(sum, at::kBFloat16) : nullptr,
                      address(out, mx ? at::kFloat8_e4m3fn : at::kBFloat16),
                      mx ? static_cast<uint8_t *>(address(scales, at::kFloat8_e8m0fnu)) : nullptr, stream_p);
    }
    if (!ok(status, "torq_add_rms_norm")) return nullptr;
    auto or_none = [](bool there, PyObject *given, const Tensor &t) {
      if (there) return wrapped(given, t);
      Py_INCREF(Py_None);
      return Py_None;
    };
    return packed({wrapped(a[6], out), or_none(mx, a[7], scales), or_none(residual != nullptr, a[5], sum)});
  });
}

// bind({entry point: address}, stream function, check function)
PyObject *bind(PyObject *, PyObject *args) {
  PyObject *entries, *stream, *check;
  if (!PyArg_ParseTuple(args, "O!OO", &PyDict_Type, &entries, &stream, &check)) return nullptr;
#define TORQ_BIND(VAR_, NAME_)                                                                    \
  {                                                                                               \
    PyObject *v = PyDict_GetItemString(entries, NAME_);                                           \
    void *p = v ? PyLong_AsVoidPtr(v) : nullptr;                                                  \
    if (!p) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_KeyError, "%s", NAME_);        \
    VAR_ = reinterpret_cast<decltype(VAR_)>(p);                                                   \
  }
  TORQ_BIND(f_linear, "torq_linear")
  TORQ_BIND(f_linear_bytes, "torq_linear_workspace_bytes_n")
  TORQ_BIND(f_rotate_quantize, "torq_rotate_quantize")
  TORQ_BIND(f_rotate_quantize_fmt, "torq_rotate_quantize_fmt")
  TORQ_BIND(f_gram, "torq_block_gram")
  TORQ_BIND(f_gram_positions, "torq_block_gram_positions")
  TORQ_BIND(f_gram_bytes, "torq_block_gram_workspace_bytes")
  TORQ_BIND(f_histogram, "torq_code_histogram")
  TORQ_BIND(f_histogram_bytes, "torq_code_histogram_workspace_bytes")
  TORQ_BIND(f_tables, "torq_block_tables")
  TORQ_BIND(f_append, "torq_cache_append")
  TORQ_BIND(f_attention, "torq_paged_attention")
  TORQ_BIND(f_attention_bytes, "torq_paged_attention_workspace_bytes")
  TORQ_BIND(f_norm, "torq_add_rms_norm")
#undef TORQ_BIND
  Py_INCREF(stream);
  Py_INCREF(check);
  Py_XDECREF(py_stream);
  Py_XDECREF(py_check);
  py_stream = stream;
  py_check = check;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"rotate_quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotate_quantize)), METH_FASTCALL, nullptr},
    {"gram", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gram)), METH_FASTCALL, nullptr},
    {"histogram", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(histogram)), METH_FASTCALL, nullptr},
    {"block_tables", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(block_tables)), METH_FASTCALL, nullptr},
    {"cache_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_append)), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_attention)), METH_FASTCALL, nullptr},
    {"add_rms_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(add_rms_norm)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() {
  s_handle = PyUnicode_InternFromString("handle");
  s_kv_handle = PyUnicode_InternFromString("kv_handle");
  s_kv_device = PyUnicode_InternFromString("kv_device");
  s_value = PyUnicode_InternFromString("value");
  s_d = PyUnicode_InternFromString("d");
  if (!s_handle || !s_kv_handle || !s_kv_device || !s_value || !s_d) return nullptr;
  PyObject *m = PyModule_Create(&module);
  // (binding.py binds no module built against another torch)
  if (m && PyModule_AddStringConstant(m, "torch_version", TORQ_TORCH_VERSION) != 0) Py_CLEAR(m);
  return m;
}
