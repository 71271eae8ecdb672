// Argument marshalling of the Python entry points (CPython C API): tensors to device pointers, shapes to counts, the
// current stream to its handle, then the C-ABI call with the interpreter lock released.  Same conversions as ctypes makes.
//
// Why native.  A call of a small step is shorter on the GPU than its marshalling was through ctypes (host time per call, one
// sequence of 137 keys: 8.2 us against 4.7 us of kernel): seven data_ptr calls, two shapes, a stream object and the
// conversion of 15 arguments cost 5 us, where the launch itself costs 2 to 3.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <pthread.h>
#include <stdint.h>

#include <vector>

#include "shiftattn.h"

namespace {

struct Entry {
  const char *name;
  void *fn;
};
enum {
  kAppend, kPrefill, kChunkStep, kDecode, kDecodeStatic, kDecodeStep, kRequired,  // a library without the others can be bound, and called for these
  kCross = kRequired, kNormRope, kReserve, kFork, kRelease, kCompact, kCopy, kEntries
};
Entry entries[kEntries] = {{"sp_kv_append", nullptr},   {"sp_attn_prefill", nullptr},       {"sp_chunk_step", nullptr},
                           {"sp_attn_decode", nullptr}, {"sp_attn_decode_static", nullptr}, {"sp_decode_step", nullptr},
                           {"sp_attn_cross", nullptr},  {"sp_norm_rope_append", nullptr},   {"sp_pages_reserve", nullptr},
                           {"sp_pages_fork", nullptr},  {"sp_pages_release", nullptr},      {"sp_pages_compact", nullptr},
                           {"sp_pages_copy", nullptr}};
PyObject *s_stride, *s_data_ptr, *s_shape, *s_numel, *s_element_size, *s_cuda_stream, *s_desc, *s_value, *s_as_parameter;
PyObject *argument_error, *c_int32, *desc_type, *table_type;  // ctypes.ArgumentError, ctypes.c_int32, sp_cache_desc, sp_page_table
PyObject *get_device, *get_stream, *first_stream;  // torch's raw accessors; the public one, for the first call of the process
bool stream_used = false;  // the public accessor has been called in this process

// Every helper returns false with a Python exception set.
bool pointer(PyObject *t, void **p) {
  *p = nullptr;
  if (t == Py_None) return true;
  PyObject *v = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!v) return false;
  *p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !(*p == nullptr && PyErr_Occurred());
}

// What ctypes takes for a c_int32: one itself, an integer (out-of-range values keep their low bits), or an object that names either
// of them in _as_parameter_.
bool int32(PyObject *o, int32_t *out) {
  PyObject *v = PyFloat_Check(o) ? nullptr : PyNumber_Index(o);
  if (!v) {
    PyErr_Clear();
    const int own = PyObject_IsInstance(o, c_int32);
    PyObject *inner = own < 0 ? nullptr : PyObject_GetAttr(o, own ? s_value : s_as_parameter);
    if (!inner) {
      PyErr_Clear();
      PyErr_SetString(argument_error, "wrong type");
      return false;
    }
    const bool deep = Py_EnterRecursiveCall(" while converting an argument") != 0;
    const bool ok = !deep && int32(inner, out);
    if (!deep) Py_LeaveRecursiveCall();
    Py_DECREF(inner);
    return ok;
  }
  *out = (int32_t)PyLong_AsUnsignedLongMask(v);
  Py_DECREF(v);
  return true;
}

bool dims(PyObject *t, int32_t *out, Py_ssize_t n, bool exactly) {  // the first n sizes
  PyObject *shape = PyObject_GetAttr(t, s_shape);
  if (!shape) return false;
  PyObject *fast = PySequence_Fast(shape, "shape is not a sequence");
  Py_DECREF(shape);
  if (!fast) return false;
  const Py_ssize_t have = PySequence_Fast_GET_SIZE(fast);
  bool ok = have >= n && !(exactly && have > n);
  if (!ok) {
    if (exactly) PyErr_Format(PyExc_ValueError, "expected %zd sizes, got %zd", n, have);
    else PyErr_SetString(PyExc_IndexError, "tuple index out of range");
  }
  for (Py_ssize_t i = 0; ok && i < n; ++i) ok = int32(PySequence_Fast_GET_ITEM(fast, i), out + i);
  Py_DECREF(fast);
  return ok;
}

bool steps_of(PyObject *t, int64_t *out, Py_ssize_t n) {
  PyObject *s = PyObject_CallMethodNoArgs(t, s_stride);
  PyObject *fast = s ? PySequence_Fast(s, "stride is not a sequence") : nullptr;
  Py_XDECREF(s);
  if (!fast) return false;
  for (Py_ssize_t i = 0; i < n; ++i) out[i] = i < PySequence_Fast_GET_SIZE(fast) ? PyLong_AsLongLong(PySequence_Fast_GET_ITEM(fast, i)) : 0;
  Py_DECREF(fast);
  return !PyErr_Occurred();
}

// A matrix of these sizes and strides whose rows follow each other; an empty one does whatever its strides say.
bool contiguous(const int32_t *size, const int64_t *step) {
  return size[0] == 0 || size[1] == 0 || ((size[1] == 1 || step[1] == 1) && (size[0] == 1 || step[0] == size[1]));
}

// Elements of the width that is read: whole numbers of 4 bytes (torch's own have 8), angles of 4, weights of 2.
bool sized(PyObject *t, const char *name, long bytes) {
  PyObject *e = PyObject_CallMethodNoArgs(t, s_element_size);
  if (!e) return false;
  const long have = PyLong_AsLong(e);
  Py_DECREF(e);
  if (have == bytes) return true;
  if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s: elements of %ld bytes, not %ld", name, bytes, have);
  return false;
}

// A list of n elements that follow each other; n -1: any number, which it becomes.
bool list_of(PyObject *t, const char *name, long bytes, int32_t *n) {
  int32_t size;
  int64_t step = 1;
  if (!dims(t, &size, 1, true) || !sized(t, name, bytes) || (size > 1 && !steps_of(t, &step, 1))) return false;
  if (step != 1) return PyErr_Format(PyExc_ValueError, "%s: not contiguous", name), false;
  if (*n >= 0 && size != *n) return PyErr_Format(PyExc_ValueError, "%s: %d entries, not %d", name, (int)size, (int)*n), false;
  *n = size;
  return true;
}

bool bytes_of(PyObject *t, size_t *out) {
  *out = 0;
  if (t == Py_None) return true;
  PyObject *n = PyObject_CallMethodNoArgs(t, s_numel), *e = n ? PyObject_CallMethodNoArgs(t, s_element_size) : nullptr;
  PyObject *b = e ? PyNumber_Multiply(n, e) : nullptr;
  if (b) *out = PyLong_AsSize_t(b);
  Py_XDECREF(n);
  Py_XDECREF(e);
  Py_XDECREF(b);
  return b && !(*out == (size_t)-1 && PyErr_Occurred());
}

bool stream_of(PyObject *s, void **out) {
  PyObject *v = nullptr;
  if (s == Py_None && stream_used) {
    PyObject *dev = PyObject_CallNoArgs(get_device);
    if (!dev) return false;
    v = PyObject_CallOneArg(get_stream, dev);
    Py_DECREF(dev);
  } else {
    PyObject *own = nullptr;
    if (s == Py_None) {  // the public accessor initialises torch's device state, or says why it cannot
      own = s = PyObject_CallNoArgs(first_stream);
      if (!s) return false;
      stream_used = true;
    }
    v = PyObject_GetAttr(s, s_cuda_stream);
    if (!v && PyErr_ExceptionMatches(PyExc_AttributeError)) {
      PyErr_Clear();
      v = PyNumber_Long(s);
    }
    Py_XDECREF(own);
  }
  if (!v) return false;
  *out = v == Py_None ? nullptr : PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !(*out == nullptr && PyErr_Occurred());
}

bool scale_of(PyObject *o, float *out) {
  PyObject *v = PyNumber_Float(o);
  if (!v) return false;
  *out = (float)PyFloat_AS_DOUBLE(v);
  Py_DECREF(v);
  return true;
}

// At least n counters of 32 bits.
bool counters(PyObject *t, const char *name, size_t n) {
  size_t bytes;
  if (t == Py_None) return true;  // the library says whether it takes none
  if (!sized(t, name, 4) || !bytes_of(t, &bytes)) return false;
  if (bytes < 4 * n) return PyErr_Format(PyExc_ValueError, "%s: at least %zu entries", name, n), false;
  return true;
}

struct Desc {  // cache.desc or table.desc, a ctypes structure: its memory
  Py_buffer view;
  bool held = false;
  bool take(PyObject *cache, PyObject *type = desc_type, const char *otherwise = "cache.desc is not a cache descriptor") {
    PyObject *d = PyObject_GetAttr(cache, s_desc);
    if (!d) return false;
    const int is = type ? PyObject_IsInstance(d, type) : 0;
    if (is > 0) held = PyObject_GetBuffer(d, &view, PyBUF_SIMPLE) == 0;
    else if (is == 0) PyErr_SetString(argument_error, otherwise);
    Py_DECREF(d);
    return held;
  }
  bool take_table(PyObject *table) { return take(table, table_type, "table.desc is not a page table"); }
  const sp_cache_desc *get() const { return (const sp_cache_desc *)view.buf; }
  const sp_page_table *table() const { return (const sp_page_table *)view.buf; }
  ~Desc() {
    if (held) PyBuffer_Release(&view);
  }
};

bool count(const char *name, Py_ssize_t have, Py_ssize_t want, int entry = kAppend) {
  if (have == want && entries[entry].fn) return true;
  PyErr_Format(PyExc_TypeError, entries[entry].fn ? "%s: %zd arguments, not %zd" : "%s: the library is not bound", name, want, have);
  return false;
}

template <typename Call>
PyObject *finish(Call call) {  // the status
  int status;
  Py_BEGIN_ALLOW_THREADS;
  status = call();
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(status);
}

// (cache, k_new, v_new, cu_seqlens_new, ctx_lens, block_table, stream)
PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[5], *stream;
  int32_t table[2], total;
  if (!count("kv_append", n, 7) || !dims(a[5], table, 2, true) || !dims(a[1], &total, 1, false) || !desc.take(a[0])) return nullptr;
  for (int i = 0; i < 5; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!stream_of(a[6], &stream)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_kv_append))entries[kAppend].fn)(desc.get(), p[0], p[1], (const int32_t *)p[2], (const int32_t *)p[3],
                                                          (const int32_t *)p[4], table[0], table[1], total, stream);
  });
}

// (cache, q, out, cu_seqlens_q, ctx_lens, block_table, max_q_len, max_kv_len, scale, causal, workspace, stream)
PyObject *attn_prefill(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[5], *ws, *stream;
  int32_t table[2], q[2], max_q, max_kv, causal;
  float scale;
  size_t ws_bytes;
  if (!count("attn_prefill", n, 12) || !dims(a[5], table, 2, true) || !dims(a[1], q, 2, false) || !bytes_of(a[10], &ws_bytes) || !desc.take(a[0]))
    return nullptr;
  for (int i = 0; i < 5; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!scale_of(a[8], &scale) || !pointer(a[10], &ws) || !stream_of(a[11], &stream) || !int32(a[6], &max_q) || !int32(a[7], &max_kv) ||
      !int32(a[9], &causal))
    return nullptr;
  return finish([&] {
    return ((decltype(&sp_attn_prefill))entries[kPrefill].fn)(desc.get(), p[0], p[1], (const int32_t *)p[2], (const int32_t *)p[3],
                                                              (const int32_t *)p[4], table[0], table[1], q[0], max_q, max_kv, q[1], scale, causal,
                                                              ws, ws_bytes, stream);
  });
}

// (cache, k_new, v_new, q, out, cu_seqlens_q, ctx_lens, block_table, max_q_len, max_kv_len, scale, workspace, stream)
PyObject *chunk_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[7], *ws, *stream;
  int32_t table[2], q[2], max_q, max_kv;
  float scale;
  size_t ws_bytes;
  if (!count("chunk_step", n, 13) || !dims(a[7], table, 2, true) || !dims(a[3], q, 2, false) || !bytes_of(a[11], &ws_bytes) || !desc.take(a[0]))
    return nullptr;
  for (int i = 0; i < 7; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!scale_of(a[10], &scale) || !pointer(a[11], &ws) || !stream_of(a[12], &stream) || !int32(a[8], &max_q) || !int32(a[9], &max_kv)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_chunk_step))entries[kChunkStep].fn)(desc.get(), p[0], p[1], p[2], p[3], (const int32_t *)p[4], (const int32_t *)p[5],
                                                              (const int32_t *)p[6], table[0], table[1], q[0], max_q, max_kv, q[1], scale, ws,
                                                              ws_bytes, stream);
  });
}

// (cache, q, out, seq_lens, block_table, max_seq_len, scale, workspace, stream)
PyObject *attn_decode(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[4], *ws, *stream;
  int32_t table[2], q[2], max_len;
  float scale;
  size_t ws_bytes;
  if (!count("attn_decode", n, 9) || !dims(a[4], table, 2, true) || !dims(a[1], q, 2, false) || !bytes_of(a[7], &ws_bytes) || !desc.take(a[0]))
    return nullptr;
  for (int i = 0; i < 4; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!scale_of(a[6], &scale) || !pointer(a[7], &ws) || !stream_of(a[8], &stream) || !int32(a[5], &max_len)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_attn_decode))entries[kDecode].fn)(desc.get(), p[0], p[1], (const int32_t *)p[2], (const int32_t *)p[3], table[0], table[1],
                                                            max_len, q[1], scale, ws, ws_bytes, stream);
  });
}

// (cache, q, out, seq_lens, block_table, max_seq_len, scale, stream)
PyObject *attn_decode_static(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[4], *stream;
  int32_t table[2], q[2], max_len;
  float scale;
  if (!count("attn_decode_static", n, 8) || !dims(a[4], table, 2, true) || !dims(a[1], q, 2, false) || !desc.take(a[0])) return nullptr;
  for (int i = 0; i < 4; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!scale_of(a[6], &scale) || !stream_of(a[7], &stream) || !int32(a[5], &max_len)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_attn_decode_static))entries[kDecodeStatic].fn)(desc.get(), p[0], p[1], (const int32_t *)p[2], (const int32_t *)p[3],
                                                                         table[0], table[1], max_len, q[1], scale, stream);
  });
}

// (cache, k_new, v_new, q, out, seq_lens, block_table, max_seq_len, scale, workspace, stream)
PyObject *decode_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[6], *ws, *stream;
  int32_t table[2], q[2], max_len;
  float scale;
  size_t ws_bytes;
  if (!count("decode_step", n, 11) || !dims(a[6], table, 2, true) || !dims(a[3], q, 2, false) || !bytes_of(a[9], &ws_bytes) || !desc.take(a[0]))
    return nullptr;
  for (int i = 0; i < 6; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!scale_of(a[8], &scale) || !pointer(a[9], &ws) || !stream_of(a[10], &stream) || !int32(a[7], &max_len)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_decode_step))entries[kDecodeStep].fn)(desc.get(), p[0], p[1], p[2], p[3], (const int32_t *)p[4], (const int32_t *)p[5],
                                                                table[0], table[1], max_len, q[1], scale, ws, ws_bytes, stream);
  });
}

// (cache, q, out, cu_seqlens_q, kv_lens, block_table, max_q_len, max_kv_len, scale, workspace, stream)
PyObject *attn_cross(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[5], *ws, *stream;
  int32_t table[2], q[2], max_q, max_kv;
  float scale;
  size_t ws_bytes;
  if (!count("attn_cross", n, 11, kCross) || !dims(a[5], table, 2, true) || !dims(a[1], q, 2, false) || !bytes_of(a[9], &ws_bytes) || !desc.take(a[0]))
    return nullptr;
  static const char *const names[] = {"cu_seqlens_q", "kv_lens", "block_table"};
  for (int i = 0; i < 5; ++i)
    if ((i >= 2 && a[1 + i] != Py_None && !sized(a[1 + i], names[i - 2], 4)) || !pointer(a[1 + i], p + i)) return nullptr;
  if (!scale_of(a[8], &scale) || !pointer(a[9], &ws) || !stream_of(a[10], &stream) || !int32(a[6], &max_q) || !int32(a[7], &max_kv)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_attn_cross))entries[kCross].fn)(desc.get(), p[0], p[1], (const int32_t *)p[2], (const int32_t *)p[3],
                                                          (const int32_t *)p[4], table[0], table[1], q[0], max_q, max_kv, q[1], scale, ws, ws_bytes,
                                                          stream);
  });
}

// The heads and the distance between the tokens of a tensor [tokens][heads][head_dim] whose rows of a token are contiguous.  tokens: those
// of the tensors before it, or -1.
bool rows_of(PyObject *t, const char *name, int32_t head_dim, int32_t *tokens, int32_t *heads, int64_t *stride) {
  int32_t size[3];
  int64_t step[3];
  if (!dims(t, size, 3, true) || !steps_of(t, step, 3)) return false;
  const int64_t row = (int64_t)size[1] * size[2];
  if (size[2] != head_dim || (*tokens >= 0 && size[0] != *tokens) || (size[0] > 0 && (step[2] != 1 || (size[1] > 1 && step[1] != size[2])))) {
    PyErr_Format(PyExc_ValueError, "%s: [tokens][heads][%d] with contiguous heads, as many tokens as the others", name, (int)head_dim);
    return false;
  }
  *tokens = size[0];
  *heads = size[1];
  *stride = size[0] <= 1 ? row : step[0];
  return true;
}

// (cache, q, k, v, q_out, cu_seqlens_new, ctx_lens, block_table, q_weight, k_weight, eps, cos_sin, interleaved, positions, stream)
PyObject *norm_rope_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[9], *cos_sin, *positions, *stream;
  int32_t table[2] = {0, 0}, tokens = -1, hq = 0, hk = 0, hv = 0, angles[2] = {0, 0};
  int64_t strides[3] = {0, 0, 0};
  float eps;
  if (!count("norm_rope_append", n, 15, kNormRope) || !desc.take(a[0])) return nullptr;
  int32_t d = desc.get()->head_dim;
  const int32_t hkv = desc.get()->num_kv_heads;
  if (a[7] == Py_None ? !dims(a[6], table, 1, false) : !dims(a[7], table, 2, true)) return nullptr;
  if (a[1] != Py_None) {
    int32_t ho;
    int64_t so;
    if (!rows_of(a[1], "q", d, &tokens, &hq, strides) || !rows_of(a[4], "q_out", d, &tokens, &ho, &so)) return nullptr;
    if (ho != hq || so != (int64_t)hq * d) {
      PyErr_SetString(PyExc_ValueError, "q_out: contiguous, with the heads of q");
      return nullptr;
    }
  }
  if (a[2] != Py_None && !rows_of(a[2], "k", d, &tokens, &hk, strides + 1)) return nullptr;
  if (a[3] != Py_None && !rows_of(a[3], "v", d, &tokens, &hv, strides + 2)) return nullptr;
  if ((a[2] != Py_None && hk != hkv) || (a[3] != Py_None && hv != hkv)) {
    PyErr_Format(PyExc_ValueError, "k and v: the cache has %d heads", (int)hkv);
    return nullptr;
  }
  if (tokens < 0) {
    PyErr_SetString(PyExc_ValueError, "norm_rope_append: k and v, queries, or both");
    return nullptr;
  }
  static const char *const names[] = {"cu_seqlens_new", "ctx_lens", "block_table", "q_weight", "k_weight"};
  for (int i = 0; i < 5; ++i)
    if (a[5 + i] != Py_None && !(i < 3 ? sized(a[5 + i], names[i], 4) : list_of(a[5 + i], names[i], 2, &d))) return nullptr;
  if (a[11] != Py_None) {
    int64_t step[2];
    if (!dims(a[11], angles, 2, true) || !sized(a[11], "cos_sin", 4) || !steps_of(a[11], step, 2)) return nullptr;
    if (!contiguous(angles, step)) {
      PyErr_SetString(PyExc_ValueError, "cos_sin: not contiguous");
      return nullptr;
    }
  }
  if (a[13] != Py_None) {
    int32_t have = -1;
    if (!list_of(a[13], "positions", 4, &have)) return nullptr;
    if (have < tokens) return PyErr_Format(PyExc_ValueError, "positions: %d entries for %d tokens", (int)have, (int)tokens);
  }
  for (int i = 0; i < 9; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!scale_of(a[10], &eps) || !pointer(a[11], &cos_sin) || !pointer(a[13], &positions) || !stream_of(a[14], &stream)) return nullptr;
  const int interleaved = PyObject_IsTrue(a[12]);
  if (interleaved < 0) return nullptr;
  const sp_rope_desc rope = {(const float *)cos_sin, angles[0], angles[1], interleaved};
  return finish([&] {
    return ((decltype(&sp_norm_rope_append))entries[kNormRope].fn)(
        desc.get(), p[0], p[1], p[2], strides[0], strides[1], strides[2], p[3], p[7], p[8], eps, a[11] == Py_None ? nullptr : &rope,
        (const int32_t *)positions, (const int32_t *)p[4], (const int32_t *)p[5], (const int32_t *)p[6], table[0], table[1], tokens, hq,
        stream);
  });
}

// (table, rows, new_lens, shortfall, workspace, stream)
PyObject *pages_reserve(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[4], *stream;
  int32_t entries_n = -1;
  size_t ws_bytes;
  if (!count("pages_reserve", n, 6, kReserve) || !list_of(a[1], "rows", 4, &entries_n) || !list_of(a[2], "new_lens", 4, &entries_n) ||
      !counters(a[3], "shortfall", 1) || !bytes_of(a[4], &ws_bytes) || !desc.take_table(a[0]))
    return nullptr;
  for (int i = 0; i < 4; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!stream_of(a[5], &stream)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_pages_reserve))entries[kReserve].fn)(desc.table(), (const int32_t *)p[0], (const int32_t *)p[1], entries_n, (int32_t *)p[2],
                                                               p[3], ws_bytes, stream);
  });
}

// (table, parents, children, copy_src, copy_dst, copy_rows, shortfall, workspace, stream)
PyObject *pages_fork(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[7], *stream;
  int32_t entries_n = -1;
  size_t ws_bytes;
  if (!count("pages_fork", n, 9, kFork)) return nullptr;
  static const char *const names[] = {"parents", "children", "copy_src", "copy_dst", "copy_rows"};
  for (int i = 0; i < 5; ++i)
    if (!list_of(a[1 + i], names[i], 4, &entries_n)) return nullptr;
  if (!counters(a[6], "shortfall", 1) || !bytes_of(a[7], &ws_bytes) || !desc.take_table(a[0])) return nullptr;
  for (int i = 0; i < 7; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!stream_of(a[8], &stream)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_pages_fork))entries[kFork].fn)(desc.table(), (const int32_t *)p[0], (const int32_t *)p[1], entries_n, (int32_t *)p[2],
                                                         (int32_t *)p[3], (int32_t *)p[4], (int32_t *)p[5], p[6], ws_bytes, stream);
  });
}

// (table, rows, keep_lens, stream)
PyObject *pages_release(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[2], *stream;
  int32_t entries_n = -1;
  if (!count("pages_release", n, 4, kRelease) || !list_of(a[1], "rows", 4, &entries_n) || !desc.take_table(a[0])) return nullptr;
  if (a[2] != Py_None && !list_of(a[2], "keep_lens", 4, &entries_n)) return nullptr;
  if (!pointer(a[1], p) || !pointer(a[2], p + 1) || !stream_of(a[3], &stream)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_pages_release))entries[kRelease].fn)(desc.table(), (const int32_t *)p[0], (const int32_t *)p[1], entries_n, stream);
  });
}

// (table, new_block_table, new_ref_counts, move_src, move_dst, moved, workspace, stream)
PyObject *pages_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
  Desc desc;
  void *p[6], *stream;
  int32_t table[2], sizes[4] = {-1, -1, -1, -1};
  int64_t step[2];
  size_t ws_bytes;
  if (!count("pages_compact", n, 8, kCompact) || !dims(a[1], table, 2, true) || !bytes_of(a[6], &ws_bytes) || !desc.take_table(a[0])) return nullptr;
  if (!sized(a[1], "new_block_table", 4) || !steps_of(a[1], step, 2)) return nullptr;
  if (!contiguous(table, step)) {
    PyErr_SetString(PyExc_ValueError, "new_block_table: not contiguous");
    return nullptr;
  }
  static const char *const names[] = {"new_ref_counts", "move_src", "move_dst", "moved"};
  for (int i = 0; i < 4; ++i)
    if (!list_of(a[2 + i], names[i], 4, sizes + i)) return nullptr;
  const sp_page_table *t = desc.table();
  if (table[0] != t->num_rows || table[1] != t->max_pages_per_seq || sizes[0] != t->num_pages || sizes[1] < t->num_pages / 2 ||
      sizes[2] < t->num_pages / 2 || sizes[3] < 2) {
    PyErr_SetString(PyExc_ValueError, "pages_compact: new arrays of the table's sizes, num_pages / 2 moves and 2 counts");
    return nullptr;
  }
  for (int i = 0; i < 6; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!stream_of(a[7], &stream)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_pages_compact))entries[kCompact].fn)(t, (int32_t *)p[0], (int32_t *)p[1], (int32_t *)p[2], (int32_t *)p[3], (int32_t *)p[4],
                                                               p[5], ws_bytes, stream);
  });
}

// (caches, src, dst, rows, count, stream): caches is a sequence
PyObject *pages_copy(PyObject *, PyObject *const *a, Py_ssize_t n) {
  void *p[4], *stream;
  int32_t pairs = -1;
  if (!count("pages_copy", n, 6, kCopy) || !list_of(a[1], "src", 4, &pairs) || !list_of(a[2], "dst", 4, &pairs) ||
      (a[3] != Py_None && !list_of(a[3], "rows", 4, &pairs)) || !counters(a[4], "count", 1))
    return nullptr;
  PyObject *fast = PySequence_Fast(a[0], "caches is not a sequence");
  if (!fast) return nullptr;
  const Py_ssize_t m = PySequence_Fast_GET_SIZE(fast);
  std::vector<sp_cache_desc> caches;
  bool ok = m <= INT32_MAX;
  try {
    caches.reserve(m);
  } catch (...) {
    ok = false;
  }
  if (!ok) PyErr_NoMemory();
  for (Py_ssize_t i = 0; ok && i < m && i < PySequence_Fast_GET_SIZE(fast); ++i) {
    Desc desc;
    ok = desc.take(PySequence_Fast_GET_ITEM(fast, i));
    if (ok) caches.push_back(*desc.get());
  }
  Py_DECREF(fast);
  if (!ok) return nullptr;
  for (int i = 0; i < 4; ++i)
    if (!pointer(a[1 + i], p + i)) return nullptr;
  if (!stream_of(a[5], &stream)) return nullptr;
  return finish([&] {
    return ((decltype(&sp_pages_copy))entries[kCopy].fn)(caches.data(), (int32_t)caches.size(), (const int32_t *)p[0], (const int32_t *)p[1],
                                                         (const int32_t *)p[2], (const int32_t *)p[3], pairs, stream);
  });
}

// bind(addresses, ArgumentError, c_int32, sp_cache_desc, get_device, get_stream, first_stream[, sp_page_table]): addresses maps the C-ABI
// names to the loaded library's functions
PyObject *bind(PyObject *, PyObject *args) {
  PyObject *table, *values[7] = {};
  if (!PyArg_ParseTuple(args, "O!OOOOOO|O", &PyDict_Type, &table, values, values + 1, values + 2, values + 3, values + 4, values + 5, values + 6))
    return nullptr;
  void *fn[kEntries];
  for (int i = 0; i < kEntries; ++i) {
    PyObject *v = PyDict_GetItemString(table, entries[i].name);
    fn[i] = nullptr;
    if (!v && i >= kRequired) continue;
    if (!v) return PyErr_Format(PyExc_KeyError, "%s", entries[i].name);
    fn[i] = PyLong_AsVoidPtr(v);
    if (!fn[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "%s is NULL", entries[i].name);
  }
  PyObject **slots[7] = {&argument_error, &c_int32, &desc_type, &get_device, &get_stream, &first_stream, &table_type};
  for (int i = 0; i < 7; ++i) {
    if (!values[i]) continue;
    Py_INCREF(values[i]);
    Py_XSETREF(*slots[i], values[i]);
  }
  for (int i = 0; i < kEntries; ++i) entries[i].fn = fn[i];
  Py_RETURN_NONE;
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr}, FAST(kv_append), FAST(attn_prefill), FAST(chunk_step), FAST(attn_decode),
                         FAST(attn_decode_static), FAST(decode_step), FAST(attn_cross), FAST(norm_rope_append), FAST(pages_reserve),
                         FAST(pages_fork), FAST(pages_release), FAST(pages_compact), FAST(pages_copy), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
  struct {
    PyObject **slot;
    const char *text;
  } names[] = {{&s_stride, "stride"},           {&s_data_ptr, "data_ptr"},       {&s_shape, "shape"}, {&s_numel, "numel"}, {&s_element_size, "element_size"},
               {&s_cuda_stream, "cuda_stream"}, {&s_desc, "desc"},   {&s_value, "value"},   {&s_as_parameter, "_as_parameter_"}};
  // In a forked child torch's device state is unusable: the public accessor says so, the raw ones go on.
  static bool registered = false;
  if (!registered && pthread_atfork(nullptr, nullptr, [] { stream_used = false; }) != 0) return PyErr_NoMemory();
  registered = true;
  for (auto &x : names)
    if (!(*x.slot = PyUnicode_InternFromString(x.text))) return nullptr;
  return PyModule_Create(&module);
}
