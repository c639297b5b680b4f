// Python extension `_marshal`: the binding's calls that a generation loop makes for every layer, with their arguments taken from
// torch tensors and lists of whole numbers in native code.  In Python an attention call's arguments took 5.4 us, as long as the whole
// launch of 64 queries, and those of an append 2.4 us.
//
// A function returns the library's status (a pack also its two lists), or None for anything but the ordinary kinds of arguments -
// exact torch.Tensor objects on a GPU, lists or tuples of int that fit the C type, a float, a stream given as int
// or not at all - or for sizes that do not go together: then nothing has been called, and binding.py takes the arguments
// its own way, with its own errors.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "df.h"

namespace {

decltype(&df_attn_fwd) attn_fwd, attn_fwd_static;
decltype(&df_head_score) head_score;
decltype(&df_kv_append) kv_append;
decltype(&df_pack_context) pack_context;
decltype(&df_page_map) page_map_entry;
decltype(&df_paged_append) paged_append_entry;
decltype(&df_paged_attn) paged_attn_entry;

// The readers below say whether an argument is of the ordinary kind.  (Nothing is thrown where it is not: that took 3 to 5 us, a third to a half of
// what a call costs that is marshalled in Python, such as one with a torch.cuda.Stream.)
const at::Tensor *tensor(PyObject *x) {
  if (!THPVariable_CheckExact(x)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(x);
  return t.is_cuda() ? &t : nullptr;
}
const at::Tensor *tensor(PyObject *x, int64_t dims) {
  const at::Tensor *t = tensor(x);
  return t && t->dim() == dims ? t : nullptr;
}
void *address(const at::Tensor &t) { return t.numel() == 0 ? nullptr : t.data_ptr(); }
template <class T>
bool address_or_null(PyObject *x, T *&to) {
  to = nullptr;
  if (x == Py_None) return true;
  const at::Tensor *t = tensor(x);
  if (t) to = static_cast<T *>(address(*t));
  return t != nullptr;
}
bool buffer_or_null(PyObject *x, void *&to, size_t &bytes) {
  to = nullptr;
  bytes = 0;
  if (x == Py_None) return true;
  const at::Tensor *t = tensor(x);
  if (t == nullptr) return false;
  to = address(*t);
  bytes = size_t(t->numel()) * t->element_size();
  return true;
}
bool size32(int64_t n, int32_t &to) {
  to = int32_t(n);
  return n <= INT32_MAX;
}

// A list or tuple of whole numbers as a C array of at least `at_least` of them.
template <class T>
struct Numbers {
  T at[2 * DF_MAX_HEADS];
  bool read(PyObject *x, Py_ssize_t at_least) {
    if (!PyList_CheckExact(x) && !PyTuple_CheckExact(x)) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(x);
    if (n < at_least || n > 2 * DF_MAX_HEADS) return false;
    PyObject **items = PySequence_Fast_ITEMS(x);
    for (Py_ssize_t i = 0; i < n; ++i) {
      if (!PyLong_CheckExact(items[i])) return false;
      int overflow = 0;
      const long long v = PyLong_AsLongLongAndOverflow(items[i], &overflow);
      at[i] = T(v);
      if (overflow || at[i] != v) return false;
    }
    return true;
  }
  // None: no list.
  template <class P>
  bool read_or_null(PyObject *x, Py_ssize_t at_least, P *&to) {
    to = nullptr;
    if (x == Py_None) return true;
    to = at;
    return read(x, at_least);
  }
};
bool number(PyObject *x, int32_t &to) {
  if (!PyLong_CheckExact(x)) return false;
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(x, &overflow);
  to = int32_t(v);
  return !overflow && to == v;
}
bool real(PyObject *x, float &to) {
  if (!PyFloat_CheckExact(x)) return false;
  to = float(PyFloat_AS_DOUBLE(x));
  return true;
}
// None: the current stream of the current device.
bool stream(PyObject *x, void *&to) {
  if (x == Py_None) {
    to = c10::hip::getCurrentHIPStream().stream();
    return true;
  }
  if (!PyLong_CheckExact(x)) return false;
  to = PyLong_AsVoidPtr(x);
  if (to != nullptr || !PyErr_Occurred()) return true;
  PyErr_Clear();
  return false;
}

template <class Call>
df_status without_gil(Call &&call) {
  df_status s;
  Py_BEGIN_ALLOW_THREADS
  s = call();
  Py_END_ALLOW_THREADS
  return s;
}
// The C struct of a binding.Cache, or null.
struct CacheOf {
  Py_buffer view{};
  df_cache *cache = nullptr;
  explicit CacheOf(PyObject *x) {
    PyObject *c = PyObject_GetAttrString(x, "c");
    if (c == nullptr || PyObject_GetBuffer(c, &view, PyBUF_WRITABLE) != 0) PyErr_Clear();
    else if (size_t(view.len) == sizeof(df_cache)) cache = static_cast<df_cache *>(view.buf);
    Py_XDECREF(c);                   // the view holds it
    if (cache && (cache->H < 0 || cache->H > DF_MAX_HEADS)) cache = nullptr;
  }
  CacheOf(const CacheOf &) = delete;
  ~CacheOf() { PyBuffer_Release(&view); }          // nothing where there is no view
};

// Runs `body`; null without a Python error, and what torch throws for a tensor that has no address, is None.
template <class Body>
PyObject *or_none(Py_ssize_t n, Py_ssize_t wanted, Body &&body) {
  if (n == wanted) {
    try {
      PyObject *result = body();
      if (result != nullptr || PyErr_Occurred()) return result;
    } catch (const std::exception &) {
    }
  }
  Py_RETURN_NONE;
}

// q, k_cur, v_cur, k_hist, v_hist, hist_off, hist_sink_len, out, softmax_scale, lse_out, score_out, workspace, stream, hist_len, static
PyObject *attn(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return or_none(n, 15, [&]() -> PyObject * {
    const at::Tensor *q = tensor(x[0], 3), *k = tensor(x[1], 3), *v = tensor(x[2]), *out = tensor(x[7], 3);
    df_attn_args a{};
    void *st;
    Numbers<int64_t> off;
    Numbers<int32_t> sink, len;
    if (!q || !k || !v || !out || !stream(x[12], st) || !real(x[8], a.softmax_scale) || v->strides() != k->strides() ||
        !size32(q->size(1), a.H) || !size32(q->size(2), a.d) || !size32(q->size(0), a.Nq) || !size32(k->size(0), a.Nc) ||
        !off.read(x[5], Py_ssize_t(a.H) + 1) || !sink.read_or_null(x[6], a.H, a.hist_sink_len) ||
        !len.read_or_null(x[13], a.H, a.hist_len) || !address_or_null(x[3], a.k_hist) || !address_or_null(x[4], a.v_hist) ||
        !address_or_null(x[9], a.lse_out) || !address_or_null(x[10], a.score_out) ||
        !buffer_or_null(x[11], a.workspace, a.workspace_bytes))
      return nullptr;
    a.q = address(*q);
    a.q_stride_tok = q->stride(0);
    a.q_stride_head = q->stride(1);
    a.k_cur = address(*k);
    a.v_cur = address(*v);
    a.kc_stride_tok = k->stride(0);
    a.kc_stride_head = k->stride(1);
    a.hist_off = off.at;
    a.out = address(*out);
    a.o_stride_tok = out->stride(0);
    a.o_stride_head = out->stride(1);
    const auto entry = x[14] == Py_True ? attn_fwd_static : attn_fwd;
    return PyLong_FromLong(without_gil([&] { return entry(&a, st); }));
  });
}

// q, k_cur, k_hist, hist_off, hist_sink_len, score_out, softmax_scale, q_sample_stride, q_offset, workspace, stream, hist_len
PyObject *score(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return or_none(n, 12, [&]() -> PyObject * {
    const at::Tensor *q = tensor(x[0], 3), *k = tensor(x[1], 3);
    df_score_args a{};
    void *st;
    Numbers<int64_t> off;
    Numbers<int32_t> sink, len;
    if (!q || !k || !stream(x[10], st) || !real(x[6], a.softmax_scale) || !number(x[7], a.q_sample_stride) || !number(x[8], a.q_offset) ||
        !size32(q->size(1), a.H) || !size32(q->size(2), a.d) || !size32(q->size(0), a.Nq) || !size32(k->size(0), a.Nc) ||
        !off.read(x[3], Py_ssize_t(a.H) + 1) || !sink.read(x[4], a.H) || !len.read_or_null(x[11], a.H, a.hist_len) ||
        !address_or_null(x[2], a.k_hist) || !address_or_null(x[5], a.score_out) ||
        !buffer_or_null(x[9], a.workspace, a.workspace_bytes))
      return nullptr;
    a.q = address(*q);
    a.q_stride_tok = q->stride(0);
    a.q_stride_head = q->stride(1);
    a.k_cur = address(*k);
    a.kc_stride_tok = k->stride(0);
    a.kc_stride_head = k->stride(1);
    a.hist_off = off.at;
    a.hist_sink_len = sink.at;
    return PyLong_FromLong(without_gil([&] { return head_score(&a, st); }));
  });
}

// cache, k_new, v_new, stream
PyObject *append(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return or_none(n, 4, [&]() -> PyObject * {
    const at::Tensor *k = tensor(x[1], 3), *v = tensor(x[2]);
    df_append_args a{};
    void *st;
    if (!k || !v || !stream(x[3], st) || v->strides() != k->strides() || !size32(k->size(0), a.Nc)) return nullptr;
    const CacheOf cache(x[0]);
    if (!cache.cache) return nullptr;
    a.cache = cache.cache;
    a.k_new = address(*k);
    a.v_new = address(*v);
    a.stride_tok = k->stride(0);
    a.stride_head = k->stride(1);
    return PyLong_FromLong(without_gil([&] { return kv_append(&a, st); }));
  });
}

// A binding.PagedCache: its C struct, and its pages for their type and place; no cache where it is no such object or not on the current GPU.
struct PagedOf {
  Py_buffer view{};
  df_paged_cache *cache = nullptr;
  at::ScalarType type{};
  c10::Device device{c10::kCPU};
  explicit PagedOf(PyObject *x) {
    PyObject *c = PyObject_GetAttrString(x, "c"), *k = c ? PyObject_GetAttrString(x, "k_pages") : nullptr;
    const at::Tensor *pages = k ? tensor(k) : nullptr;
    if (c == nullptr || k == nullptr || PyObject_GetBuffer(c, &view, PyBUF_WRITABLE) != 0) PyErr_Clear();
    else if (pages && size_t(view.len) == sizeof(df_paged_cache)) {
      type = pages->scalar_type();
      device = pages->device();
      if (device.index() == c10::hip::current_device()) cache = static_cast<df_paged_cache *>(view.buf);
    }
    Py_XDECREF(k);                   // the object holds it
    Py_XDECREF(c);                   // the view holds it
  }
  PagedOf(const PagedOf &) = delete;
  ~PagedOf() { PyBuffer_Release(&view); }

  // An array of the cache's device: its address, null for an empty one.
  template <class T>
  bool array(PyObject *x, at::ScalarType t, std::initializer_list<int64_t> shape, T *&to) const {
    const at::Tensor *a = tensor(x);
    if (!a || a->scalar_type() != t || a->device() != device || !a->sizes().equals(shape) || !a->is_contiguous()) return false;
    to = static_cast<T *>(address(*a));
    return true;
  }
  // Rows [tokens, heads, d] of the cache's type; strides of dimensions of one do not matter.
  bool rows(const at::Tensor *t, int64_t heads, int64_t &tok, int64_t &head) const {
    if (!t || t->dim() != 3 || t->size(1) != heads || t->size(2) != cache->d || t->scalar_type() != type || t->device() != device || t->stride(2) != 1)
      return false;
    tok = t->size(0) > 1 ? t->stride(0) : heads * cache->d;
    head = heads > 1 ? t->stride(1) : cache->d;
    return true;
  }
};

// cache, cu_new, slot_map, status, release, len_out, n_free_out, stream
PyObject *page_map(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return or_none(n, 8, [&]() -> PyObject * {
    const at::Tensor *slots = tensor(x[2], 2);
    df_page_map_args a{};
    void *st;
    if (!slots || !stream(x[7], st) || !size32(slots->size(0), a.total_new)) return nullptr;
    const PagedOf p(x[0]);
    if (!p.cache) return nullptr;
    const int64_t B = p.cache->B;
    if (!p.array(x[1], at::kInt, {B + 1}, a.cu_new) || !p.array(x[2], at::kLong, {a.total_new, p.cache->H_kv}, a.slot_map) ||
        !p.array(x[3], at::kInt, {1}, a.status) || (x[4] != Py_None && !p.array(x[4], at::kByte, {B}, a.release)) ||
        !p.array(x[5], at::kInt, {B}, a.len_out) || !p.array(x[6], at::kInt, {1}, a.n_free_out))
      return nullptr;
    a.cache = p.cache;
    return PyLong_FromLong(without_gil([&] { return page_map_entry(&a, st); }));
  });
}

// cache, k_new, v_new, slot_map, stream
PyObject *paged_append(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return or_none(n, 5, [&]() -> PyObject * {
    const at::Tensor *k = tensor(x[1], 3), *v = tensor(x[2], 3);
    df_paged_append_args a{};
    void *st;
    int64_t tok, head;
    if (!k || !v || !stream(x[4], st) || !size32(k->size(0), a.total_new)) return nullptr;
    const PagedOf p(x[0]);
    if (!p.cache || !p.rows(k, p.cache->H_kv, a.stride_tok, a.stride_head) || !p.rows(v, p.cache->H_kv, tok, head) || tok != a.stride_tok ||
        head != a.stride_head || v->size(0) != k->size(0) || !p.array(x[3], at::kLong, {a.total_new, p.cache->H_kv}, a.slot_map))
      return nullptr;
    a.cache = p.cache;
    a.k_new = address(*k);
    a.v_new = address(*v);
    return PyLong_FromLong(without_gil([&] { return paged_append_entry(&a, st); }));
  });
}

// q, k_cur, v_cur, cache, cu_new, out, softmax_scale, block, max_new, lse_out, workspace, stream
PyObject *paged_attn(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return or_none(n, 12, [&]() -> PyObject * {
    const at::Tensor *q = tensor(x[0], 3), *out = tensor(x[5], 3);
    df_paged_attn_args a{};
    void *st;
    if (!q || !out || !stream(x[11], st) || !size32(q->size(0), a.total_new) || !size32(q->size(1), a.H_q) || !real(x[6], a.softmax_scale) ||
        !number(x[7], a.block) || !(x[8] == Py_None || number(x[8], a.max_new)) || !buffer_or_null(x[10], a.workspace, a.workspace_bytes))
      return nullptr;
    if (x[8] == Py_None) a.max_new = a.total_new;
    const PagedOf p(x[3]);
    const at::Tensor *ws = tensor(x[10]);
    if (!p.cache || (ws && !(ws->is_contiguous() && ws->device() == p.device)) || !p.rows(q, a.H_q, a.q_stride_tok, a.q_stride_head) || !p.rows(out, a.H_q, a.o_stride_tok, a.o_stride_head) ||
        out->size(0) != a.total_new || !p.array(x[4], at::kInt, {int64_t(p.cache->B) + 1}, a.cu_new) ||
        (x[9] != Py_None && !p.array(x[9], at::kFloat, {a.H_q, a.total_new}, a.lse_out)))
      return nullptr;
    if (x[1] != Py_None || x[2] != Py_None) {
      const at::Tensor *k = tensor(x[1], 3), *v = tensor(x[2], 3);
      int64_t tok, head;
      if (!p.rows(k, p.cache->H_kv, a.kc_stride_tok, a.kc_stride_head) || !p.rows(v, p.cache->H_kv, tok, head) || tok != a.kc_stride_tok ||
          head != a.kc_stride_head || k->size(0) != a.total_new || v->size(0) != a.total_new)
        return nullptr;
      a.k_cur = address(*k);
      a.v_cur = address(*v);
    }
    a.cache = p.cache;
    a.q = address(*q);
    a.out = address(*out);
    return PyLong_FromLong(without_gil([&] { return paged_attn_entry(&a, st); }));
  });
}

template <class T>
PyObject *list_of(const T *x, int n) {
  PyObject *list = PyList_New(n);
  for (int i = 0; list && i < n; ++i) {
    PyObject *v = PyLong_FromLongLong(x[i]);
    if (v == nullptr) {
      Py_DECREF(list);
      return nullptr;
    }
    PyList_SET_ITEM(list, i, v);
  }
  return list;
}
// cache, take_sink, take_win, k_out, v_out, stream -> status, hist_off, sink_len
PyObject *pack(PyObject *, PyObject *const *x, Py_ssize_t n) {
  return or_none(n, 6, [&]() -> PyObject * {
    const at::Tensor *k = tensor(x[3]), *v = tensor(x[4]);
    void *st;
    if (!k || !v || k->dim() < 1 || !stream(x[5], st)) return nullptr;
    const CacheOf cache(x[0]);
    if (!cache.cache) return nullptr;
    const int H = cache.cache->H;
    Numbers<int32_t> sink, win;
    if (!sink.read(x[1], H) || !win.read(x[2], H)) return nullptr;
    int64_t off[DF_MAX_HEADS + 1] = {};
    int32_t sink_len[DF_MAX_HEADS] = {};
    df_pack_args a{};
    a.cache = cache.cache;
    a.take_sink = sink.at;
    a.take_win = win.at;
    a.k_out = address(*k);
    a.v_out = address(*v);
    a.out_capacity_rows = k->size(0);
    a.hist_off_out = off;
    a.sink_len_out = sink_len;
    const df_status s = without_gil([&] { return pack_context(&a, st); });
    PyObject *o = list_of(off, H + 1), *l = o ? list_of(sink_len, H) : nullptr;
    if (l == nullptr) {
      Py_XDECREF(o);
      return nullptr;
    }
    return Py_BuildValue("iNN", int(s), o, l);
  });
}

// The addresses of N functions.
template <int N>
bool addresses(PyObject *const *x, Py_ssize_t n, void *(&f)[N]) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d addresses", N);
    return false;
  }
  for (int i = 0; i < N; ++i) {
    f[i] = PyLong_AsVoidPtr(x[i]);
    if (f[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a function has no address");
      return false;
    }
  }
  return true;
}
// Addresses of df_attn_fwd, df_attn_fwd_static, df_head_score, df_kv_append and df_pack_context in the library that the binding loaded.
PyObject *setup(PyObject *, PyObject *const *x, Py_ssize_t n) {
  void *f[5];
  if (!addresses(x, n, f)) return nullptr;
  attn_fwd = reinterpret_cast<decltype(attn_fwd)>(f[0]);
  attn_fwd_static = reinterpret_cast<decltype(attn_fwd_static)>(f[1]);
  head_score = reinterpret_cast<decltype(head_score)>(f[2]);
  kv_append = reinterpret_cast<decltype(kv_append)>(f[3]);
  pack_context = reinterpret_cast<decltype(pack_context)>(f[4]);
  Py_RETURN_NONE;
}
// Those of df_page_map, df_paged_append and df_paged_attn.
PyObject *setup_paged(PyObject *, PyObject *const *x, Py_ssize_t n) {
  void *f[3];
  if (!addresses(x, n, f)) return nullptr;
  page_map_entry = reinterpret_cast<decltype(page_map_entry)>(f[0]);
  paged_append_entry = reinterpret_cast<decltype(paged_append_entry)>(f[1]);
  paged_attn_entry = reinterpret_cast<decltype(paged_attn_entry)>(f[2]);
  Py_RETURN_NONE;
}

template <class F>
PyCFunction as_c(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }
PyMethodDef methods[] = {{"setup", as_c(setup), METH_FASTCALL, nullptr},   {"attn", as_c(attn), METH_FASTCALL, nullptr},
                         {"score", as_c(score), METH_FASTCALL, nullptr},   {"append", as_c(append), METH_FASTCALL, nullptr},
                         {"pack", as_c(pack), METH_FASTCALL, nullptr},     {"setup_paged", as_c(setup_paged), METH_FASTCALL, nullptr},
                         {"page_map", as_c(page_map), METH_FASTCALL, nullptr}, {"paged_append", as_c(paged_append), METH_FASTCALL, nullptr},
                         {"paged_attn", as_c(paged_attn), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
