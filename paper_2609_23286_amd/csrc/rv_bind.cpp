// rv_bind.cpp -- the argument marshalling of rv.py's per-frame calls, as a CPython module.
//
// The calls around a frame's attention (projections, sequences) are made from here as a whole where their
// arguments are plain tensors and integers: through Python's attributes and ctypes the call that prepares
// one token took 17 us for a kernel of 4.
//
// A frame of 24 layers passes some 150 tensors to one admission call.  Checking shape, type,
// device and layout and taking the address costs about 0.7 us a tensor through Python's
// attributes (112 us for an admission call whose kernels take 40), and about 0.03 us here.
// Checks, their order and their exceptions are those of rv._ptr; tensor subclasses
// and anything that is not a tensor go to that function.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstdint>
#include <exception>
#include <initializer_list>
#include <vector>

#include "../../include/rv.h"

namespace {

PyObject* g_ptr_fallback = nullptr;  // rv._ptr_python(t, shape, itemsize, what)
// librv's functions, from the handle rv.py loaded it by.
decltype(&rv_mem_view) g_mem_view = nullptr;
decltype(&rv_mem_len) g_mem_len = nullptr;

// A shape as rv.py's calls state it: up to four extents.
struct Shape {
  int n = 0;
  int64_t d[4];
};

bool parse_shape(PyObject* o, Shape* s) {
  if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) > 4) {
    PyErr_SetString(PyExc_TypeError, "shape: a tuple of up to four integers");
    return false;
  }
  s->n = (int)PyTuple_GET_SIZE(o);
  for (int i = 0; i < s->n; ++i) {
    s->d[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
    if (s->d[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

// What the checks accept without a word; anything else is rv._ptr_python's to word or pass.
bool plain_ptr(PyObject* o, const Shape& s, int itemsize, void** out) {
  if (o == Py_None) {
    *out = nullptr;
    return true;
  }
  if (!THPVariable_CheckExact(o)) return false;
  try {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.unsafeGetTensorImpl()->is_python_dispatch() || !t.is_contiguous() ||
        (int64_t)t.element_size() != itemsize || t.dim() != s.n)
      return false;
    for (int i = 0; i < s.n; ++i)
      if (t.size(i) != s.d[i]) return false;
    *out = t.data_ptr();
    return true;
  } catch (const std::exception&) {
    return false;  // (the same access from Python raises it)
  }
}

// The device address of a tensor argument (NULL for None); false with an exception set.
bool take_ptr(PyObject* o, PyObject* shape_obj, const Shape& s, int itemsize, const char* what, Py_ssize_t index,
              void** out) {
  if (plain_ptr(o, s, itemsize, out)) return true;
  PyObject* name = index < 0 ? PyUnicode_FromString(what) : PyUnicode_FromFormat("%s[%zd]", what, index);
  if (!name) return false;
  PyObject* r = PyObject_CallFunction(g_ptr_fallback, "OOiN", o, shape_obj, itemsize, name);
  if (!r) return false;
  bool ok = true;
  if (r == Py_None) {
    *out = nullptr;
  } else {
    *out = PyLong_AsVoidPtr(r);
    ok = !(*out == nullptr && PyErr_Occurred());
  }
  Py_DECREF(r);
  return ok;
}

// ptr(tensor, shape, itemsize, what) -> address
PyObject* py_ptr(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4) return PyErr_Format(PyExc_TypeError, "ptr takes 4 arguments (%zd given)", n);
  Shape s;
  const long itemsize = PyLong_AsLong(args[2]);
  if (itemsize == -1 && PyErr_Occurred()) return nullptr;
  const char* what = PyUnicode_AsUTF8(args[3]);
  if (!what || !parse_shape(args[1], &s)) return nullptr;
  void* p;
  if (!take_ptr(args[0], args[1], s, (int)itemsize, what, -1, &p)) return nullptr;
  return PyLong_FromVoidPtr(p);
}

// ptrs(tensors, n_layers, shape, itemsize, what) -> bytes holding n_layers addresses
PyObject* py_ptrs(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 5) return PyErr_Format(PyExc_TypeError, "ptrs takes 5 arguments (%zd given)", n);
  const Py_ssize_t layers = PyLong_AsSsize_t(args[1]);
  if (layers == -1 && PyErr_Occurred()) return nullptr;
  const long itemsize = PyLong_AsLong(args[3]);
  if (itemsize == -1 && PyErr_Occurred()) return nullptr;
  const char* what = PyUnicode_AsUTF8(args[4]);
  Shape s;
  if (!what || !parse_shape(args[2], &s)) return nullptr;
  PyObject* seq = PySequence_Fast(args[0], "expected a sequence of tensors");
  if (!seq) return nullptr;
  PyObject* out = PyBytes_FromStringAndSize(nullptr, layers * (Py_ssize_t)sizeof(void*));
  if (out) {
    void** p = reinterpret_cast<void**>(PyBytes_AS_STRING(out));
    for (Py_ssize_t i = 0; i < layers; ++i) p[i] = nullptr;  // (a shorter list: the library refuses NULLs)
    // (the size is read each time round: a subclass's accessors may run code that changes it)
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(seq); ++i) {
      void* x = nullptr;
      PyObject* o = PySequence_Fast_GET_ITEM(seq, i);
      Py_INCREF(o);
      const bool ok = take_ptr(o, args[2], s, (int)itemsize, what, i, &x);
      Py_DECREF(o);
      if (ok && i >= layers) PyErr_SetString(PyExc_IndexError, "invalid index");
      if (!ok || i >= layers) {
        Py_CLEAR(out);
        break;
      }
      p[i] = x;
    }
  }
  Py_DECREF(seq);
  return out;
}

// mem_state(handle) -> (memK, memV, head stride, length), or the status of a failed view
PyObject* py_mem_state(PyObject*, PyObject* handle) {
  void* h = handle == Py_None ? nullptr : PyLong_AsVoidPtr(handle);
  if (!h && PyErr_Occurred()) return nullptr;
  const void *k = nullptr, *v = nullptr;
  int64_t hs = 0;
  const rv_status st = g_mem_view((rv_mem)h, &k, &v, &hs);
  if (st != RV_OK) return PyLong_FromLong((long)st);
  return Py_BuildValue("(KKLL)", (unsigned long long)(uintptr_t)k, (unsigned long long)(uintptr_t)v, (long long)hs,
                       (long long)g_mem_len((rv_mem)h));
}

// setup(rv._ptr_python, address of rv_mem_view, address of rv_mem_len)
PyObject* py_setup(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 3) return PyErr_Format(PyExc_TypeError, "setup takes 3 arguments (%zd given)", n);
  void *view = PyLong_AsVoidPtr(args[1]), *len = PyLong_AsVoidPtr(args[2]);
  if (!view || !len) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "NULL function");
  g_mem_view = reinterpret_cast<decltype(g_mem_view)>(view);
  g_mem_len = reinterpret_cast<decltype(g_mem_len)>(len);
  Py_INCREF(args[0]);
  Py_XDECREF(g_ptr_fallback);
  g_ptr_fallback = args[0];
  Py_RETURN_NONE;
}

// ---- whole calls --------------------------------------------------------------------------
//
// Each takes the arguments of the function of the same name in rv.py, its stream as an integer and the
// current device, and returns the call's status, or None if some argument is not a plain one: rv.py then
// goes its own way, which words the refusal.

decltype(&rv_prepare_qkv) g_prepare = nullptr;
decltype(&rv_prepare_qkv_bwd) g_prepare_bwd = nullptr;
decltype(&rv_pool_fork) g_fork = nullptr;
decltype(&rv_pool_close) g_close = nullptr;
decltype(&rv_pool_append) g_append = nullptr;
decltype(&rv_pool_gather) g_gather = nullptr;
decltype(&rv_pool_compact) g_compact = nullptr;
decltype(&rv_attend_seqs) g_attend = nullptr;

constexpr int64_t kHeadDim = 64;
constexpr c10::ScalarType kBF16 = c10::ScalarType::BFloat16;

// Arguments read one after another; `plain` turns false at the first that is not as expected.
class Args {
 public:
  Args(PyObject* const* a, Py_ssize_t n, Py_ssize_t want) : a_(a), plain(n == want) {}

  int64_t integer() {
    PyObject* o = a_[i_++];
    if (!plain || !PyLong_CheckExact(o)) return plain = false, 0;
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      plain = false;
    }
    return v;
  }
  int small() {  // an int
    const int64_t v = integer();
    if (v != (int)v) plain = false;
    return (int)v;
  }
  void* address() { return reinterpret_cast<void*>((uintptr_t)integer()); }

  // A list or tuple of integers that fit T; none: whether None may stand for it (false if it does).
  template <class T>
  bool integers(std::vector<T>* out, bool none = false) {
    PyObject* o = a_[i_++];
    if (!plain || (none && o == Py_None)) return false;
    const bool list = PyList_CheckExact(o);
    if (!list && !PyTuple_CheckExact(o)) return plain = false;
    const Py_ssize_t n = list ? PyList_GET_SIZE(o) : PyTuple_GET_SIZE(o);
    out->resize(n);
    for (Py_ssize_t k = 0; k < n && plain; ++k) {
      PyObject* x = list ? PyList_GET_ITEM(o, k) : PyTuple_GET_ITEM(o, k);
      long long v = 0;
      if (!PyLong_CheckExact(x) || ((v = PyLong_AsLongLong(x)) == -1 && PyErr_Occurred()) || v != (T)v) {
        PyErr_Clear();
        plain = false;
      }
      (*out)[k] = (T)v;
    }
    return plain;
  }

  // The next argument as a plain tensor on `device`, NULL for None.
  const at::Tensor* tensor(int64_t device) {
    PyObject* o = a_[i_++];
    if (!plain || o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) return plain = false, nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.unsafeGetTensorImpl()->is_python_dispatch() || t.layout() != at::kStrided ||
        t.get_device() != device)
      return plain = false, nullptr;
    return &t;
  }
  // Its address, if contiguous, of `type` (BFloat16: or its bits as whole numbers) and of this shape; d[0] < 0: any
  // shape of -d[0] - 1 elements.
  void* exact(int64_t device, c10::ScalarType type, std::initializer_list<int64_t> d) {
    const at::Tensor* t = tensor(device);
    if (!t) return nullptr;
    const c10::ScalarType ty = t->scalar_type();
    bool ok = t->is_contiguous() && (ty == type || (type == c10::ScalarType::BFloat16 &&
                                                    (ty == c10::ScalarType::Short || ty == c10::ScalarType::UInt16)));
    if (*d.begin() < 0) {
      ok = ok && t->numel() == -*d.begin() - 1;
    } else {
      ok = ok && t->dim() == (int64_t)d.size();
      int64_t k = 0;
      for (int64_t x : d) ok = ok && t->size(k++) == x;
    }
    if (!ok) plain = false;
    return ok ? t->data_ptr() : nullptr;
  }
  // Rows [n, heads * 64] or [n, heads, 64] at any distance; *n < 0: sets it; *type Undefined: sets it.
  void* rows(int64_t device, int64_t heads, int64_t* n, c10::ScalarType* type, int64_t* stride) {
    *stride = 0;
    const at::Tensor* t = tensor(device);
    if (!t) return nullptr;
    const int64_t dim = t->dim();
    bool ok = dim == 2 ? t->size(1) == heads * kHeadDim
                       : dim == 3 && t->size(1) == heads && t->size(2) == kHeadDim &&
                             (heads == 1 || t->stride(1) == kHeadDim);
    ok = ok && t->stride(dim - 1) == 1;
    const c10::ScalarType ty = t->scalar_type();
    ok = ok && (ty == c10::ScalarType::BFloat16 || ty == c10::ScalarType::Float) &&
         (*type == c10::ScalarType::Undefined || *type == ty) && (*n < 0 || t->size(0) == *n);
    if (!ok) return plain = false, nullptr;
    *type = ty;
    *n = t->size(0);
    *stride = *n > 1 ? t->stride(0) : heads * kHeadDim;
    return t->data_ptr();
  }

 private:
  PyObject* const* a_;
  Py_ssize_t i_ = 0;

 public:
  bool plain;
};

template <class F>
PyObject* made(bool plain, F call) {
  if (!plain) Py_RETURN_NONE;
  int st;
  Py_BEGIN_ALLOW_THREADS st = (int)call();
  Py_END_ALLOW_THREADS return PyLong_FromLong(st);
}

// (the checks of the tensors' accessors throw; what throws is not plain)
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

rv_dtype dtype_of(c10::ScalarType t) { return t == c10::ScalarType::Float ? RV_F32 : RV_BF16; }

// prepare(prep address, axes, q_heads, kv_heads, device, stream, q, k, v, pos, Q, K, V)
PyObject* py_prepare(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 13);
    if (!a.plain) Py_RETURN_NONE;
    const auto* prep = static_cast<const rv_qkv_prep*>(a.address());
    const int64_t axes = a.integer(), hq = a.integer(), hk = a.integer(), dev = a.integer();
    void* const s = a.address();
    int64_t N = -1, sq, sk, sv;
    c10::ScalarType ty = c10::ScalarType::Undefined;
    void *q = a.rows(dev, hq, &N, &ty, &sq), *k = a.rows(dev, hk, &N, &ty, &sk), *v = a.rows(dev, hk, &N, &ty, &sv);
    if (!q || N > INT32_MAX) a.plain = false;
    void* pos = a.exact(dev, c10::ScalarType::Int, {N, axes});
    void *Q = a.exact(dev, kBF16, {N, hq, kHeadDim}), *K = a.exact(dev, kBF16, {N, hk, kHeadDim}),
         *V = a.exact(dev, kBF16, {N, hk, kHeadDim});
    return made(a.plain && !(axes == 0 && pos), [&] {
      return g_prepare(prep, q, sq, k, sk, v, sv, dtype_of(ty), (int)N, (const int32_t*)pos, Q, K, V, s);
    });
  });
}

// prepare_bwd(prep address, axes, q_heads, kv_heads, device, stream, q, k, pos, dQ, dK, dV, dq, dk, dv, dq_weight,
//             dq_bias, dk_weight, dk_bias)
PyObject* py_prepare_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 19);
    if (!a.plain) Py_RETURN_NONE;
    const auto* prep = static_cast<const rv_qkv_prep*>(a.address());
    const int64_t axes = a.integer(), hq = a.integer(), hk = a.integer(), dev = a.integer();
    void* const s = a.address();
    int64_t N = -1, sq, sk, tq, tk, tv;
    c10::ScalarType ty = c10::ScalarType::Undefined;
    void *q = a.rows(dev, hq, &N, &ty, &sq), *k = a.rows(dev, hk, &N, &ty, &sk);
    if (!q || N > INT32_MAX) a.plain = false;
    void* pos = a.exact(dev, c10::ScalarType::Int, {N, axes});
    void *dQ = a.exact(dev, kBF16, {N, hq, kHeadDim}), *dK = a.exact(dev, kBF16, {N, hk, kHeadDim}),
         *dV = a.exact(dev, kBF16, {N, hk, kHeadDim});
    void *dq = a.rows(dev, hq, &N, &ty, &tq), *dk = a.rows(dev, hk, &N, &ty, &tk), *dv = a.rows(dev, hk, &N, &ty, &tv);
    float* sums[4];
    for (float*& x : sums) x = (float*)a.exact(dev, c10::ScalarType::Float, {kHeadDim});
    return made(a.plain && !(axes == 0 && pos), [&] {
      return g_prepare_bwd(prep, q, sq, k, sk, dtype_of(ty), (int)N, (const int32_t*)pos, dQ, dK, dV, dq, tq, dk, tk, dv,
                           tv, sums[0], sums[1], sums[2], sums[3], s);
    });
  });
}

// fork(pool, stream, seq, n_rows, n) -> status, or the list of children
PyObject* py_fork(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 5);
    if (!a.plain) Py_RETURN_NONE;
    void *pool = a.address(), *s = a.address();
    const int seq = a.small();
    const int64_t rows = a.integer();
    const int count = a.small();
    if (!a.plain || count < 0) Py_RETURN_NONE;
    std::vector<int> out((size_t)count);
    const rv_status st = g_fork((rv_pool)pool, seq, rows, count, out.data(), s);
    if (st != RV_OK) return PyLong_FromLong((long)st);
    PyObject* list = PyList_New(count);
    for (int i = 0; list && i < count; ++i) PyList_SET_ITEM(list, i, PyLong_FromLong(out[i]));
    return list;
  });
}

// release(pool, seqs)
PyObject* py_release(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 2);
    if (!a.plain) Py_RETURN_NONE;
    void* pool = a.address();
    std::vector<int> seqs;
    a.integers(&seqs);
    return made(a.plain, [&] { return g_close((rv_pool)pool, (int)seqs.size(), seqs.data()); });
  });
}

template <class T>
int64_t sum(const std::vector<T>& v) {
  int64_t t = 0;
  for (T x : v) t += x;
  return t;
}

// append(pool, n_heads, device, stream, seqs, K, V, n_rows)
PyObject* py_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 8);
    if (!a.plain) Py_RETURN_NONE;
    void* pool = a.address();
    const int64_t H = a.integer(), dev = a.integer();
    void* s = a.address();
    std::vector<int> seqs, rows;
    a.integers(&seqs);
    Args r(args + 7, 1, 1);
    r.integers(&rows);
    if (!r.plain || rows.size() != seqs.size()) a.plain = false;
    const int64_t total = sum(rows);
    void *K = a.exact(dev, kBF16, {total, H, kHeadDim}), *V = a.exact(dev, kBF16, {total, H, kHeadDim});
    return made(a.plain, [&] { return g_append((rv_pool)pool, (int)seqs.size(), seqs.data(), K, V, rows.data(), s); });
  });
}

// gather(pool, n_heads, device, stream, seqs, n_rows, first, K, V)
PyObject* py_gather(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 9);
    if (!a.plain) Py_RETURN_NONE;
    void* pool = a.address();
    const int64_t H = a.integer(), dev = a.integer();
    void* s = a.address();
    std::vector<int> seqs;
    std::vector<int64_t> rows, first;
    a.integers(&seqs);
    a.integers(&rows);
    const bool has_first = a.integers(&first, true);
    if (rows.size() != seqs.size() || (has_first && first.size() != seqs.size())) a.plain = false;
    const int64_t size = sum(rows) * H * kHeadDim;
    if (size < 0) a.plain = false;
    void *K = a.exact(dev, kBF16, {-size - 1}), *V = a.exact(dev, kBF16, {-size - 1});
    return made(a.plain, [&] {
      return g_gather((rv_pool)pool, (int)seqs.size(), seqs.data(), has_first ? first.data() : nullptr, rows.data(), K, V, s);
    });
  });
}

// compact(pool, n_heads, device, stream, seqs, n_keep, first, keep)
PyObject* py_compact(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 8);
    if (!a.plain) Py_RETURN_NONE;
    void* pool = a.address();
    const int64_t H = a.integer(), dev = a.integer();
    void* s = a.address();
    std::vector<int> seqs;
    std::vector<int64_t> keeps, first;
    a.integers(&seqs);
    a.integers(&keeps);
    const bool has_first = a.integers(&first, true);
    if (keeps.size() != seqs.size() || (has_first && first.size() != seqs.size())) a.plain = false;
    const int64_t size = sum(keeps) * H;
    if (size < 0) a.plain = false;
    void* keep = a.exact(dev, c10::ScalarType::Int, {-size - 1});
    return made(a.plain, [&] {
      return g_compact((rv_pool)pool, (int)seqs.size(), seqs.data(), has_first ? first.data() : nullptr, keeps.data(),
                       (const int32_t*)keep, s);
    });
  });
}

// attend(pool, n_heads, device, stream, seqs, n_tokens, Q, K, V, out, lse)
PyObject* py_attend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 11);
    if (!a.plain) Py_RETURN_NONE;
    void* pool = a.address();
    const int64_t H = a.integer(), dev = a.integer();
    void* s = a.address();
    std::vector<int> seqs, tokens;
    a.integers(&seqs);
    a.integers(&tokens);
    if (tokens.size() != seqs.size() || !THPVariable_CheckExact(args[6])) a.plain = false;
    const int64_t total = sum(tokens);
    if (!a.plain || total < 0 || THPVariable_Unpack(args[6]).dim() != 3) Py_RETURN_NONE;
    const int64_t hq = THPVariable_Unpack(args[6]).size(1);
    void *Q = a.exact(dev, kBF16, {total, hq, kHeadDim}), *K = a.exact(dev, kBF16, {total, H, kHeadDim}),
         *V = a.exact(dev, kBF16, {total, H, kHeadDim}), *out = a.exact(dev, kBF16, {total, hq, kHeadDim});
    void* lse = a.exact(dev, c10::ScalarType::Float, {-total * hq - 1});
    return made(a.plain && hq == (int)hq, [&] {
      return g_attend((rv_pool)pool, (int)seqs.size(), seqs.data(), tokens.data(), Q, K, V, (int)hq, out, (float*)lse, s);
    });
  });
}

// setup_calls(addresses of rv_prepare_qkv, rv_prepare_qkv_bwd, rv_pool_fork, rv_pool_close, rv_pool_append,
//             rv_pool_gather, rv_pool_compact, rv_attend_seqs)
PyObject* py_setup_calls(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 8) return PyErr_Format(PyExc_TypeError, "setup_calls takes 8 arguments (%zd given)", n);
  void* f[8];
  for (int i = 0; i < 8; ++i)
    if (!(f[i] = PyLong_AsVoidPtr(args[i])))
      return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "NULL function");
  g_prepare = reinterpret_cast<decltype(g_prepare)>(f[0]);
  g_prepare_bwd = reinterpret_cast<decltype(g_prepare_bwd)>(f[1]);
  g_fork = reinterpret_cast<decltype(g_fork)>(f[2]);
  g_close = reinterpret_cast<decltype(g_close)>(f[3]);
  g_append = reinterpret_cast<decltype(g_append)>(f[4]);
  g_gather = reinterpret_cast<decltype(g_gather)>(f[5]);
  g_compact = reinterpret_cast<decltype(g_compact)>(f[6]);
  g_attend = reinterpret_cast<decltype(g_attend)>(f[7]);
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"ptr", (PyCFunction)(void (*)(void))py_ptr, METH_FASTCALL, nullptr},
    {"ptrs", (PyCFunction)(void (*)(void))py_ptrs, METH_FASTCALL, nullptr},
    {"mem_state", py_mem_state, METH_O, nullptr},
    {"prepare", (PyCFunction)(void (*)(void))py_prepare, METH_FASTCALL, nullptr},
    {"prepare_bwd", (PyCFunction)(void (*)(void))py_prepare_bwd, METH_FASTCALL, nullptr},
    {"fork", (PyCFunction)(void (*)(void))py_fork, METH_FASTCALL, nullptr},
    {"release", (PyCFunction)(void (*)(void))py_release, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)(void))py_append, METH_FASTCALL, nullptr},
    {"gather", (PyCFunction)(void (*)(void))py_gather, METH_FASTCALL, nullptr},
    {"compact", (PyCFunction)(void (*)(void))py_compact, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))py_attend, METH_FASTCALL, nullptr},
    {"setup_calls", (PyCFunction)(void (*)(void))py_setup_calls, METH_FASTCALL, nullptr},
    {"setup", (PyCFunction)(void (*)(void))py_setup, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_rv_bind", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and Python whose headers this was compiled with.  It reads their
// objects directly, so rv.py loads it with the same ones only.
PyMODINIT_FUNC PyInit__rv_bind(void) {
  PyObject* m = PyModule_Create(&kModule);
  if (m && PyModule_AddObject(m, "built_for", Py_BuildValue("(sii)", TORCH_VERSION, PY_MAJOR_VERSION, PY_MINOR_VERSION)))
    Py_CLEAR(m);
  return m;
}
