// The op calls of the Python binding, marshalled in native code.
//
// A short kernel's call from Python is host work: for a float32 RMSNorm of
// 1024 x 128 the interpreter's shape checks, stride and pointer queries and
// argument conversion took 4.5 of the call's 7.0 us. A Handle (one per
// SpecCache) takes the same tensors in one C call: it makes the binding's
// checks on the unpacked tensors, allocates the outputs that were not given
// and issues the entry call.
//
// Only the plain case is taken here: exact torch.Tensor / Parameter operands
// on the cache's device, float32 or bfloat16, of the expected shapes and
// strides, no torch function or dispatch mode, default stream or a stream
// object. For anything else -- wrong arguments included -- a method returns
// None before it has done anything, and the Python method of the same name
// makes its checks and raises its errors. A MISS is handled by the owner's
// _on_miss, as in the Python methods.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/TensorSubclassLikeUtils.h>
#include <c10/core/StreamGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "tri.h"

namespace {

PyObject *g_error = nullptr;        // TriError
PyObject *g_rope_ext = nullptr;     // the ctypes structures
PyObject *g_chain_args = nullptr;

struct Handle {
  PyObject_HEAD
  tri_cache *cache;                 // null once the cache is closed
  int dev;
};

// Releases the GIL for its lifetime, as a ctypes call does.
struct NoGil {
  PyThreadState *s = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(s); }
};

// A plain tensor on GPU `dev`, or null.
const at::Tensor *plain(PyObject *o, int dev) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided ||
      t.device().index() != dev || at::isTensorSubclassLike(t) || t._is_zerotensor())
    return nullptr;
  return &t;
}

int dtype_of(const at::Tensor &t) {
  switch (t.scalar_type()) {
    case at::kFloat: return TRI_F32;
    case at::kBFloat16: return TRI_BF16;
    default: return -1;
  }
}

bool same(const at::Tensor &t, const at::Tensor &like) {
  return t.scalar_type() == like.scalar_type() && t.sizes() == like.sizes();
}

bool weight(const at::Tensor &t, int64_t n, const at::Tensor &like) {
  return t.dim() == 1 && t.size(0) == n && t.scalar_type() == like.scalar_type() &&
         (n <= 1 || t.stride(0) == 1);
}

// Row stride of a [T, W] tensor with unit inner stride, or -1; a single row
// reports at least W.
int64_t rows(const at::Tensor &t) {
  const int64_t T = t.size(0), W = t.size(1), s = t.stride(0);
  if (W > 1 && t.stride(1) != 1) return -1;
  return T > 1 || s >= W ? s : W;
}

// Token stride of a [T, nh, hd] tensor with packed heads, or -1.
int64_t tokens(const at::Tensor &t) {
  const int64_t T = t.size(0), nh = t.size(1), hd = t.size(2), s = t.stride(0);
  if ((hd > 1 && t.stride(2) != 1) || (nh > 1 && t.stride(1) != hd)) return -1;
  return T > 1 || s >= nh * hd ? s : nh * hd;
}

bool number(PyObject *o, float *v) {
  if (!PyFloat_Check(o) && !PyLong_Check(o)) return false;
  const double d = PyFloat_AsDouble(o);
  if (d == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *v = float(d);
  return true;
}

bool stream_of(const Handle *h, PyObject *o, void **s) {
  if (o == Py_None) {
    *s = c10::hip::getCurrentHIPStream(c10::DeviceIndex(h->dev)).stream();
    return true;
  }
  PyObject *p = PyObject_GetAttrString(o, "cuda_stream");
  if (p) {
    *s = PyLong_AsVoidPtr(p);
    Py_DECREF(p);
  }
  if (!PyErr_Occurred()) return true;
  PyErr_Clear();
  return false;
}

// While it lives torch allocates on the call's stream `s` (given as `o`), where
// the outputs and workspaces made meanwhile are written: their memory is handed
// on only after that work. Nothing where no stream was given: it is the current.
// (The allocator knows streams by their address, so any wrapper of it will do.)
struct MakingOn {
  c10::OptionalStreamGuard g;
  MakingOn(const Handle *h, PyObject *o, void *s) {
    if (o == Py_None) return;
    const auto d = c10::DeviceIndex(h->dev);
    g.reset_stream(c10::Stream(c10::Stream::UNSAFE, c10::Device(at::kCUDA, d),
                               c10::hip::getStreamFromExternal(hipStream_t(s), d).id()));
  }
};

bool modes() {
  return at::impl::torch_function_mode_enabled() ||
         c10::impl::TorchDispatchModeTLS::any_modes_set();
}

// The bytes of a ctypes structure of class `type` (which the caller keeps
// alive), or null.
void *structure(PyObject *o, PyObject *type, size_t size) {
  if (reinterpret_cast<PyObject *>(Py_TYPE(o)) != type) return nullptr;
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
    PyErr_Clear();
    return nullptr;
  }
  void *p = size_t(b.len) >= size ? b.buf : nullptr;
  PyBuffer_Release(&b);
  return p;
}

// `call` until it no longer misses, at most `misses` times handled by the
// owner's _on_miss; raises TriError for any other status. True on OK.
template <class F>
bool issue(PyObject *owner, const char *what, F &&call, int64_t misses = 1) {
  int st;
  {
    NoGil g;
    st = call();
  }
  for (int64_t i = 0; st == TRI_MISS && i < misses; ++i) {
    PyObject *r = PyObject_CallMethod(owner, "_on_miss", nullptr);
    if (!r) return false;
    Py_DECREF(r);
    NoGil g;
    st = call();
  }
  if (st == TRI_OK) return true;
  if (PyObject *e = PyObject_CallFunction(g_error, "is", st, what)) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return false;
}

// An output: the tensor given (checked against `like`), or a new one.
struct Out {
  at::Tensor t;
  PyObject *given = nullptr;
  bool take(PyObject *o, const at::Tensor &like, const Handle *h, PyObject *stream, void *s) {
    if (o == Py_None) {
      MakingOn on(h, stream, s);
      NoGil g;
      t = at::empty_like(like);
      return true;
    }
    const at::Tensor *p = plain(o, h->dev);
    if (!p || !same(*p, like)) return false;
    t = *p;
    given = o;
    return true;
  }
  PyObject *result() {
    if (!given) return THPVariable_Wrap(std::move(t));
    Py_INCREF(given);
    return given;
  }
};

PyObject *pair(PyObject *a, PyObject *b) {
  if (!a || !b) {
    Py_XDECREF(a);
    Py_XDECREF(b);
    return nullptr;
  }
  PyObject *r = PyTuple_Pack(2, a, b);
  Py_DECREF(a);
  Py_DECREF(b);
  return r;
}

// A method: `n` positional arguments after the owner; not the plain case or
// a C++ exception (nothing has been launched then): None.
typedef PyObject *(*Body)(Handle *h, PyObject *owner, PyObject *const *a);
template <Body B, int N>
PyObject *method(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  Handle *h = reinterpret_cast<Handle *>(self);
  if (n != N + 1 || !h->cache || modes()) Py_RETURN_NONE;
  try {
    return B(h, args[0], args + 1);
  } catch (...) {
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
}

// rmsnorm(owner, x, w, eps, out, stream)
PyObject *rmsnorm(Handle *h, PyObject *owner, PyObject *const *a) {
  const at::Tensor *x = plain(a[0], h->dev), *w = plain(a[1], h->dev);
  float eps;
  void *s;
  if (!x || !w || x->dim() != 2 || dtype_of(*x) < 0 || !weight(*w, x->size(1), *x) ||
      !number(a[2], &eps) || !stream_of(h, a[4], &s))
    Py_RETURN_NONE;
  const int64_t T = x->size(0), H = x->size(1), xs = rows(*x);
  Out y;
  if (xs < 0 || !y.take(a[3], *x, h, a[4], s)) Py_RETURN_NONE;
  const int64_t ys = rows(y.t);
  if (ys < 0) Py_RETURN_NONE;
  const tri_dtype dt = tri_dtype(dtype_of(*x));
  const void *xp = x->data_ptr(), *wp = w->data_ptr();
  void *yp = y.t.data_ptr();
  if (!issue(owner, "tri_rmsnorm",
             [&] { return tri_rmsnorm(h->cache, dt, xp, xs, wp, yp, ys, T, H, eps, s); }))
    return nullptr;
  return y.result();
}

// residual_rmsnorm(owner, x, residual, w, eps, out, residual_out, stream)
PyObject *residual_rmsnorm(Handle *h, PyObject *owner, PyObject *const *a) {
  const at::Tensor *x = plain(a[0], h->dev), *r = plain(a[1], h->dev), *w = plain(a[2], h->dev);
  float eps;
  void *s;
  if (!x || !r || !w || x->dim() != 2 || dtype_of(*x) < 0 || !same(*r, *x) ||
      !weight(*w, x->size(1), *x) || !number(a[3], &eps) || !stream_of(h, a[6], &s))
    Py_RETURN_NONE;
  const int64_t T = x->size(0), H = x->size(1), xs = rows(*x), rs = rows(*r);
  Out y, o;
  if (xs < 0 || rs < 0 || !y.take(a[4], *x, h, a[6], s) ||
      !o.take(a[5], *r, h, a[6], s))
    Py_RETURN_NONE;
  const int64_t ys = rows(y.t), os = rows(o.t);
  if (ys < 0 || os < 0) Py_RETURN_NONE;
  const tri_dtype dt = tri_dtype(dtype_of(*x));
  const void *xp = x->data_ptr(), *rp = r->data_ptr(), *wp = w->data_ptr();
  void *yp = y.t.data_ptr(), *op = o.t.data_ptr();
  if (!issue(owner, "tri_residual_rmsnorm", [&] {
        return tri_residual_rmsnorm(h->cache, dt, xp, xs, rp, rs, wp, yp, ys, op, os, T, H, eps, s);
      }))
    return nullptr;
  return pair(y.result(), o.result());
}

// Two inputs and an output of one shape [T, W] (swiglu, add), or one input
// (silu): (owner, a, [b,] out, stream).
template <int OP>
PyObject *flat(Handle *h, PyObject *owner, PyObject *const *a) {
  constexpr bool one = OP == TRI_OP_SILU;
  const at::Tensor *x = plain(a[0], h->dev);
  const at::Tensor *b = one ? x : plain(a[1], h->dev);
  PyObject *const *rest = a + (one ? 1 : 2);
  void *s;
  if (!x || !b || x->dim() != 2 || dtype_of(*x) < 0 || !same(*b, *x) || !stream_of(h, rest[1], &s))
    Py_RETURN_NONE;
  const int64_t T = x->size(0), W = x->size(1), xs = rows(*x), bs = rows(*b);
  Out y;
  if (xs < 0 || bs < 0 || !y.take(rest[0], *x, h, rest[1], s)) Py_RETURN_NONE;
  const int64_t ys = rows(y.t);
  if (ys < 0) Py_RETURN_NONE;
  const tri_dtype dt = tri_dtype(dtype_of(*x));
  const void *xp = x->data_ptr(), *bp = b->data_ptr();
  void *yp = y.t.data_ptr();
  const char *what = OP == TRI_OP_SWIGLU ? "tri_swiglu" : one ? "tri_silu" : "tri_add";
  if (!issue(owner, what, [&] {
        if constexpr (OP == TRI_OP_SWIGLU)
          return tri_swiglu(h->cache, dt, xp, xs, bp, bs, yp, ys, T, W, s);
        else if constexpr (one)
          return tri_silu(h->cache, dt, xp, xs, yp, ys, T, W, s);
        else
          return tri_add(h->cache, dt, xp, xs, bp, bs, yp, ys, T, W, s);
      }))
    return nullptr;
  return y.result();
}

// masked_fill(owner, x, mask, value, out, stream)
PyObject *masked_fill(Handle *h, PyObject *owner, PyObject *const *a) {
  const at::Tensor *x = plain(a[0], h->dev), *m = plain(a[1], h->dev);
  float value;
  void *s;
  if (!x || !m || x->dim() != 2 || dtype_of(*x) < 0 || m->sizes() != x->sizes() ||
      (m->scalar_type() != at::kByte && m->scalar_type() != at::kBool) || !number(a[2], &value) ||
      !stream_of(h, a[4], &s))
    Py_RETURN_NONE;
  const int64_t T = x->size(0), W = x->size(1), xs = rows(*x), ms = rows(*m);
  Out y;
  if (xs < 0 || ms < 0 || !y.take(a[3], *x, h, a[4], s)) Py_RETURN_NONE;
  const int64_t ys = rows(y.t);
  if (ys < 0) Py_RETURN_NONE;
  const tri_dtype dt = tri_dtype(dtype_of(*x));
  const void *xp = x->data_ptr();
  const uint8_t *mp = static_cast<const uint8_t *>(m->data_ptr());
  void *yp = y.t.data_ptr();
  if (!issue(owner, "tri_masked_fill", [&] {
        return tri_masked_fill(h->cache, dt, xp, xs, mp, ms, value, yp, ys, T, W, s);
      }))
    return nullptr;
  return y.result();
}

// embedding(owner, table, ids, out, stream)
PyObject *embedding(Handle *h, PyObject *owner, PyObject *const *a) {
  const at::Tensor *t = plain(a[0], h->dev), *ids = plain(a[1], h->dev);
  void *s;
  if (!t || !ids || t->dim() != 2 || dtype_of(*t) < 0 || ids->dim() != 1 ||
      (ids->scalar_type() != at::kInt && ids->scalar_type() != at::kLong) ||
      !stream_of(h, a[3], &s))
    Py_RETURN_NONE;
  const int64_t n = t->size(0), H = t->size(1), T = ids->size(0), ts = rows(*t);
  if (ts < 0 || (T > 1 && ids->stride(0) != 1)) Py_RETURN_NONE;
  Out y;
  if (a[2] == Py_None) {
    MakingOn on(h, a[3], s);
    NoGil g;
    y.t = at::empty({T, H}, t->options());
  } else {
    const at::Tensor *o = plain(a[2], h->dev);
    if (!o || o->dim() != 2 || o->size(0) != T || o->size(1) != H ||
        o->scalar_type() != t->scalar_type())
      Py_RETURN_NONE;
    y.t = *o;
    y.given = a[2];
  }
  const int64_t ys = rows(y.t);
  if (ys < 0) Py_RETURN_NONE;
  const tri_dtype dt = tri_dtype(dtype_of(*t));
  const void *tp = t->data_ptr(), *ip = ids->data_ptr();
  const int32_t wide = ids->scalar_type() == at::kLong;
  void *yp = y.t.data_ptr();
  if (!issue(owner, "tri_embedding", [&] {
        return tri_embedding(h->cache, dt, tp, ts, n, ip, wide, yp, ys, T, H, s);
      }))
    return nullptr;
  return y.result();
}

// The rotation: (owner, q, k, pos, base, ext, q_w, k_w, eps, stream, kind),
// kind 0: tri_rope_qk, 1: tri_qk_norm_rope, 2: tri_rope_qk_ext.
PyObject *rope(Handle *h, PyObject *owner, PyObject *const *a) {
  const at::Tensor *q = plain(a[0], h->dev), *pos = plain(a[2], h->dev);
  const at::Tensor *k = nullptr, *qw = nullptr, *kw = nullptr;
  float base, eps;
  void *s;
  if (!q || !pos || q->dim() != 3 || dtype_of(*q) < 0 || !number(a[3], &base) ||
      !number(a[7], &eps) || !stream_of(h, a[8], &s))
    Py_RETURN_NONE;
  const int64_t T = q->size(0), nq = q->size(1), hd = q->size(2), qs = tokens(*q);
  if (qs < 0 || nq > INT32_MAX || hd > INT32_MAX) Py_RETURN_NONE;
  const tri_rope_ext *ext = nullptr;
  if (a[4] != Py_None) {
    ext = static_cast<const tri_rope_ext *>(structure(a[4], g_rope_ext, sizeof(tri_rope_ext)));
    if (!ext) Py_RETURN_NONE;
    if (ext->cos_sin) {
      // the table's tensor travels with the struct: its width and device
      // must be what the kernels read through the bare address
      PyObject *to = PyObject_GetAttrString(a[4], "_cos_sin");
      if (!to) {
        PyErr_Clear();
        Py_RETURN_NONE;
      }
      const at::Tensor *t = plain(to, h->dev);
      const bool ok = t && t->dim() == 2 && t->size(1) == (ext->rotary_dim ? ext->rotary_dim : hd);
      Py_DECREF(to);
      if (!ok) Py_RETURN_NONE;
    }
  }
  int64_t nk = 0, ks = 0;
  void *kp = nullptr;
  if (a[1] != Py_None) {
    k = plain(a[1], h->dev);
    if (!k || k->dim() != 3 || k->size(0) != T || k->size(2) != hd ||
        k->scalar_type() != q->scalar_type() || k->size(1) > INT32_MAX)
      Py_RETURN_NONE;
    nk = k->size(1);
    if (nk) {
      ks = tokens(*k);
      if (ks < 0) Py_RETURN_NONE;
      kp = k->data_ptr();
    }
  }
  if (pos->dim() != 1 || pos->size(0) != T || (T > 1 && pos->stride(0) != 1) ||
      pos->scalar_type() != (ext && ext->pos_int64 ? at::kLong : at::kInt))
    Py_RETURN_NONE;
  if (a[5] != Py_None && (!(qw = plain(a[5], h->dev)) || !weight(*qw, hd, *q))) Py_RETURN_NONE;
  if (a[6] != Py_None && (!(kw = plain(a[6], h->dev)) || !weight(*kw, hd, *q))) Py_RETURN_NONE;
  const long kind = PyLong_AsLong(a[9]);
  if (kind == 1 && !qw) Py_RETURN_NONE;
  const tri_dtype dt = tri_dtype(dtype_of(*q));
  void *qp = q->data_ptr(), *pp = pos->data_ptr();
  const void *qwp = qw ? qw->data_ptr() : nullptr, *kwp = kw ? kw->data_ptr() : nullptr;
  const int32_t q_ = int32_t(nq), k_ = int32_t(nk), d_ = int32_t(hd);
  const char *what = kind == 0 ? "tri_rope_qk" : kind == 1 ? "tri_qk_norm_rope" : "tri_rope_qk_ext";
  if (!issue(owner, what, [&] {
        if (kind == 0)
          return tri_rope_qk(h->cache, dt, qp, qs, kp, ks, static_cast<const int32_t *>(pp), T, q_,
                             k_, d_, base, s);
        if (kind == 1)
          return tri_qk_norm_rope(h->cache, dt, qp, qs, kp, ks, static_cast<const int32_t *>(pp),
                                  T, q_, k_, d_, base, qwp, kwp, eps, s);
        return tri_rope_qk_ext(h->cache, dt, qp, qs, kp, ks, pp, T, q_, k_, d_, base, ext, qwp,
                               kwp, eps, s);
      }))
    return nullptr;
  return PyTuple_Pack(2, a[0], a[1]);
}

bool integer(PyObject *o, int64_t *v) {
  if (!PyLong_CheckExact(o)) return false;
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *v = x;
  return true;
}

// n contiguous integers (at least n with `more`) of type `st` on GPU `dev`.
template <class T>
bool integers(PyObject *o, int dev, at::ScalarType st, int64_t n, bool more, T **p) {
  const at::Tensor *t = plain(o, dev);
  if (!t || t->dim() != 1 || t->scalar_type() != st || (more ? t->size(0) < n : t->size(0) != n) ||
      (t->size(0) > 1 && t->stride(0) != 1))
    return false;
  *p = static_cast<T *>(t->data_ptr());
  return true;
}

// A block table [R, cols]: its size and row stride.
bool block_table(PyObject *o, int dev, int32_t **p, int64_t *R, int64_t *cols, int64_t *rs,
                 const at::Tensor **out) {
  const at::Tensor *t = plain(o, dev);
  if (!t || t->dim() != 2 || t->scalar_type() != at::kInt || t->size(0) > INT32_MAX ||
      t->size(1) > INT32_MAX)
    return false;
  *R = t->size(0);
  *cols = t->size(1);
  *rs = rows(*t);
  *p = static_cast<int32_t *>(t->data_ptr());
  *out = t;
  return *rs >= 0;
}

// The cache of k and v [n_pages, page, nk, hd] of type `st`; a dimension
// of one reports what a packed cache has.
bool kv_cache(PyObject *ko, PyObject *vo, int dev, at::ScalarType st, tri_kv_cache *c) {
  const at::Tensor *k = plain(ko, dev), *v = plain(vo, dev);
  if (!k || !v || k->dim() != 4 || k->scalar_type() != st || !same(*v, *k)) return false;
  const int64_t n = k->size(0), page = k->size(1), nk = k->size(2), hd = k->size(3);
  if (n > INT32_MAX || page > INT32_MAX || nk > INT32_MAX || hd > INT32_MAX) return false;
  const auto view = [&](const at::Tensor &t, int64_t *ps, int64_t *ss, int64_t *hs) {
    if (hd > 1 && t.stride(3) != 1) return false;
    *hs = nk > 1 ? t.stride(2) : hd;
    *ss = page > 1 ? t.stride(1) : std::max(hd, nk * *hs);
    *ps = n > 1 ? t.stride(0) : page * std::max(*ss, nk * *hs);
    return true;
  };
  c->k = k->data_ptr();
  c->v = v->data_ptr();
  c->n_pages = int32_t(n);
  c->page = int32_t(page);
  c->nk = int32_t(nk);
  c->hd = int32_t(hd);
  return view(*k, &c->k_ps, &c->k_ss, &c->k_hs) && view(*v, &c->v_ps, &c->v_ss, &c->v_hs);
}

// kv_slots(owner, kv_len, new_len, block_table, free_pages, free_count, page,
// T, slots, pos, q_start, kv_len_out, free_out, stream)
PyObject *kv_slots(Handle *h, PyObject *owner, PyObject *const *a) {
  tri_kv_slots_args x{};
  const at::Tensor *table;
  int64_t R, cols, page;
  void *s;
  int32_t *kv, *more, *count, *stack = nullptr;
  const at::Tensor *fp = plain(a[3], h->dev);
  if (!block_table(a[2], h->dev, &x.table, &R, &cols, &x.table_rs, &table) ||
      !integers(a[0], h->dev, at::kInt, R, false, &kv) ||
      !integers(a[1], h->dev, at::kInt, R, false, &more) || !fp || fp->size(0) > INT32_MAX ||
      !integers(a[3], h->dev, at::kInt, 0, true, &stack) ||
      !integers(a[4], h->dev, at::kInt, 1, true, &count) || !integer(a[5], &page) ||
      page > INT32_MAX || page < INT32_MIN || !integer(a[6], &x.T) || x.T < 0 ||
      !stream_of(h, a[12], &s))
    Py_RETURN_NONE;
  x.R = int32_t(R);
  x.cols = int32_t(cols);
  x.page = int32_t(page);
  x.n_free = int32_t(fp->size(0));
  x.kv_len = kv;
  x.new_len = more;
  x.free_pages = stack;
  x.free_count = count;
  const int64_t n[5] = {x.T, x.T, R + 1, R, 2};
  void *p[5];
  for (int i = 0; i < 5; ++i) {
    if (a[7 + i] == Py_None) continue;
    int32_t *q;
    if (i == 0 ? !integers(a[7], h->dev, at::kLong, n[0], false, &x.slots)
               : !integers(a[7 + i], h->dev, at::kInt, n[i], false, &q))
      Py_RETURN_NONE;
    p[i] = i == 0 ? static_cast<void *>(x.slots) : q;
  }
  // those not given: the step's (slots, pos, q_start) share one allocation,
  // what the next step takes (kv_len_out, free_out) another
  at::Tensor made[5];
  {
    MakingOn on(h, a[12], s);
    NoGil g;
    for (int b = 0; b < 5; b = b ? 5 : 3) {
      const int e = b ? 5 : 3;
      int64_t at[5], bytes = 0;
      for (int i = b; i < e; ++i) {
        at[i] = bytes;
        if (a[7 + i] == Py_None) bytes += (n[i] * (i ? 4 : 8) + 15) / 16 * 16;
      }
      if (!bytes) continue;
      const at::Tensor all = at::empty({bytes}, table->options().dtype(at::kByte));
      for (int i = b; i < e; ++i) {
        if (a[7 + i] != Py_None) continue;
        made[i] = at::detail::make_tensor<c10::TensorImpl>(
            c10::Storage(all.storage()), all.key_set(),
            c10::scalarTypeToTypeMeta(i ? at::kInt : at::kLong));
        made[i].unsafeGetTensorImpl()->set_sizes_contiguous({n[i]});
        made[i].unsafeGetTensorImpl()->set_storage_offset(at[i] / (i ? 4 : 8));
        p[i] = static_cast<char *>(all.data_ptr()) + at[i];
      }
    }
  }
  x.slots = static_cast<int64_t *>(p[0]);
  x.pos = static_cast<int32_t *>(p[1]);
  x.q_start = static_cast<int32_t *>(p[2]);
  x.kv_len_out = static_cast<int32_t *>(p[3]);
  x.free_out = static_cast<int32_t *>(p[4]);
  if (!issue(owner, "tri_kv_slots", [&] { return tri_kv_slots(h->cache, &x, s); })) return nullptr;
  PyObject *r = PyTuple_New(5);
  if (!r) return nullptr;
  for (int i = 0; i < 5; ++i) {
    PyObject *o = a[7 + i];
    if (o == Py_None) {
      o = THPVariable_Wrap(std::move(made[i]));
      if (!o) {
        Py_DECREF(r);
        return nullptr;
      }
    } else {
      Py_INCREF(o);
    }
    PyTuple_SET_ITEM(r, i, o);
  }
  return r;
}

// kv_write(owner, k, v, slots, k_cache, v_cache, stream)
PyObject *kv_write(Handle *h, PyObject *owner, PyObject *const *a) {
  const at::Tensor *k = plain(a[0], h->dev), *v = plain(a[1], h->dev);
  tri_kv_cache c;
  int64_t *slots;
  void *s;
  if (!k || !v || k->dim() != 3 || dtype_of(*k) < 0 || !same(*v, *k) ||
      !integers(a[2], h->dev, at::kLong, k->size(0), false, &slots) ||
      !kv_cache(a[3], a[4], h->dev, k->scalar_type(), &c) || c.nk != k->size(1) || c.hd != k->size(2) ||
      !stream_of(h, a[5], &s))
    Py_RETURN_NONE;
  const int64_t T = k->size(0), ks = tokens(*k), vs = tokens(*v);
  if (ks < 0 || vs < 0) Py_RETURN_NONE;
  const tri_dtype dt = tri_dtype(dtype_of(*k));
  const void *kp = k->data_ptr(), *vp = v->data_ptr();
  if (!issue(owner, "tri_kv_write",
             [&] { return tri_kv_write(h->cache, dt, kp, ks, vp, vs, slots, T, &c, s); }))
    return nullptr;
  return PyTuple_Pack(2, a[3], a[4]);
}

// The cache of 8-bit codes and its scales at a[0 .. 3]: k_cache, v_cache, k_scale, v_scale.
bool kv_q8(PyObject *const *a, int dev, tri_kv_cache *c, tri_kv_q8 *q) {
  const at::Tensor *k = plain(a[0], dev), *ks = plain(a[2], dev), *vs = plain(a[3], dev);
  if (!k || !ks || !vs) return false;
  const at::ScalarType st = k->scalar_type();
  if ((st != at::kChar && st != at::kFloat8_e4m3fn) || !kv_cache(a[0], a[1], dev, st, c)) return false;
  if (ks->dim() != 3 || ks->scalar_type() != at::kFloat || !same(*vs, *ks)) return false;
  const int64_t n = ks->size(0), blocks = ks->size(1), nk = ks->size(2);
  if (n != c->n_pages || nk != c->nk || blocks < 1 || c->page % blocks) return false;
  q->code = st == at::kChar ? TRI_INT8 : TRI_E4M3;
  q->block = int32_t(c->page / blocks);
  const auto view = [&](const at::Tensor &t, float **p, int64_t *ps, int64_t *bs, int64_t *hs) {
    *p = static_cast<float *>(t.data_ptr());
    *hs = nk > 1 ? t.stride(2) : 1;
    *bs = blocks > 1 ? t.stride(1) : nk * *hs;
    *ps = n > 1 ? t.stride(0) : blocks * std::max(*bs, nk * *hs);
  };
  view(*ks, &q->k_scale, &q->k_ps, &q->k_bs, &q->k_hs);
  view(*vs, &q->v_scale, &q->v_ps, &q->v_bs, &q->v_hs);
  return true;
}

// Rows k, v of a call over an 8-bit cache whose codes and scales, table, lengths and starts are
// a[0 .. 6].
bool rows_q8(const at::Tensor &k, const at::Tensor &v, PyObject *const *a, int dev,
             tri_kv_rows_args *x) {
  int64_t R, cols;
  int32_t *tp, *kv, *starts;
  const at::Tensor *table;
  if (!block_table(a[4], dev, &tp, &R, &cols, &x->table_rs, &table) ||
      !integers(a[5], dev, at::kInt, R, false, &kv) ||
      !integers(a[6], dev, at::kInt, R + 1, false, &starts) || x->kv.nk != k.size(1) ||
      x->kv.hd != k.size(2))
    return false;
  x->dtype = dtype_of(k);
  x->R = int32_t(R);
  x->T = k.size(0);
  x->k = k.data_ptr();
  x->k_ts = tokens(k);
  x->v = v.data_ptr();
  x->v_ts = tokens(v);
  x->table = tp;
  x->kv_len = kv;
  x->q_start = starts;
  x->cols = int32_t(cols);
  return x->k_ts >= 0 && x->v_ts >= 0;
}

// kv_write_q8(owner, k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, q_start,
// stream)
PyObject *kv_write_q8(Handle *h, PyObject *owner, PyObject *const *a) {
  const at::Tensor *k = plain(a[0], h->dev), *v = plain(a[1], h->dev);
  tri_kv_rows_args x{};
  void *s;
  if (!k || !v || k->dim() != 3 || dtype_of(*k) < 0 || !same(*v, *k) ||
      !kv_q8(a + 2, h->dev, &x.kv, &x.q8) || !rows_q8(*k, *v, a + 2, h->dev, &x) ||
      !stream_of(h, a[9], &s))
    Py_RETURN_NONE;
  if (!issue(owner, "tri_kv_write_quant", [&] { return tri_kv_write_quant(h->cache, &x, s); }))
    return nullptr;
  return PyTuple_Pack(4, a[2], a[3], a[4], a[5]);
}

// kv_read_q8(owner, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, q_start, T, dtype, k, v,
// stream)
PyObject *kv_read_q8(Handle *h, PyObject *owner, PyObject *const *a) {
  tri_kv_rows_args x{};
  int64_t T;
  void *s;
  if (!kv_q8(a, h->dev, &x.kv, &x.q8) || !integer(a[7], &T) || T < 0 || !THPDtype_Check(a[8]) ||
      !stream_of(h, a[11], &s))
    Py_RETURN_NONE;
  const at::ScalarType st = reinterpret_cast<THPDtype *>(a[8])->scalar_type;
  if (st != at::kFloat && st != at::kBFloat16) Py_RETURN_NONE;
  Out o[2];
  for (int i = 0; i < 2; ++i) {
    if (a[9 + i] == Py_None) continue;
    const at::Tensor *t = plain(a[9 + i], h->dev);
    if (!t || t->dim() != 3 || t->scalar_type() != st || t->size(0) != T || t->size(1) != x.kv.nk ||
        t->size(2) != x.kv.hd)
      Py_RETURN_NONE;
    o[i].t = *t;
    o[i].given = a[9 + i];
  }
  {
    MakingOn on(h, a[11], s);
    NoGil g;
    for (Out &y : o)
      if (!y.given)
        y.t = at::empty({T, x.kv.nk, x.kv.hd},
                        at::TensorOptions().dtype(st).device(at::kCUDA, c10::DeviceIndex(h->dev)));
  }
  if (!rows_q8(o[0].t, o[1].t, a, h->dev, &x)) Py_RETURN_NONE;
  if (!issue(owner, "tri_kv_read_quant", [&] { return tri_kv_read_quant(h->cache, &x, s); }))
    return nullptr;
  return pair(o[0].result(), o[1].result());
}

// paged_attention(owner, q, k_cache, v_cache, block_table, kv_len, q_start,
// scale, window, max_kv, out, stream), and paged_attention_q8 with k_scale and v_scale after
// v_cache.
template <bool Q8>
PyObject *paged_attention(Handle *h, PyObject *owner, PyObject *const *args) {
  const at::Tensor *q = plain(args[0], h->dev), *table;
  PyObject *const *a = args + (Q8 ? 2 : 0);   // (block_table and what follows at a[3])
  tri_attention_args x{};
  tri_kv_q8 q8{};
  int64_t R, cols, window;
  int32_t *tp, *kv, *starts;
  void *s;
  if (!q || q->dim() != 3 || dtype_of(*q) < 0 || q->size(1) > INT32_MAX ||
      !(Q8 ? kv_q8(args + 1, h->dev, &x.kv, &q8)
           : kv_cache(args[1], args[2], h->dev, q->scalar_type(), &x.kv)) ||
      x.kv.hd != q->size(2) ||
      !block_table(a[3], h->dev, &tp, &R, &cols, &x.table_rs, &table) ||
      !integers(a[4], h->dev, at::kInt, R, false, &kv) ||
      !integers(a[5], h->dev, at::kInt, R + 1, false, &starts) ||
      !integer(a[7], &window) || window > INT32_MAX || window < INT32_MIN ||
      !integer(a[8], &x.max_kv) || !stream_of(h, a[10], &s))
    Py_RETURN_NONE;
  if (a[6] == Py_None)
    x.scale = float(1.0 / std::sqrt(double(q->size(2))));
  else if (!number(a[6], &x.scale))
    Py_RETURN_NONE;
  Out y;
  if (a[9] == Py_None && !q->is_contiguous()) Py_RETURN_NONE;
  if (!y.take(a[9], *q, h, a[10], s)) Py_RETURN_NONE;
  x.dtype = dtype_of(*q);
  x.nq = int32_t(q->size(1));
  x.T = q->size(0);
  x.R = int32_t(R);
  x.cols = int32_t(cols);
  x.q = q->data_ptr();
  x.q_ts = tokens(*q);
  x.out = y.t.data_ptr();
  x.o_ts = tokens(y.t);
  if (x.q_ts < 0 || x.o_ts < 0) Py_RETURN_NONE;
  x.table = tp;
  x.kv_len = kv;
  x.q_start = starts;
  x.window = int32_t(window);
  at::Tensor work;
  if (const int64_t need = Q8 ? tri_paged_attention_quant_workspace(&x)
                              : tri_paged_attention_workspace(&x)) {
    MakingOn on(h, a[10], s);
    NoGil g;
    work = at::empty({need}, q->options().dtype(at::kByte));
    x.workspace = work.data_ptr();
    x.workspace_bytes = need;
  }
  if (!issue(owner, Q8 ? "tri_paged_attention_quant" : "tri_paged_attention", [&] {
        return Q8 ? tri_paged_attention_quant(h->cache, &x, &q8, s)
                  : tri_paged_attention(h->cache, &x, s);
      }))
    return nullptr;
  return y.result();
}

// decode_chain_args(owner, args, stream)
PyObject *chain(Handle *h, PyObject *owner, PyObject *const *a) {
  const void *p = structure(a[0], g_chain_args, sizeof(tri_chain_args));
  void *s;
  if (!p || !stream_of(h, a[1], &s)) Py_RETURN_NONE;
  if (!issue(owner, "tri_decode_chain", [&] {
        return tri_decode_chain(h->cache, static_cast<const tri_chain_args *>(p), s);
      }))
    return nullptr;
  Py_RETURN_TRUE;
}

// decode_chain_layers(owner, list of args, stream)
PyObject *layers(Handle *h, PyObject *owner, PyObject *const *a) {
  void *s;
  if (!PyList_CheckExact(a[0]) || !stream_of(h, a[1], &s)) Py_RETURN_NONE;
  const Py_ssize_t n = PyList_GET_SIZE(a[0]);
  std::vector<tri_chain_args> v;
  v.reserve(size_t(n) + 1);
  for (Py_ssize_t i = 0; i < n; ++i) {
    const void *p = structure(PyList_GET_ITEM(a[0], i), g_chain_args, sizeof(tri_chain_args));
    if (!p) Py_RETURN_NONE;
    v.push_back(*static_cast<const tri_chain_args *>(p));
  }
  if (n > TRI_MAX_LAYERS) Py_RETURN_NONE;
  if (!issue(owner, "tri_decode_chain_layers",
             [&] { return tri_decode_chain_layers(h->cache, v.data(), uint32_t(n), s); }, n))
    return nullptr;
  Py_RETURN_TRUE;
}

PyObject *close(PyObject *self, PyObject *) {
  reinterpret_cast<Handle *>(self)->cache = nullptr;
  Py_RETURN_NONE;
}

template <Body B, int N>
PyCFunction fn() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&method<B, N>));
}

PyMethodDef g_methods[] = {
    {"rmsnorm", fn<rmsnorm, 5>(), METH_FASTCALL, nullptr},
    {"residual_rmsnorm", fn<residual_rmsnorm, 7>(), METH_FASTCALL, nullptr},
    {"swiglu", fn<flat<TRI_OP_SWIGLU>, 4>(), METH_FASTCALL, nullptr},
    {"silu", fn<flat<TRI_OP_SILU>, 3>(), METH_FASTCALL, nullptr},
    {"add", fn<flat<TRI_OP_ADD>, 4>(), METH_FASTCALL, nullptr},
    {"masked_fill", fn<masked_fill, 5>(), METH_FASTCALL, nullptr},
    {"embedding", fn<embedding, 4>(), METH_FASTCALL, nullptr},
    {"rope", fn<rope, 10>(), METH_FASTCALL, nullptr},
    {"kv_slots", fn<kv_slots, 13>(), METH_FASTCALL, nullptr},
    {"kv_write", fn<kv_write, 6>(), METH_FASTCALL, nullptr},
    {"paged_attention", fn<paged_attention<false>, 11>(), METH_FASTCALL, nullptr},
    {"kv_write_q8", fn<kv_write_q8, 10>(), METH_FASTCALL, nullptr},
    {"kv_read_q8", fn<kv_read_q8, 12>(), METH_FASTCALL, nullptr},
    {"paged_attention_q8", fn<paged_attention<true>, 13>(), METH_FASTCALL, nullptr},
    {"chain", fn<chain, 2>(), METH_FASTCALL, nullptr},
    {"layers", fn<layers, 2>(), METH_FASTCALL, nullptr},
    {"close", close, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};

// Handle(cache address, device index)
PyObject *handle_new(PyTypeObject *type, PyObject *args, PyObject *) {
  unsigned long long p;
  int dev;
  if (!PyArg_ParseTuple(args, "Ki", &p, &dev)) return nullptr;
  Handle *h = reinterpret_cast<Handle *>(type->tp_alloc(type, 0));
  if (h) {
    h->cache = reinterpret_cast<tri_cache *>(p);
    h->dev = dev;
  }
  return reinterpret_cast<PyObject *>(h);
}

void handle_free(PyObject *self) {
  PyTypeObject *type = Py_TYPE(self);
  type->tp_free(self);
  Py_DECREF(type);
}

PyType_Slot g_slots[] = {{Py_tp_new, reinterpret_cast<void *>(&handle_new)},
                         {Py_tp_dealloc, reinterpret_cast<void *>(&handle_free)},
                         {Py_tp_methods, g_methods},
                         {0, nullptr}};
PyType_Spec g_spec = {"paper_2609_37241_amd._fast.Handle", int(sizeof(Handle)), 0,
                      Py_TPFLAGS_DEFAULT, g_slots};

// setup(TriError, RopeExt, ChainArgs)
PyObject *setup(PyObject *, PyObject *args) {
  PyObject *e, *r, *c;
  if (!PyArg_ParseTuple(args, "OOO", &e, &r, &c)) return nullptr;
  Py_INCREF(e);
  Py_INCREF(r);
  Py_INCREF(c);
  g_error = e;
  g_rope_ext = r;
  g_chain_args = c;
  Py_RETURN_NONE;
}

PyMethodDef g_functions[] = {{"setup", setup, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_fast", nullptr, -1, g_functions,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast() {
  PyObject *m = PyModule_Create(&g_module);
  if (!m) return nullptr;
  PyObject *type = PyType_FromSpec(&g_spec);
  if (!type || PyModule_AddObject(m, "Handle", type) < 0) {
    Py_XDECREF(type);
    Py_DECREF(m);
    return nullptr;
  }
  // what the package compares with the torch it runs on
  if (PyModule_AddStringConstant(m, "torch_version", TRI_TORCH_VERSION) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
