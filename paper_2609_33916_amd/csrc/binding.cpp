// Native form of the Python entry points a program calls per step (attn_fwd,
// attn_fwd_bwd, attn_bwd, attn_decode, attn_rope, attn_rope_bwd, attn_paged_append,
// attn_paged_gather, attn_paged_decode): argument checks, output and workspace
// allocation and the call into the library, without per-argument Python work.
//
// Each function answers NotImplemented, having done nothing, for anything but
// plain arguments that pass every check (tensors of exactly torch.Tensor, strided,
// on one GPU, contiguous (or, where views are taken, with a contiguous last
// axis), of matching types and shapes; numbers of exactly int,
// float or bool). The Python form then runs, with its full checks and errors.
// A status code of the library other than 0 is answered as an int.
//
// The library is reached through the addresses that bind() and bind_paged() receive, so both
// forms call the same loaded library.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/TensorSubclassLikeUtils.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

namespace {

using WsFn = size_t (*)(int, int, int, int);
using DecWsFn = size_t (*)(int, int, int, int, int, int);
using FwdFn = int (*)(const void*, const void*, const void*, void*, float*, int, int, int, int, float, int, int, void*);
using FwdBwdFn = int (*)(const void*, const void*, const void*, const void*, void*, float*, void*, void*, void*, void*,
                         size_t, int, int, int, int, float, int, int, void*);
using BwdFn = int (*)(const void*, const void*, const void*, const void*, const float*, const void*, void*, void*, void*,
                      void*, size_t, int, int, int, int, float, int, int, void*);
using DecodeFn = int (*)(const void*, const void*, const void*, void*, void*, const int*, void*, float*, void*, size_t,
                         int, int, int, int, int, int, float, int, void*);

WsFn ws_bytes;
DecWsFn dec_ws_bytes;
FwdFn c_fwd;
FwdBwdFn c_fwd_bwd;
BwdFn c_bwd;
DecodeFn c_decode;
PyObject* raw_stream;   // device index -> the current stream's handle

PyObject* not_mine() { Py_RETURN_NOTIMPLEMENTED; }

// a dense, contiguous GPU tensor of exactly torch.Tensor
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.is_contiguous() || at::isTensorSubclassLike(t))
    return nullptr;
  return &t;
}
bool like(const at::Tensor* t, const at::Tensor& ref) {
  return t && t->scalar_type() == ref.scalar_type() && t->device() == ref.device() && t->sizes() == ref.sizes();
}
bool is(const at::Tensor* t, at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& ref) {
  return t && t->scalar_type() == type && t->device() == ref.device() && t->sizes() == sizes;
}
int dtype_code(const at::Tensor& t) {
  return t.scalar_type() == at::kBFloat16 ? 0 : t.scalar_type() == at::kFloat ? 1 : -1;
}
bool fits_int(at::IntArrayRef sizes) {
  for (int64_t s : sizes)
    if (s > INT_MAX) return false;
  return true;
}
bool get_scale(PyObject* o, int64_t d, float& s) {
  if (o == Py_None) {
    s = (float)(1.0 / std::sqrt((double)d));
    return d > 0;
  }
  if (!PyFloat_CheckExact(o)) return false;
  s = (float)PyFloat_AS_DOUBLE(o);
  return true;
}
bool get_stream(const at::Tensor& t, void*& st) {
  PyObject* idx = PyLong_FromLong(t.get_device());
  if (!idx) return false;
  PyObject* r = PyObject_CallOneArg(raw_stream, idx);
  Py_DECREF(idx);
  if (!r) return false;
  st = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !PyErr_Occurred();
}
// the caller's workspace, or a new one of `need` bytes (at least one) in `own`
bool get_workspace(PyObject* o, size_t need, const at::Tensor& ref, at::Tensor& own, void*& p, size_t& bytes) {
  if (o == Py_None) {
    bytes = std::max<size_t>(need, 1);
    own = at::empty({(int64_t)bytes}, ref.options().dtype(at::kByte));
    p = own.data_ptr();
    return true;
  }
  const at::Tensor* t = plain(o);
  if (!t || t->device() != ref.device()) return false;
  bytes = t->nbytes();
  p = t->data_ptr();
  return bytes >= need;
}
// N outputs: the caller's tuple, or new tensors; output `l` is the float32 row
// vector (-1: none), the others are like `ref`
template <int N> struct Outputs {
  at::Tensor t[N];
  void* p[N];
  bool get(PyObject* o, const at::Tensor& ref, int l) {
    const auto rows = ref.sizes().slice(0, ref.dim() - 1);
    if (o == Py_None) {
      for (int i = 0; i < N; ++i) {
        t[i] = i == l ? at::empty(rows, ref.options().dtype(at::kFloat)) : at::empty_like(ref);
        p[i] = t[i].data_ptr();
      }
      return true;
    }
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != N) return false;
    for (int i = 0; i < N; ++i) {
      const at::Tensor* x = plain(PyTuple_GET_ITEM(o, i));
      if (!(i == l ? is(x, rows, at::kFloat, ref) : like(x, ref))) return false;
      p[i] = x->data_ptr();
    }
    return true;
  }
  PyObject* answer(PyObject* o) {
    if (o != Py_None) return Py_NewRef(o);
    PyObject* r = PyTuple_New(N);
    if (!r) return nullptr;
    for (int i = 0; i < N; ++i) {
      PyObject* x = THPVariable_Wrap(std::move(t[i]));
      if (!x) {
        Py_DECREF(r);
        return nullptr;
      }
      PyTuple_SET_ITEM(r, i, x);
    }
    return r;
  }
};
// C++ exceptions (a failed allocation) become the Python errors torch gives
template <typename F> PyObject* guarded(F f) {
  HANDLE_TH_ERRORS
  return f();
  END_HANDLE_TH_ERRORS
}
template <typename F> int released(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return rc;
}

// fwd(q, k, v, scale, causal, out)
PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    if (na != 6) return not_mine();
    const at::Tensor *q = plain(a[0]), *k = plain(a[1]), *v = plain(a[2]);
    float scale;
    if (!q || q->dim() != 4 || !like(k, *q) || !like(v, *q) || !PyBool_Check(a[4]) || !fits_int(q->sizes()) ||
        dtype_code(*q) < 0 || !get_scale(a[3], q->size(3), scale))
      return not_mine();
    Outputs<2> out;
    if (!out.get(a[5], *q, 1)) return not_mine();
    void* st;
    if (!get_stream(*q, st)) return nullptr;
    const auto s = q->sizes();
    const int rc = released([&] {
      return c_fwd(q->data_ptr(), k->data_ptr(), v->data_ptr(), out.p[0], (float*)out.p[1], s[0], s[1], s[2], s[3], scale,
                   a[4] == Py_True, dtype_code(*q), st);
    });
    return rc ? PyLong_FromLong(rc) : out.answer(a[5]);
  });
}

// fwd_bwd(q, k, v, do, scale, causal, out, workspace)
PyObject* fwd_bwd(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    if (na != 8) return not_mine();
    const at::Tensor *q = plain(a[0]), *k = plain(a[1]), *v = plain(a[2]), *g = plain(a[3]);
    float scale;
    if (!q || q->dim() != 4 || !like(k, *q) || !like(v, *q) || !like(g, *q) || !PyBool_Check(a[5]) ||
        !fits_int(q->sizes()) || dtype_code(*q) < 0 || !get_scale(a[4], q->size(3), scale))
      return not_mine();
    const auto s = q->sizes();
    Outputs<5> out;
    at::Tensor own;
    void *ws, *st;
    size_t bytes;
    if (!out.get(a[6], *q, 1) || !get_workspace(a[7], ws_bytes(s[0], s[1], s[2], s[3]), *q, own, ws, bytes)) return not_mine();
    if (!get_stream(*q, st)) return nullptr;
    const int rc = released([&] {
      return c_fwd_bwd(q->data_ptr(), k->data_ptr(), v->data_ptr(), g->data_ptr(), out.p[0], (float*)out.p[1], out.p[2],
                       out.p[3], out.p[4], ws, bytes, s[0], s[1], s[2], s[3], scale, a[5] == Py_True, dtype_code(*q), st);
    });
    return rc ? PyLong_FromLong(rc) : out.answer(a[6]);
  });
}

// bwd(q, k, v, o, lse, do, scale, causal, out, workspace)
PyObject* bwd(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    if (na != 10) return not_mine();
    const at::Tensor *q = plain(a[0]), *k = plain(a[1]), *v = plain(a[2]), *o = plain(a[3]), *l = plain(a[4]), *g = plain(a[5]);
    float scale;
    if (!q || q->dim() != 4 || !like(k, *q) || !like(v, *q) || !like(o, *q) || !like(g, *q) ||
        !is(l, q->sizes().slice(0, 3), at::kFloat, *q) || !PyBool_Check(a[7]) || !fits_int(q->sizes()) ||
        dtype_code(*q) < 0 || !get_scale(a[6], q->size(3), scale))
      return not_mine();
    const auto s = q->sizes();
    Outputs<3> out;
    at::Tensor own;
    void *ws, *st;
    size_t bytes;
    if (!out.get(a[8], *q, -1) || !get_workspace(a[9], ws_bytes(s[0], s[1], s[2], s[3]), *q, own, ws, bytes)) return not_mine();
    if (!get_stream(*q, st)) return nullptr;
    const int rc = released([&] {
      return c_bwd(q->data_ptr(), k->data_ptr(), v->data_ptr(), o->data_ptr(), (const float*)l->data_ptr(), g->data_ptr(),
                   out.p[0], out.p[1], out.p[2], ws, bytes, s[0], s[1], s[2], s[3], scale, a[7] == Py_True, dtype_code(*q), st);
    });
    return rc ? PyLong_FromLong(rc) : out.answer(a[8]);
  });
}

// decode(q, k_cache, v_cache, k_new, v_new, cache_lens, n, scale, out, workspace)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    if (na != 10) return not_mine();
    const at::Tensor *q = plain(a[0]), *kc = plain(a[1]), *vc = plain(a[2]), *kn = nullptr, *vn = nullptr, *lens = nullptr;
    float scale;
    if (!q || q->dim() != 3 || !kc || kc->dim() != 4 || !like(vc, *kc) || kc->scalar_type() != q->scalar_type() ||
        kc->device() != q->device() || kc->size(0) != q->size(0) || kc->size(3) != q->size(2) || !fits_int(q->sizes()) ||
        !fits_int(kc->sizes()) || dtype_code(*q) < 0 || !PyLong_CheckExact(a[6]) || !get_scale(a[7], q->size(2), scale))
      return not_mine();
    const int64_t B = q->size(0), Hq = q->size(1), d = q->size(2), Hkv = kc->size(1), n_cap = kc->size(2);
    if (a[3] != Py_None) {
      const int64_t rows[3] = {B, Hkv, d};
      kn = plain(a[3]), vn = plain(a[4]);
      if (!is(kn, rows, q->scalar_type(), *q) || !is(vn, rows, q->scalar_type(), *q)) return not_mine();
    }
    if (a[5] != Py_None) {
      lens = plain(a[5]);
      if (!is(lens, {B}, at::kInt, *q)) return not_mine();
    }
    int over;
    const long n = PyLong_AsLongAndOverflow(a[6], &over);
    if (over || n < INT_MIN || n > INT_MAX) return not_mine();
    if (n == -1 && PyErr_Occurred()) return nullptr;
    Outputs<2> out;
    if (!out.get(a[8], *q, 1)) return not_mine();
    const size_t need = dec_ws_bytes(B, Hq, Hkv, n, d, kn != nullptr);
    at::Tensor own;
    void *ws = nullptr, *st;
    size_t bytes = 0;
    if ((need > 0 || a[9] != Py_None) && !get_workspace(a[9], need, *q, own, ws, bytes)) return not_mine();
    if (!get_stream(*q, st)) return nullptr;
    const int rc = released([&] {
      return c_decode(q->data_ptr(), kn ? kn->data_ptr() : nullptr, vn ? vn->data_ptr() : nullptr, kc->data_ptr(),
                      vc->data_ptr(), lens ? (const int*)lens->data_ptr() : nullptr, out.p[0], (float*)out.p[1], ws, bytes,
                      B, Hq, Hkv, n, n_cap, d, scale, dtype_code(*q), st);
    });
    return rc ? PyLong_FromLong(rc) : out.answer(a[8]);
  });
}

// bind(workspace_bytes, decode_workspace_bytes, fwd, fwd_bwd, bwd, decode
//      [addresses], function that gives a device's current raw stream)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t na) {
  if (na != 7) {
    PyErr_SetString(PyExc_TypeError, "bind takes six addresses and a function");
    return nullptr;
  }
  void* p[6];
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: null address");
      return nullptr;
    }
  }
  ws_bytes = (WsFn)p[0];
  dec_ws_bytes = (DecWsFn)p[1];
  c_fwd = (FwdFn)p[2];
  c_fwd_bwd = (FwdBwdFn)p[3];
  c_bwd = (BwdFn)p[4];
  c_decode = (DecodeFn)p[5];
  Py_XSETREF(raw_stream, Py_NewRef(a[6]));
  Py_RETURN_NONE;
}

// ------------------------------------------- rotary positions, paged cache --
using RopeFn = int (*)(const void*, const void*, void*, void*, const long long*, const double*, const int*, long long, int,
                       int, int, int, int, int, int, float, int, int, void*);
using AppendFn = int (*)(const void*, const void*, const long long*, void*, void*, void*, void*, const int*, const int*,
                         const int*, const double*, const int*, int, int, int, int, int, int, int, int, float, int, int,
                         void*);
using GatherFn = int (*)(const void*, const void*, const void*, const void*, const int*, const int*, const int*, void*,
                         void*, int, int, int, int, int, int, int, int, void*);
using PagedWsFn = size_t (*)(int, int, int, int, int, int, int);
using PagedFn = int (*)(const void*, const void*, const void*, const long long*, void*, void*, void*, void*, const int*,
                        const int*, const double*, const int*, void*, float*, void*, size_t, int, int, int, int, int, int,
                        int, int, int, float, int, float, int, void*);

RopeFn c_rope[2];
AppendFn c_append;
GatherFn c_gather;
PagedWsFn paged_ws_bytes;
PagedFn c_paged;

// a strided GPU tensor of exactly torch.Tensor whose last axis is contiguous
const at::Tensor* rows(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.dim() < 1 || t.stride(-1) != 1 ||
      at::isTensorSubclassLike(t))
    return nullptr;
  return &t;
}
// an optional int32 tensor of `sizes`
bool get_ints(PyObject* o, at::IntArrayRef sizes, const at::Tensor& ref, const int*& p) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = plain(o);
  if (!is(t, sizes, at::kInt, ref)) return false;
  p = (const int*)t->data_ptr();
  return true;
}
// an optional table of frequencies for rows of d columns
bool get_rotation(PyObject* o, int64_t d, const at::Tensor& ref, const double*& p, int& r) {
  p = nullptr;
  r = 0;
  if (o == Py_None) return true;
  const at::Tensor* t = plain(o);
  if (!t || t->scalar_type() != at::kDouble || t->device() != ref.device() || t->dim() != 1 || t->numel() == 0 || 2 * t->numel() > d)
    return false;
  p = (const double*)t->data_ptr();
  r = (int)(2 * t->numel());
  return true;
}
bool get_float(PyObject* o, float& f) {
  if (!PyFloat_CheckExact(o)) return false;
  f = (float)PyFloat_AS_DOUBLE(o);
  return true;
}
bool get_int(PyObject* o, int& i) {
  if (!PyLong_CheckExact(o)) return false;
  int over;
  const long v = PyLong_AsLongAndOverflow(o, &over);
  if (over || v < INT_MIN || v > INT_MAX) return false;
  i = (int)v;
  return true;
}

// rope(q, k, freqs, amplitude, interleaved, positions, start, out, backward)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    if (na != 9) return not_mine();
    const at::Tensor *q = rows(a[0]), *k = nullptr;
    float amplitude;
    int start, r;
    const double* freqs;
    if (!q || q->dim() != 4 || dtype_code(*q) < 0 || !fits_int(q->sizes()) || a[2] == Py_None || !get_float(a[3], amplitude) ||
        !PyBool_Check(a[4]) || !get_int(a[6], start) || !PyBool_Check(a[8]) || !get_rotation(a[2], q->size(3), *q, freqs, r))
      return not_mine();
    const int64_t B = q->size(0), Hq = q->size(1), n = q->size(2), d = q->size(3);
    int64_t Hk = 0;
    if (a[1] != Py_None) {
      k = rows(a[1]);
      if (!k || k->dim() != 4) return not_mine();
      Hk = k->size(1);
      const int64_t want[4] = {B, Hk, n, d};
      if (!is(k, want, q->scalar_type(), *q) || Hk > INT_MAX) return not_mine();
    }
    const int* pos = nullptr;
    bool per_sequence = false;
    if (a[5] != Py_None) {
      const at::Tensor* p = plain(a[5]);
      per_sequence = p && p->dim() == 2;
      if (!(per_sequence ? is(p, {B, n}, at::kInt, *q) : is(p, {n}, at::kInt, *q))) return not_mine();
      pos = (const int*)p->data_ptr();
    }
    at::Tensor own[2];
    const at::Tensor* out[2] = {nullptr, nullptr};
    if (a[7] == Py_None) {
      own[0] = at::empty(q->sizes(), q->options());
      out[0] = &own[0];
      if (k) {
        own[1] = at::empty(k->sizes(), k->options());
        out[1] = &own[1];
      }
    } else {
      if (!PyTuple_CheckExact(a[7]) || PyTuple_GET_SIZE(a[7]) != 2) return not_mine();
      out[0] = rows(PyTuple_GET_ITEM(a[7], 0));
      if (!like(out[0], *q)) return not_mine();
      if (k) {
        out[1] = rows(PyTuple_GET_ITEM(a[7], 1));
        if (!like(out[1], *k)) return not_mine();
      } else if (PyTuple_GET_ITEM(a[7], 1) != Py_None) {
        return not_mine();
      }
    }
    long long strides[12];
    const at::Tensor* all[4] = {q, k, out[0], out[1]};
    for (int i = 0; i < 12; ++i) strides[i] = all[i / 3] ? all[i / 3]->stride(i % 3) : 0;
    const c10::DeviceGuard device(q->device());
    void* st;
    if (!get_stream(*q, st)) return nullptr;
    const int rc = released([&] {
      return c_rope[a[8] == Py_True](q->data_ptr(), k ? k->data_ptr() : nullptr, out[0]->data_ptr(),
                                     k ? out[1]->data_ptr() : nullptr, strides, freqs, pos, per_sequence ? n : 0,
                                     pos ? 0 : start, B, Hq, Hk, n, d, r, amplitude, a[4] == Py_True, dtype_code(*q), st);
    });
    if (rc) return PyLong_FromLong(rc);
    if (a[7] != Py_None) return Py_NewRef(a[7]);
    PyObject* x = THPVariable_Wrap(std::move(own[0]));
    PyObject* y = k ? THPVariable_Wrap(std::move(own[1])) : Py_NewRef(Py_None);
    PyObject* both = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
  });
}

// a pool, its tables and what they say of the sizes
struct Pool {
  const at::Tensor *kp, *vp, *ks = nullptr, *vs = nullptr;
  const int *table, *lens;
  int64_t B, Hkv, P, ps, width, d;
  bool get(PyObject* k, PyObject* v, PyObject* ksc, PyObject* vsc, PyObject* t, PyObject* l) {
    kp = plain(k), vp = plain(v);
    if (!kp || kp->dim() != 4 || !like(vp, *kp) || (ksc == Py_None) != (vsc == Py_None) || !fits_int(kp->sizes())) return false;
    const bool four = ksc != Py_None;
    if (kp->scalar_type() != (four ? at::kByte : at::kBFloat16)) return false;
    P = kp->size(0), Hkv = kp->size(1), ps = kp->size(2), d = kp->size(3) * (four ? 2 : 1);
    if (four) {
      const int64_t want[4] = {P, Hkv, ps, d / 32};
      ks = plain(ksc), vs = plain(vsc);
      if (!is(ks, want, at::kByte, *kp) || !is(vs, want, at::kByte, *kp)) return false;
    }
    const at::Tensor* tab = plain(t);
    if (!tab || tab->dim() != 2 || tab->scalar_type() != at::kInt || tab->device() != kp->device() || !fits_int(tab->sizes()))
      return false;
    B = tab->size(0), width = tab->size(1);
    table = (const int*)tab->data_ptr();
    return l != Py_None && get_ints(l, {B}, *kp, lens);
  }
  void* scale(const at::Tensor* t) const { return t ? t->data_ptr() : nullptr; }
};

// paged_append(k_new, v_new, k_pages, v_pages, block_table, lens, new_lens, k_scales, v_scales, freqs, amplitude,
//              interleaved, positions)
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    Pool p;
    if (na != 13 || !p.get(a[2], a[3], a[7], a[8], a[4], a[5])) return not_mine();
    const at::Tensor *k = rows(a[0]), *v = rows(a[1]);
    if (!k || k->dim() != 4) return not_mine();
    const int64_t T = k->size(2), want[4] = {p.B, p.Hkv, T, p.d};
    const int *news, *pos;
    const double* freqs;
    float amplitude;
    int r;
    if (!is(k, want, at::kBFloat16, *p.kp) || !is(v, want, at::kBFloat16, *p.kp) || T > INT_MAX ||
        !get_ints(a[6], {p.B}, *p.kp, news) || !get_rotation(a[9], p.d, *p.kp, freqs, r) || !get_float(a[10], amplitude) ||
        !PyBool_Check(a[11]) || !get_ints(a[12], {p.B, T}, *p.kp, pos))
      return not_mine();
    const long long strides[6] = {k->stride(0), k->stride(1), k->stride(2), v->stride(0), v->stride(1), v->stride(2)};
    const c10::DeviceGuard device(p.kp->device());
    void* st;
    if (!get_stream(*p.kp, st)) return nullptr;
    const int rc = released([&] {
      return c_append(k->data_ptr(), v->data_ptr(), strides, p.kp->data_ptr(), p.vp->data_ptr(), p.scale(p.ks),
                      p.scale(p.vs), p.table, p.lens, news, freqs, pos, p.B, p.Hkv, T, p.P, p.ps, p.width, p.d, r,
                      amplitude, a[11] == Py_True, 0, st);
    });
    if (rc) return PyLong_FromLong(rc);
    Py_RETURN_NONE;
  });
}

// paged_gather(k_pages, v_pages, block_table, lens, n, starts, k_scales, v_scales, out)
PyObject* paged_gather(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    Pool p;
    int n;
    const int* starts;
    if (na != 9 || !p.get(a[0], a[1], a[6], a[7], a[2], a[3]) || !get_int(a[4], n) || n < 1 ||
        !get_ints(a[5], {p.B}, *p.kp, starts))
      return not_mine();
    const int64_t want[4] = {p.B, p.Hkv, n, p.d};
    at::Tensor own[2];
    const at::Tensor* out[2];
    if (a[8] == Py_None) {
      for (int i = 0; i < 2; ++i) out[i] = &(own[i] = at::empty(want, p.kp->options().dtype(at::kBFloat16)));
    } else {
      if (!PyTuple_CheckExact(a[8]) || PyTuple_GET_SIZE(a[8]) != 2) return not_mine();
      for (int i = 0; i < 2; ++i) {
        out[i] = plain(PyTuple_GET_ITEM(a[8], i));
        if (!is(out[i], want, at::kBFloat16, *p.kp)) return not_mine();
      }
    }
    const c10::DeviceGuard device(p.kp->device());
    void* st;
    if (!get_stream(*p.kp, st)) return nullptr;
    const int rc = released([&] {
      return c_gather(p.kp->data_ptr(), p.vp->data_ptr(), p.scale(p.ks), p.scale(p.vs), p.table, p.lens, starts,
                      out[0]->data_ptr(), out[1]->data_ptr(), p.B, p.Hkv, n, p.P, p.ps, p.width, p.d, 0, st);
    });
    if (rc) return PyLong_FromLong(rc);
    if (a[8] != Py_None) return Py_NewRef(a[8]);
    PyObject *x = THPVariable_Wrap(std::move(own[0])), *y = THPVariable_Wrap(std::move(own[1]));
    PyObject* both = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
  });
}

// paged_decode(q, k_pages, v_pages, block_table, lens, k_new, v_new, n, scale, k_scales, v_scales, freqs, amplitude,
//              interleaved, positions, out, workspace)
PyObject* paged_decode(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    Pool p;
    if (na != 17 || !p.get(a[1], a[2], a[9], a[10], a[3], a[4])) return not_mine();
    const at::Tensor *q = rows(a[0]), *kn = nullptr, *vn = nullptr;
    if (!q || q->dim() != 3) return not_mine();
    const int64_t Hq = q->size(1);
    const int64_t want_q[3] = {p.B, Hq, p.d}, want_kv[3] = {p.B, p.Hkv, p.d};
    auto dense_heads = [&](const at::Tensor* t) { return t->size(1) == 1 || t->stride(1) == p.d; };
    if (!is(q, want_q, at::kBFloat16, *p.kp) || !dense_heads(q) || Hq > INT_MAX) return not_mine();
    if ((a[5] == Py_None) != (a[6] == Py_None)) return not_mine();
    if (a[5] != Py_None) {
      kn = rows(a[5]), vn = rows(a[6]);
      if (!is(kn, want_kv, at::kBFloat16, *p.kp) || !is(vn, want_kv, at::kBFloat16, *p.kp) || !dense_heads(kn) ||
          !dense_heads(vn))
        return not_mine();
    }
    int n, r;
    float scale, amplitude;
    const double* freqs;
    const int* pos;
    if (a[7] == Py_None) n = (int)std::min<int64_t>(p.width * p.ps - (kn != nullptr), INT_MAX - 2047);
    else if (!get_int(a[7], n)) return not_mine();
    if (!get_scale(a[8], p.d, scale) || !get_rotation(a[11], p.d, *p.kp, freqs, r) || !get_float(a[12], amplitude) ||
        !PyBool_Check(a[13]) || !get_ints(a[14], {p.B}, *p.kp, pos))
      return not_mine();
    Outputs<2> out;
    if (a[15] == Py_None) {   // dense, whatever q's strides
      out.t[0] = at::empty(want_q, q->options());
      out.t[1] = at::empty({p.B, Hq}, q->options().dtype(at::kFloat));
      for (int i = 0; i < 2; ++i) out.p[i] = out.t[i].data_ptr();
    } else if (!out.get(a[15], *q, 1)) {
      return not_mine();
    }
    const size_t need = paged_ws_bytes(p.B, Hq, p.Hkv, n, p.d, kn != nullptr, p.ks ? 4 : 16);
    at::Tensor own;
    void *ws = nullptr, *st;
    size_t bytes = 0;
    if ((need > 0 || a[16] != Py_None) && !get_workspace(a[16], need, *q, own, ws, bytes)) return not_mine();
    const long long strides[3] = {q->stride(0), kn ? kn->stride(0) : 0, kn ? vn->stride(0) : 0};
    const c10::DeviceGuard device(q->device());
    if (!get_stream(*q, st)) return nullptr;
    const int rc = released([&] {
      return c_paged(q->data_ptr(), kn ? kn->data_ptr() : nullptr, vn ? vn->data_ptr() : nullptr, strides,
                     p.kp->data_ptr(), p.vp->data_ptr(), p.scale(p.ks), p.scale(p.vs), p.table, p.lens, freqs, pos, out.p[0],
                     (float*)out.p[1], ws, bytes, p.B, Hq, p.Hkv, n, p.P, p.ps, p.width, p.d, r, amplitude,
                     a[13] == Py_True, scale, 0, st);
    });
    return rc ? PyLong_FromLong(rc) : out.answer(a[15]);
  });
}

// bind_paged(rope, rope_bwd, paged_append, paged_gather, paged_decode_workspace_bytes, paged_decode [addresses])
PyObject* bind_paged(PyObject*, PyObject* const* a, Py_ssize_t na) {
  if (na != 6) {
    PyErr_SetString(PyExc_TypeError, "bind_paged takes six addresses");
    return nullptr;
  }
  void* p[6];
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind_paged: null address");
      return nullptr;
    }
  }
  c_rope[0] = (RopeFn)p[0];
  c_rope[1] = (RopeFn)p[1];
  c_append = (AppendFn)p[2];
  c_gather = (GatherFn)p[3];
  paged_ws_bytes = (PagedWsFn)p[4];
  c_paged = (PagedFn)p[5];
  Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL
PyMethodDef methods[] = {{"bind", FAST(bind), nullptr},       {"fwd", FAST(fwd), nullptr}, {"fwd_bwd", FAST(fwd_bwd), nullptr},
                         {"bwd", FAST(bwd), nullptr},         {"decode", FAST(decode), nullptr},
                         {"bind_paged", FAST(bind_paged), nullptr}, {"rope", FAST(rope), nullptr},
                         {"paged_append", FAST(paged_append), nullptr}, {"paged_gather", FAST(paged_gather), nullptr},
                         {"paged_decode", FAST(paged_decode), nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
