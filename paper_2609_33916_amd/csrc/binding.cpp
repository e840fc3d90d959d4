// Native form of the Python entry points a program calls per step (attn_fwd,
// attn_fwd_bwd, attn_bwd, attn_decode, attn_rope, attn_rope_bwd, attn_paged_append,
// attn_paged_gather, attn_paged_decode, attn_cross_fwd, attn_cross_bwd, attn_prefix_decode): argument checks, output and workspace
// allocation and the call into the library, without per-argument Python work.
//
// Each function answers NotImplemented, having done nothing, for anything but
// plain arguments that pass every check (tensors of exactly torch.Tensor, strided,
// on one GPU, contiguous (or, where views are taken, with a contiguous last
// axis), of matching types and shapes; numbers of exactly int,
// float or bool). The Python form then runs, with its full checks and errors.
// A status code of the library other than 0 is answered as an int.
//
// The library is reached through the addresses that the bind functions receive, so both
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

// --------------------------------- keys of another length, shared prefix --
using CrossWsFn = size_t (*)(int, int, int, int, int, int, int, int);
using CrossFwdFn = int (*)(const void*, const void*, const void*, void*, float*, const long long*, const int*, const int*, int,
                           const void*, const int*, int, int, int, void*, size_t, int, int, int, int, int, int, float, int, int,
                           void*);
using CrossBwdFn = int (*)(const void*, const void*, const void*, const void*, const float*, const void*, void*, void*, void*,
                           void*, const long long*, const int*, const int*, int, const void*, const int*, int, int, int, void*,
                           size_t, int, int, int, int, int, int, float, int, int, void*);
using PrefixWsFn = size_t (*)(int, int, int, int, int, int);
using PrefixFn = int (*)(const void*, const void*, const void*, const void*, const void*, void*, void*, const int*, void*, float*,
                         void*, size_t, int, int, int, int, int, int, int, float, int, void*);

CrossWsFn cross_fwd_ws, cross_bwd_ws;
CrossFwdFn c_cross_fwd;
CrossBwdFn c_cross_bwd;
PrefixWsFn prefix_ws;
PrefixFn c_prefix;

// what the forward and the backward share: q, k, v, and scale, causal, start, starts, k_lens, bias, bias_rows, bias_first
struct Cross {
  const at::Tensor *q, *k, *v, *bias = nullptr;
  int64_t B, Hq, Hkv, nq, nk, d;
  float scale;
  bool causal;
  int start, first, R = 0, buckets = 0;
  const int *lens, *starts, *bias_rows = nullptr;
  bool get(PyObject* const* qkv, PyObject* const* a) {
    q = rows(qkv[0]), k = rows(qkv[1]), v = rows(qkv[2]);
    if (!q || q->dim() != 4 || dtype_code(*q) < 0 || !fits_int(q->sizes()) || !k || k->dim() != 4 || !fits_int(k->sizes()))
      return false;
    B = q->size(0), Hq = q->size(1), nq = q->size(2), d = q->size(3), Hkv = k->size(1), nk = k->size(2);
    const int64_t want[4] = {B, Hkv, nk, d};
    if (!is(k, want, q->scalar_type(), *q) || !is(v, want, q->scalar_type(), *q) || q->numel() == 0 || k->numel() == 0) return false;
    if (!get_scale(a[0], d, scale) || !PyBool_Check(a[1]) || !get_int(a[2], start) || !get_ints(a[3], {B}, *q, starts) ||
        !get_ints(a[4], {B}, *q, lens) || !get_int(a[7], first))
      return false;
    causal = a[1] == Py_True;
    if (starts) start = 0;
    if (a[5] == Py_None) return a[6] == Py_None;
    bias = plain(a[5]);
    const at::Tensor* r = plain(a[6]);
    if (!bias || bias->dim() != 2 || !fits_int(bias->sizes()) || !is(bias, {bias->size(0), Hq}, q->scalar_type(), *q) || !r ||
        r->dim() != 1 || !fits_int(r->sizes()) || !is(r, r->sizes(), at::kInt, *q))
      return false;
    bias_rows = (const int*)r->data_ptr();
    R = (int)r->size(0), buckets = (int)bias->size(0);
    return true;
  }
  const void* table() const { return bias ? bias->data_ptr() : nullptr; }
};
void put_strides(long long* s, const at::Tensor& t) {
  for (int i = 0; i < 3; ++i) s[i] = t.stride(i);
}

// cross_fwd(q, k, v, scale, causal, start, starts, k_lens, bias, bias_rows, bias_first, out, workspace)
PyObject* cross_fwd(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    Cross c;
    if (na != 13 || !c.get(a, a + 3)) return not_mine();
    at::Tensor own[2], ws_own;
    const at::Tensor* out[2];
    if (a[11] == Py_None) {
      out[0] = &(own[0] = at::empty(c.q->sizes(), c.q->options()));
      out[1] = &(own[1] = at::empty(c.q->sizes().slice(0, 3), c.q->options().dtype(at::kFloat)));
    } else {
      if (!PyTuple_CheckExact(a[11]) || PyTuple_GET_SIZE(a[11]) != 2) return not_mine();
      out[0] = rows(PyTuple_GET_ITEM(a[11], 0)), out[1] = plain(PyTuple_GET_ITEM(a[11], 1));
      if (!like(out[0], *c.q) || !is(out[1], c.q->sizes().slice(0, 3), at::kFloat, *c.q)) return not_mine();
    }
    const size_t need = cross_fwd_ws(c.B, c.Hq, c.Hkv, c.nq, c.nk, c.d, dtype_code(*c.q), c.R);
    void *ws = nullptr, *st;
    size_t bytes = 0;
    if ((need > 0 || a[12] != Py_None) && !get_workspace(a[12], need, *c.q, ws_own, ws, bytes)) return not_mine();
    long long s[12];
    const at::Tensor* all[4] = {c.q, c.k, c.v, out[0]};
    for (int i = 0; i < 4; ++i) put_strides(s + 3 * i, *all[i]);
    const c10::DeviceGuard device(c.q->device());
    if (!get_stream(*c.q, st)) return nullptr;
    const int rc = released([&] {
      return c_cross_fwd(c.q->data_ptr(), c.k->data_ptr(), c.v->data_ptr(), out[0]->data_ptr(), (float*)out[1]->data_ptr(), s, c.lens,
                         c.starts, c.start, c.table(), c.bias_rows, c.first, c.R, c.buckets, ws, bytes, c.B, c.Hq, c.Hkv, c.nq, c.nk,
                         c.d, c.scale, c.causal, dtype_code(*c.q), st);
    });
    if (rc) return PyLong_FromLong(rc);
    if (a[11] != Py_None) return Py_NewRef(a[11]);
    PyObject *x = THPVariable_Wrap(std::move(own[0])), *y = THPVariable_Wrap(std::move(own[1]));
    PyObject* both = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
  });
}

// cross_bwd(q, k, v, o, lse, do, scale, causal, start, starts, k_lens, bias, bias_rows, bias_first, out, workspace)
PyObject* cross_bwd(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    Cross c;
    if (na != 16 || !c.get(a, a + 6)) return not_mine();
    const at::Tensor *o = rows(a[3]), *l = plain(a[4]), *g = rows(a[5]);
    if (!like(o, *c.q) || !is(l, c.q->sizes().slice(0, 3), at::kFloat, *c.q) || !like(g, *c.q)) return not_mine();
    const int N = c.bias ? 4 : 3;
    const at::Tensor* ref[4] = {c.q, c.k, c.v, c.bias};
    at::Tensor own[4], ws_own;
    const at::Tensor* out[4] = {nullptr, nullptr, nullptr, nullptr};
    if (a[14] == Py_None) {
      for (int i = 0; i < N; ++i) out[i] = &(own[i] = at::empty(ref[i]->sizes(), ref[i]->options()));
    } else {
      if (!PyTuple_CheckExact(a[14]) || PyTuple_GET_SIZE(a[14]) != N) return not_mine();
      for (int i = 0; i < N; ++i) {
        PyObject* x = PyTuple_GET_ITEM(a[14], i);
        if (i == 3 && x == Py_None) break;
        out[i] = i < 3 ? rows(x) : plain(x);
        if (!like(out[i], *ref[i])) return not_mine();
      }
    }
    const size_t need = cross_bwd_ws(c.B, c.Hq, c.Hkv, c.nq, c.nk, c.d, dtype_code(*c.q), out[3] ? c.R : 0);
    void *ws = nullptr, *st;
    size_t bytes = 0;
    if ((need > 0 || a[15] != Py_None) && !get_workspace(a[15], need, *c.q, ws_own, ws, bytes)) return not_mine();
    long long s[24];
    const at::Tensor* all[8] = {c.q, c.k, c.v, o, g, out[0], out[1], out[2]};
    for (int i = 0; i < 8; ++i) put_strides(s + 3 * i, *all[i]);
    const c10::DeviceGuard device(c.q->device());
    if (!get_stream(*c.q, st)) return nullptr;
    const int rc = released([&] {
      return c_cross_bwd(c.q->data_ptr(), c.k->data_ptr(), c.v->data_ptr(), o->data_ptr(), (const float*)l->data_ptr(), g->data_ptr(),
                         out[0]->data_ptr(), out[1]->data_ptr(), out[2]->data_ptr(), out[3] ? out[3]->data_ptr() : nullptr, s, c.lens,
                         c.starts, c.start, c.table(), c.bias_rows, c.first, c.R, c.buckets, ws, bytes, c.B, c.Hq, c.Hkv, c.nq, c.nk,
                         c.d, c.scale, c.causal, dtype_code(*c.q), st);
    });
    if (rc) return PyLong_FromLong(rc);
    if (a[14] != Py_None) return Py_NewRef(a[14]);
    PyObject* r = PyTuple_New(N);
    if (!r) return nullptr;
    for (int i = 0; i < N; ++i) {
      PyObject* x = THPVariable_Wrap(std::move(own[i]));
      if (!x) {
        Py_DECREF(r);
        return nullptr;
      }
      PyTuple_SET_ITEM(r, i, x);
    }
    return r;
  });
}

// prefix_decode(q, k_prefix, v_prefix, k_cache, v_cache, k_new, v_new, cache_lens, n, scale, out, workspace)
PyObject* prefix_decode(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded([&]() -> PyObject* {
    if (na != 12) return not_mine();
    const at::Tensor *q = plain(a[0]), *kp = plain(a[1]), *vp = plain(a[2]), *kc = plain(a[3]), *vc = plain(a[4]), *kn = nullptr, *vn = nullptr;
    if (!q || q->dim() != 3 || q->scalar_type() != at::kBFloat16 || !kp || kp->dim() != 3 || !kc || kc->dim() != 4 ||
        !fits_int(q->sizes()) || !fits_int(kp->sizes()) || !fits_int(kc->sizes()))
      return not_mine();
    const int64_t B = q->size(0), Hq = q->size(1), d = q->size(2), Hkv = kp->size(0), np = kp->size(1), n_cap = kc->size(2);
    const int64_t want_p[3] = {Hkv, np, d}, want_c[4] = {B, Hkv, n_cap, d}, want_new[3] = {B, Hkv, d};
    if (!is(kp, want_p, at::kBFloat16, *q) || !is(vp, want_p, at::kBFloat16, *q) || !is(kc, want_c, at::kBFloat16, *q) ||
        !is(vc, want_c, at::kBFloat16, *q) || (a[5] == Py_None) != (a[6] == Py_None))
      return not_mine();
    if (a[5] != Py_None) {
      kn = plain(a[5]), vn = plain(a[6]);
      if (!is(kn, want_new, at::kBFloat16, *q) || !is(vn, want_new, at::kBFloat16, *q)) return not_mine();
    }
    const int* lens;
    int n;
    float scale;
    if (!get_ints(a[7], {B}, *q, lens) || !get_scale(a[9], d, scale)) return not_mine();
    if (a[8] != Py_None) {
      if (!get_int(a[8], n)) return not_mine();
    } else {
      if (!lens) return not_mine();
      n = (int)n_cap - (kn != nullptr);
    }
    Outputs<2> out;
    if (!out.get(a[10], *q, 1)) return not_mine();
    const size_t need = prefix_ws(B, Hq, Hkv, np, n, d);
    at::Tensor own;
    void *ws, *st;
    size_t bytes;
    if (!get_workspace(a[11], need, *q, own, ws, bytes)) return not_mine();
    const c10::DeviceGuard device(q->device());
    if (!get_stream(*q, st)) return nullptr;
    const int rc = released([&] {
      return c_prefix(q->data_ptr(), kn ? kn->data_ptr() : nullptr, kn ? vn->data_ptr() : nullptr, kp->data_ptr(), vp->data_ptr(),
                      kc->data_ptr(), vc->data_ptr(), lens, out.p[0], (float*)out.p[1], ws, bytes, B, Hq, Hkv, np, n, n_cap, d, scale, 0,
                      st);
    });
    return rc ? PyLong_FromLong(rc) : out.answer(a[10]);
  });
}

// bind_cross(cross_fwd_workspace_bytes, cross_fwd, cross_bwd_workspace_bytes, cross_bwd, prefix_decode_workspace_bytes,
//            prefix_decode [addresses])
PyObject* bind_cross(PyObject*, PyObject* const* a, Py_ssize_t na) {
  if (na != 6) {
    PyErr_SetString(PyExc_TypeError, "bind_cross takes six addresses");
    return nullptr;
  }
  void* p[6];
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind_cross: null address");
      return nullptr;
    }
  }
  cross_fwd_ws = (CrossWsFn)p[0];
  c_cross_fwd = (CrossFwdFn)p[1];
  cross_bwd_ws = (CrossWsFn)p[2];
  c_cross_bwd = (CrossBwdFn)p[3];
  prefix_ws = (PrefixWsFn)p[4];
  c_prefix = (PrefixFn)p[5];
  Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL
PyMethodDef methods[] = {{"bind", FAST(bind), nullptr},       {"fwd", FAST(fwd), nullptr}, {"fwd_bwd", FAST(fwd_bwd), nullptr},
                         {"bwd", FAST(bwd), nullptr},         {"decode", FAST(decode), nullptr},
                         {"bind_paged", FAST(bind_paged), nullptr}, {"rope", FAST(rope), nullptr},
                         {"paged_append", FAST(paged_append), nullptr}, {"paged_gather", FAST(paged_gather), nullptr},
                         {"paged_decode", FAST(paged_decode), nullptr},
                         {"bind_cross", FAST(bind_cross), nullptr},     {"cross_fwd", FAST(cross_fwd), nullptr},
                         {"cross_bwd", FAST(cross_bwd), nullptr},       {"prefix_decode", FAST(prefix_decode), nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
