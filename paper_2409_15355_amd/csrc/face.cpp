// The Python face's native half: takes a call's arguments apart (torch tensors, NumPy arrays, ba_heads) and makes
// the call.  Each function takes exactly what the Python function of its name takes and returns the call's status,
// or None where an argument is anything but the plain case (a tensor subclass, a list for an array, a shape that
// does not fit the call): nothing has been launched then, and the Python function goes through its own checks,
// which convert what can be converted and say what is wrong with the rest.
//
// A call of a few microseconds on the device spent more on this in Python: 5 us of 12 for per-block encoding, 6 of 15
// for a final block, 19 of 39 for encoding, re-encoding and final block of one prompt.
//
// It sees inside torch's tensors, so it serves the torch it was built with and no other: torch_version.
#define NPY_NO_DEPRECATED_API NPY_1_7_API_VERSION
#include <Python.h>

#include <numpy/arrayobject.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cxxabi.h>

#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/ba.h"

namespace {

// The library's entry points (loaded by the Python face, which hands over their addresses).
struct {
  decltype(&ba_encode_blocks) encode;
  decltype(&ba_reencode_positions) reencode;
  decltype(&ba_final_block_attention) final_block;
  decltype(&ba_final_block_attention_static) final_static;
  decltype(&ba_final_block_attention_cached) final_cached;
  decltype(&ba_block_attention_prompts) prompts;
  decltype(&ba_block_attention_prompts_backward) prompts_backward;
} lib;
struct {
  decltype(&ba_norm_rotate) norm_rotate;
  decltype(&ba_norm_rotate_backward) norm_rotate_backward;
  decltype(&ba_paged_append) paged_append;
  decltype(&ba_paged_attention) paged_attention;
} paged;
struct {
  decltype(&ba_paged_key_weights) key_weights;
  decltype(&ba_paged_evict) evict;
  decltype(&ba_page_bounds) page_bounds;
  decltype(&ba_page_select) page_select;
  decltype(&ba_paged_attention_selected) attention_selected;
} longer;
PyTypeObject *heads_type, *norm_type, *cache_type, *bounds_type;
PyObject *name_c, *name_known, *name_cuda_stream, *get_device, *get_raw_stream;

// Arguments that are not the plain case.
struct Declined {};
void need(bool ok) {
  if (!ok) throw Declined();
}

// The structure that an object of a known type keeps in an attribute, held for the call.
template <typename T>
struct Held {
  Py_buffer view{};
  const T *h = nullptr;
  Held(PyObject *o, PyTypeObject *type, PyObject *attribute) {
    need(Py_TYPE(o) == type);
    PyObject *c = PyObject_GetAttr(o, attribute);
    need(c != nullptr);
    const int rc = PyObject_GetBuffer(c, &view, PyBUF_SIMPLE);  // (the view holds a reference of its own)
    Py_DECREF(c);
    need(rc == 0);
    if (view.len != (Py_ssize_t)sizeof(T)) {
      PyBuffer_Release(&view);
      throw Declined();
    }
    h = (const T *)view.buf;
  }
  ~Held() { PyBuffer_Release(&view); }
  Held(const Held &) = delete;
};
// The ba_heads inside a Heads object.
struct HeadsArg : Held<ba_heads> {
  explicit HeadsArg(PyObject *o) : Held(o, heads_type, name_c) {}
};
// What a HeadNorm and a PagedCache know, the sizes that the library's structures do not have among them.
struct KnownNorm {
  ba_head_norm norm;
  int32_t head_dim;  // 0: no gains
};
struct KnownCache {
  ba_paged_cache cache;
  int32_t n_kv_heads, head_dim;
};
struct NormArg : Held<KnownNorm> {
  NormArg(PyObject *o, int64_t d) : Held(o, norm_type, name_known) { need(!h->head_dim || h->head_dim == d); }
};
struct CacheArg : Held<KnownCache> {
  CacheArg(PyObject *o, const ba_heads *heads) : Held(o, cache_type, name_known) { need(h->n_kv_heads == heads->n_kv_heads && h->head_dim == heads->head_dim); }
};

struct KnownBounds {
  ba_page_bound_table bounds;
  int32_t n_pages, n_kv_heads, head_dim;
};
struct BoundsArg : Held<KnownBounds> {
  BoundsArg(PyObject *o, const ba_heads *heads, const ba_paged_cache &cache) : Held(o, bounds_type, name_known) {
    need(h->n_kv_heads == heads->n_kv_heads && h->head_dim == heads->head_dim && h->n_pages >= cache.n_pages);
  }
};

bool is_int32_array(PyObject *o) {
  if (!PyArray_CheckExact(o)) return false;
  PyArrayObject *a = (PyArrayObject *)o;
  return PyArray_TYPE(a) == NPY_INT32 && PyArray_NDIM(a) == 1 && PyArray_ISCARRAY_RO(a);
}
// int32 host array (as guarded has seen) or None, copied: the call runs without the interpreter's lock.
struct Ints {
  int32_t few[96];
  std::vector<int32_t> many;
  const int32_t *p = nullptr;
  int64_t n = 0;
  explicit Ints(PyObject *o) {
    if (o == Py_None) return;
    PyArrayObject *a = (PyArrayObject *)o;
    n = PyArray_DIM(a, 0);
    const int32_t *from = (const int32_t *)PyArray_DATA(a);
    int32_t *to = few;
    if (n > (int64_t)(sizeof(few) / 4)) {
      many.resize((size_t)n);
      to = many.data();
    }
    if (n) memcpy(to, from, (size_t)n * 4);
    p = to;
  }
  Ints(const Ints &) = delete;
  int64_t last() const { return n ? p[n - 1] : 0; }
};
void same_len(int64_t n, const Ints &a) { need(!a.p || a.n == n); }
// rows that blocks [off, off + len) reach (empty blocks touch nothing)
int64_t reach(const Ints &off, const Ints &len) {
  if (!off.p || !len.p || !len.n) return 0;
  need(off.n == len.n);
  int64_t most = 0;
  bool any = false;
  for (int64_t i = 0; i < len.n; ++i)
    if (len.p[i] > 0) {
      const int64_t end = (int64_t)off.p[i] + len.p[i];
      most = any ? std::max(most, end) : end;
      any = true;
    }
  return most;
}

const at::Tensor &plain_tensor(PyObject *o) {
  need(THPVariable_CheckExact(o));
  const at::Tensor &t = THPVariable_Unpack(o);
  need(t.defined() && t.is_cuda() && t.layout() == at::kStrided);
  return t;
}
// [tokens, heads, D] on the GPU, D contiguous, with the call's heads and at least the rows it reaches; with `layers`
// the first layer of a [layers, tokens, heads, D] one.
struct TensorArg {
  ba_tensor t{};
  const ba_tensor *p = nullptr;
  TensorArg(PyObject *o, int64_t heads, int64_t d, int64_t min_tokens, bool allow_f32 = false, bool layers = false) {
    if (o == Py_None) return;
    const at::Tensor &x = plain_tensor(o);
    const auto type = x.scalar_type();
    need(type == at::kBFloat16 || (allow_f32 && type == at::kFloat));
    const auto size = x.sizes(), stride = x.strides();
    const size_t at = layers ? 1 : 0;
    need(size.size() == at + 3);
    need(size[at + 2] <= 1 || stride[at + 2] == 1);
    need(size[at + 1] == heads && size[at + 2] == d && size[at] >= min_tokens);
    t.ptr = x.data_ptr();
    t.stride_tok = stride[at];
    t.stride_head = stride[at + 1];
    t.dtype = type == at::kFloat ? BA_DTYPE_F32 : BA_DTYPE_BF16;
    p = &t;
  }
  TensorArg(const TensorArg &) = delete;
};
float *lse_of(PyObject *o, int64_t tokens, int64_t n_q_heads) {
  if (o == Py_None) return nullptr;
  const at::Tensor &x = plain_tensor(o);
  need(x.scalar_type() == at::kFloat && x.dim() == 2 && x.is_contiguous() && x.size(1) == n_q_heads && x.size(0) >= tokens);
  return (float *)x.data_ptr();
}
// at least n integers, or floats, in GPU memory
template <typename T>
T *device_array(PyObject *o, at::ScalarType type, int64_t n) {
  if (o == Py_None) return nullptr;
  const at::Tensor &x = plain_tensor(o);
  need(x.scalar_type() == type && x.dim() == 1 && x.is_contiguous() && x.size(0) >= n);
  return (T *)x.data_ptr();
}
// float32 [sequences, KV heads, at least `least`], sequences n_kv_heads heads apart
struct PerKey {
  float *p = nullptr;
  int64_t stride = 0;
  PerKey(PyObject *o, int64_t heads, int64_t seqs, int64_t least) {
    if (o == Py_None) return;
    const at::Tensor &x = plain_tensor(o);
    need(x.scalar_type() == at::kFloat && x.dim() == 3);
    const auto size = x.sizes(), st = x.strides();
    need((size[2] <= 1 || st[2] == 1) && size[1] == heads && size[0] >= seqs && size[2] >= least);
    stride = heads > 1 ? st[1] : size[0] > 1 ? st[0] : std::max<int64_t>(size[2], 1);
    need(size[0] <= 1 || st[0] == heads * stride);
    p = (float *)x.data_ptr();
  }
};
// [sequences, KV heads, n]; width: n, or -1 for any
template <typename T>
T *device_lists(PyObject *o, at::ScalarType type, int64_t seqs, int64_t heads, int64_t width, int32_t *n = nullptr) {
  if (o == Py_None) return nullptr;
  const at::Tensor &x = plain_tensor(o);
  need(x.scalar_type() == type && x.dim() == 3 && x.is_contiguous() && x.size(0) >= seqs && x.size(1) == heads && (width < 0 || x.size(2) == width) &&
       x.size(2) <= INT32_MAX);
  if (n) *n = (int32_t)x.size(2);
  return (T *)x.data_ptr();
}
float *gain_grad(PyObject *o, int64_t d) {
  need(o == Py_None || plain_tensor(o).numel() == d);
  return device_array<float>(o, at::kFloat, d);
}
int64_t tokens_of(PyObject *q, PyObject *k) {
  need(q != Py_None || k != Py_None);
  const at::Tensor &x = plain_tensor(q != Py_None ? q : k);
  need(x.dim() == 3 && x.size(0) <= INT32_MAX);
  if (q != Py_None && k != Py_None) {
    const at::Tensor &y = plain_tensor(k);
    need(y.dim() == 3 && y.size(0) == x.size(0));
  }
  return x.size(0);
}
struct Workspace {
  void *p = nullptr;
  size_t bytes = 0;
  explicit Workspace(PyObject *o) {
    if (o == Py_None) return;
    const at::Tensor &x = plain_tensor(o);
    need(x.is_contiguous());
    p = x.data_ptr();
    bytes = (size_t)x.numel() * x.element_size();
  }
};
int32_t int_of(PyObject *o) {
  need(PyLong_CheckExact(o));
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  need(!overflow && v == (int32_t)v);
  return (int32_t)v;
}
float float_of(PyObject *o) {
  need(PyFloat_CheckExact(o));
  return (float)PyFloat_AS_DOUBLE(o);
}
void *stream_of(PyObject *o) {
  PyObject *h = nullptr;
  if (o != Py_None) {
    h = PyObject_GetAttr(o, name_cuda_stream);
  } else {
    need(get_raw_stream != nullptr);
    PyObject *dev = PyObject_CallNoArgs(get_device);
    need(dev != nullptr);
    h = PyObject_CallOneArg(get_raw_stream, dev);
    Py_DECREF(dev);
  }
  need(h != nullptr);
  void *s = PyLong_Check(h) ? PyLong_AsVoidPtr(h) : nullptr;
  const bool ok = PyLong_Check(h) && !PyErr_Occurred();
  Py_DECREF(h);
  need(ok);
  return s;
}

// An exception out of the library: its call may have launched something, so it is an error and never "not the plain case".
struct Threw {
  bool memory;
};
// body() makes the call and returns its status.  Arguments 1 .. tensors are tensors or None, those from there to `arrays`
// int32 arrays or None: looked at first, without an exception, which costs 3.5 us (lists and 64-bit arrays are ordinary arguments).
template <typename Body>
PyObject *guarded(PyObject *const *a, Py_ssize_t n, Py_ssize_t want, int tensors, int arrays, Body &&body) {
  if (n != want) Py_RETURN_NONE;
  for (int i = 1; i <= arrays; ++i)
    if (a[i] != Py_None && !(i <= tensors ? THPVariable_CheckExact(a[i]) : is_int32_array(a[i]))) Py_RETURN_NONE;
  try {
    return PyLong_FromLong(body());
  } catch (const Threw &t) {
    PyErr_SetString(t.memory ? PyExc_MemoryError : PyExc_RuntimeError, "an exception inside the library");
    return nullptr;
  } catch (abi::__forced_unwind &) {  // (a thread that ends with the interpreter, waiting for its lock)
    throw;
  } catch (...) {
    PyErr_Clear();  // (the Python function meets the same argument again and raises what there is to raise)
  }
  Py_RETURN_NONE;
}
template <typename Call>
int32_t unlocked(Call &&call) {
  int32_t rc = 0;
  int threw = 0;
  PyThreadState *const state = PyEval_SaveThread();
  try {
    rc = call();
  } catch (const std::bad_alloc &) {
    threw = 2;
  } catch (...) {
    threw = 1;
  }
  PyEval_RestoreThread(state);
  if (threw) throw Threw{threw == 2};
  return rc;
}

PyObject *encode_blocks(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 10, 5, 6, [&] {
    const HeadsArg h(a[0]);
    const Ints offs(a[6]);
    need(offs.p && offs.n > 0);
    const int64_t T = offs.last(), hq = h.h->n_q_heads, hkv = h.h->n_kv_heads, d = h.h->head_dim;
    const TensorArg q(a[1], hq, d, T), k(a[2], hkv, d, T), v(a[3], hkv, d, T), o(a[4], hq, d, T), kl(a[5], hkv, d, T);
    const int32_t mode = int_of(a[7]);
    const Workspace ws(a[8]);
    void *const stream = stream_of(a[9]);
    return unlocked([&] {
      return lib.encode(h.h, q.p, k.p, v.p, o.p, kl.p, (int32_t)(offs.n - 1), offs.p, mode, ws.p, ws.bytes, stream);
    });
  });
}

PyObject *reencode_positions(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 10, 2, 7, [&] {
    const HeadsArg h(a[0]);
    const at::Tensor &s = plain_tensor(a[1]), &t = plain_tensor(a[2]);
    const bool layers = s.dim() == 4;
    need(s.dim() == t.dim() && (layers ? s.size(0) == t.size(0) && s.size(0) > 0 : s.dim() == 3));
    const Ints so(a[3]), to(a[4]), ln(a[5]), op(a[6]), np(a[7]);
    need(so.p && to.p && ln.p);
    for (const Ints *x : {&so, &to, &op, &np}) same_len(ln.n, *x);
    const int64_t hkv = h.h->n_kv_heads, d = h.h->head_dim;
    const TensorArg src(a[1], hkv, d, reach(so, ln), true, layers), dst(a[2], hkv, d, reach(to, ln), true, layers);
    // (one layer: the stride that a view with a leading dimension of one has)
    const int64_t n_layers = layers ? s.size(0) : 1;
    need(n_layers <= INT32_MAX && ln.n <= INT32_MAX);
    const int64_t sl = layers ? s.stride(0) : s.size(0) * s.stride(0), tl = layers ? t.stride(0) : t.size(0) * t.stride(0);
    const int32_t mode = int_of(a[8]);
    void *const stream = stream_of(a[9]);
    return unlocked([&] {
      return lib.reencode(h.h, src.p, dst.p, (int32_t)n_layers, sl, tl, (int32_t)ln.n, so.p, to.p, ln.p, op.p, np.p, mode, stream);
    });
  });
}

// ba_final_block_attention and, without a workspace, ba_final_block_attention_static
template <bool kStatic>
PyObject *final_block(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, kStatic ? 13 : 14, 7, 10, [&] {
    const HeadsArg h(a[0]);
    const Ints cq(a[8]), cc(a[9]), qp(a[10]);
    need(cq.p && cc.p && cq.n > 0 && cq.n == cc.n);
    same_len(cq.n - 1, qp);
    const int64_t hq = h.h->n_q_heads, hkv = h.h->n_kv_heads, d = h.h->head_dim, tq = cq.last(), tc = cc.last();
    const TensorArg q(a[1], hq, d, tq), kc(a[2], hkv, d, tc), vc(a[3], hkv, d, tc), kf(a[4], hkv, d, tq), vf(a[5], hkv, d, tq),
        o(a[6], hq, d, tq), kr(a[7], hkv, d, tq);
    const int32_t mode = int_of(a[11]);
    const Workspace ws(kStatic ? Py_None : a[12]);
    void *const stream = stream_of(a[kStatic ? 12 : 13]);
    return unlocked([&] {
      const int32_t np = (int32_t)(cq.n - 1);
      return kStatic ? lib.final_static(h.h, q.p, kc.p, vc.p, kf.p, vf.p, o.p, kr.p, np, cq.p, cc.p, qp.p, mode, stream)
                     : lib.final_block(h.h, q.p, kc.p, vc.p, kf.p, vf.p, o.p, kr.p, np, cq.p, cc.p, qp.p, mode, ws.p, ws.bytes, stream);
    });
  });
}

PyObject *final_block_cached(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 18, 7, 14, [&] {
    const HeadsArg h(a[0]);
    const Ints cq(a[8]), cb(a[9]), bo(a[10]), bl(a[11]), op(a[12]), np(a[13]), qp(a[14]);
    need(cq.p && cb.p && bo.p && bl.p && cq.n > 0 && cq.n == cb.n);
    for (const Ints *x : {&bo, &bl, &op, &np}) same_len(cb.last(), *x);
    same_len(cq.n - 1, qp);
    const int64_t hq = h.h->n_q_heads, hkv = h.h->n_kv_heads, d = h.h->head_dim, tq = cq.last(), tc = reach(bo, bl);
    const TensorArg q(a[1], hq, d, tq), kc(a[2], hkv, d, tc), vc(a[3], hkv, d, tc), kf(a[4], hkv, d, tq), vf(a[5], hkv, d, tq),
        o(a[6], hq, d, tq), kr(a[7], hkv, d, tq);
    const Workspace ws(a[15]);
    void *const stream = stream_of(a[16]);
    const int32_t below = int_of(a[17]);
    return unlocked([&] {
      return lib.final_cached(h.h, q.p, kc.p, vc.p, kf.p, vf.p, o.p, kr.p, (int32_t)(cq.n - 1), cq.p, cb.p, bo.p, bl.p, op.p, np.p, qp.p,
                              below, ws.p, ws.bytes, stream);
    });
  });
}

PyObject *prompts(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 12, 6, 8, [&] {
    const HeadsArg h(a[0]);
    const Ints cb(a[7]), offs(a[8]);
    need(cb.p && offs.p && cb.n > 0 && offs.n > 0 && cb.last() == offs.n - 1);
    const int64_t T = offs.last(), hq = h.h->n_q_heads, hkv = h.h->n_kv_heads, d = h.h->head_dim;
    const TensorArg q(a[1], hq, d, T), k(a[2], hkv, d, T), v(a[3], hkv, d, T), o(a[4], hq, d, T), kr(a[5], hkv, d, T);
    float *const lse = lse_of(a[6], T, hq);
    const int32_t mode = int_of(a[9]);
    const Workspace ws(a[10]);
    void *const stream = stream_of(a[11]);
    return unlocked([&] {
      return lib.prompts(h.h, q.p, k.p, v.p, o.p, kr.p, lse, (int32_t)(cb.n - 1), cb.p, offs.p, mode, ws.p, ws.bytes, stream);
    });
  });
}

PyObject *prompts_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 14, 9, 11, [&] {
    const HeadsArg h(a[0]);
    const Ints cb(a[10]), offs(a[11]);
    need(cb.p && offs.p && cb.n > 0 && offs.n > 0 && cb.last() == offs.n - 1 && a[5] != Py_None);
    const int64_t T = offs.last(), hq = h.h->n_q_heads, hkv = h.h->n_kv_heads, d = h.h->head_dim;
    const TensorArg q(a[1], hq, d, T), k(a[2], hkv, d, T), v(a[3], hkv, d, T), o(a[4], hq, d, T), g(a[6], hq, d, T), dq(a[7], hq, d, T),
        dk(a[8], hkv, d, T), dv(a[9], hkv, d, T);
    const float *const lse = lse_of(a[5], T, hq);
    const Workspace ws(a[12]);
    void *const stream = stream_of(a[13]);
    return unlocked([&] {
      return lib.prompts_backward(h.h, q.p, k.p, v.p, o.p, lse, g.p, dq.p, dk.p, dv.p, (int32_t)(cb.n - 1), cb.p, offs.p, ws.p, ws.bytes, stream);
    });
  });
}

// (arguments in another order than the Python functions': tensors, integer arrays, the rest)
PyObject *norm_rotate(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 9, 5, 5, [&] {
    const HeadsArg h(a[0]);
    const int64_t T = tokens_of(a[1], a[2]), hq = h.h->n_q_heads, hkv = h.h->n_kv_heads, d = h.h->head_dim;
    const TensorArg q(a[1], hq, d, T, true), k(a[2], hkv, d, T, true), qo(a[3], hq, d, T, true), ko(a[4], hkv, d, T, true);
    const int32_t *const at = device_array<int32_t>(a[5], at::kInt, T);
    const NormArg norm(a[6], d);
    const int32_t mode = int_of(a[7]);
    void *const stream = stream_of(a[8]);
    return unlocked([&] { return paged.norm_rotate(h.h, &norm.h->norm, q.p, k.p, qo.p, ko.p, (int32_t)T, at, mode, stream); });
  });
}

PyObject *norm_rotate_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 14, 9, 9, [&] {
    const HeadsArg h(a[0]);
    const int64_t T = tokens_of(a[1], a[2]), hq = h.h->n_q_heads, hkv = h.h->n_kv_heads, d = h.h->head_dim;
    const TensorArg q(a[1], hq, d, T, true), k(a[2], hkv, d, T, true), gq(a[3], hq, d, T, true), gk(a[4], hkv, d, T, true),
        dq(a[5], hq, d, T, true), dk(a[6], hkv, d, T, true);
    float *const dwq = gain_grad(a[7], d), *const dwk = gain_grad(a[8], d);
    const int32_t *const at = device_array<int32_t>(a[9], at::kInt, T);
    const NormArg norm(a[10], d);
    const int32_t mode = int_of(a[11]);
    const Workspace ws(a[12]);
    void *const stream = stream_of(a[13]);
    return unlocked([&] {
      return paged.norm_rotate_backward(h.h, &norm.h->norm, q.p, k.p, gq.p, gk.p, dq.p, dk.p, dwq, dwk, (int32_t)T, at, mode, ws.p, ws.bytes, stream);
    });
  });
}

PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 12, 7, 7, [&] {
    const HeadsArg h(a[0]);
    const int64_t T = tokens_of(a[2], a[2]), hq = h.h->n_q_heads, hkv = h.h->n_kv_heads, d = h.h->head_dim;
    const TensorArg q(a[1], hq, d, T), k(a[2], hkv, d, T), v(a[3], hkv, d, T), qo(a[4], hq, d, T);
    const int32_t *const at = device_array<int32_t>(a[5], at::kInt, T), *const seq = device_array<int32_t>(a[6], at::kInt, T),
                         *const pos = device_array<int32_t>(a[7], at::kInt, T);
    const CacheArg cache(a[9], h.h);
    const int32_t mode = int_of(a[10]);
    void *const stream = stream_of(a[11]);
    auto call = [&](const ba_head_norm *norm) {
      return unlocked([&] { return paged.paged_append(h.h, norm, &cache.h->cache, q.p, k.p, v.p, qo.p, (int32_t)T, at, seq, pos, mode, stream); });
    };
    if (a[8] == Py_None) return call(nullptr);
    const NormArg norm(a[8], d);
    return call(&norm.h->norm);
  });
}

PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 12, 4, 6, [&] {
    const HeadsArg h(a[0]);
    const CacheArg cache(a[7], h.h);
    const Ints cu(a[5]), prefix(a[6]);
    need(!cu.p == !prefix.p && (!cu.p || cu.n == prefix.n + 1));
    const int32_t max_len = int_of(a[8]), nq = int_of(a[9]);
    const int64_t seqs = cache.h->cache.n_seqs, T = seqs * std::max(nq, 0), hq = h.h->n_q_heads, d = h.h->head_dim;
    const TensorArg q(a[1], hq, d, T), o(a[2], hq, d, T);
    float *const lse = lse_of(a[3], T, hq);
    const int32_t *const len = device_array<int32_t>(a[4], at::kInt, seqs);
    const Workspace ws(a[10]);
    void *const stream = stream_of(a[11]);
    return unlocked([&] {
      return paged.paged_attention(h.h, &cache.h->cache, q.p, o.p, lse, nq, len, max_len, (int32_t)prefix.n, cu.p, prefix.p, ws.p, ws.bytes, stream);
    });
  });
}

PyObject *key_weights(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 14, 5, 7, [&] {
    const HeadsArg h(a[0]);
    const CacheArg cache(a[8], h.h);
    const Ints cu(a[6]), prefix(a[7]);
    need(!cu.p == !prefix.p && (!cu.p || cu.n == prefix.n + 1));
    const float decay = float_of(a[9]);
    const int32_t max_len = int_of(a[10]), nq = int_of(a[11]);
    const int64_t seqs = cache.h->cache.n_seqs, T = seqs * std::max(nq, 0), hq = h.h->n_q_heads, hkv = h.h->n_kv_heads;
    const TensorArg q(a[1], hq, h.h->head_dim, T);
    const float *const lse = lse_of(a[2], T, hq);
    const PerKey in(a[3], hkv, seqs, max_len), out(a[4], hkv, seqs, max_len);
    need(!in.p || !out.p || in.stride == out.stride);
    const int32_t *const len = device_array<int32_t>(a[5], at::kInt, seqs);
    const Workspace ws(a[12]);
    void *const stream = stream_of(a[13]);
    return unlocked([&] {
      return longer.key_weights(h.h, &cache.h->cache, q.p, lse, in.p, out.p, out.stride, decay, nq, len, max_len, (int32_t)prefix.n, cu.p, prefix.p, ws.p,
                                ws.bytes, stream);
    });
  });
}

PyObject *evict(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 14, 5, 5, [&] {
    const HeadsArg h(a[0]);
    const CacheArg cache(a[6], h.h), to(a[7], h.h);
    const int32_t max_len = int_of(a[8]), n_keep = int_of(a[9]), n_first = int_of(a[10]), n_last = int_of(a[11]);
    const int64_t seqs = cache.h->cache.n_seqs, hkv = h.h->n_kv_heads;
    const PerKey w(a[1], hkv, seqs, max_len), out(a[4], hkv, seqs, n_keep);
    const int32_t *const len = device_array<int32_t>(a[2], at::kInt, seqs);
    int32_t *const kept = device_lists<int32_t>(a[3], at::kInt, seqs, hkv, n_keep), *const new_len = device_array<int32_t>(a[5], at::kInt, seqs);
    const Workspace ws(a[12]);
    void *const stream = stream_of(a[13]);
    return unlocked([&] {
      return longer.evict(h.h, &cache.h->cache, &to.h->cache, w.p, w.stride, len, max_len, n_keep, n_first, n_last, kept, out.p, out.stride, new_len, ws.p,
                          ws.bytes, stream);
    });
  });
}

PyObject *page_bounds(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 7, 2, 2, [&] {
    const HeadsArg h(a[0]);
    const CacheArg cache(a[3], h.h);
    const BoundsArg bounds(a[4], h.h, cache.h->cache);
    const int64_t seqs = cache.h->cache.n_seqs;
    const int32_t *const from = device_array<int32_t>(a[1], at::kInt, seqs), *const len = device_array<int32_t>(a[2], at::kInt, seqs);
    const int32_t max_len = int_of(a[5]);
    void *const stream = stream_of(a[6]);
    return unlocked([&] { return longer.page_bounds(h.h, &cache.h->cache, &bounds.h->bounds, from, len, max_len, stream); });
  });
}

PyObject *page_select(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 13, 4, 4, [&] {
    const HeadsArg h(a[0]);
    const CacheArg cache(a[5], h.h);
    const BoundsArg bounds(a[6], h.h, cache.h->cache);
    const int32_t max_len = int_of(a[7]), n_first = int_of(a[8]), n_last = int_of(a[9]), nq = int_of(a[10]);
    const int64_t seqs = cache.h->cache.n_seqs, hkv = h.h->n_kv_heads;
    const TensorArg q(a[1], h.h->n_q_heads, h.h->head_dim, seqs * std::max(nq, 0));
    const int32_t *const len = device_array<int32_t>(a[2], at::kInt, seqs);
    int32_t n_select = 0;
    int32_t *const selected = device_lists<int32_t>(a[3], at::kInt, seqs, hkv, -1, &n_select);
    float *const scores = device_lists<float>(a[4], at::kFloat, seqs, hkv, n_select);
    const Workspace ws(a[11]);
    void *const stream = stream_of(a[12]);
    return unlocked([&] {
      return longer.page_select(h.h, &cache.h->cache, &bounds.h->bounds, q.p, nq, len, max_len, n_select, n_first, n_last, selected, scores, ws.p, ws.bytes,
                                stream);
    });
  });
}

PyObject *paged_attention_selected(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 11, 5, 5, [&] {
    const HeadsArg h(a[0]);
    const CacheArg cache(a[6], h.h);
    const int32_t max_len = int_of(a[7]), nq = int_of(a[8]);
    const int64_t seqs = cache.h->cache.n_seqs, T = seqs * std::max(nq, 0), hq = h.h->n_q_heads, d = h.h->head_dim;
    const TensorArg q(a[1], hq, d, T), o(a[2], hq, d, T);
    float *const lse = lse_of(a[3], T, hq);
    const int32_t *const len = device_array<int32_t>(a[4], at::kInt, seqs);
    int32_t n_select = 0;
    const int32_t *const selected = device_lists<int32_t>(a[5], at::kInt, seqs, h.h->n_kv_heads, -1, &n_select);
    const Workspace ws(a[9]);
    void *const stream = stream_of(a[10]);
    return unlocked([&] {
      return longer.attention_selected(h.h, &cache.h->cache, q.p, o.p, lse, nq, len, max_len, selected, n_select, ws.p, ws.bytes, stream);
    });
  });
}

// setup(Heads class, current_device(), raw_stream(device) or None, addresses of the entry points in the order of `lib`)
PyObject *setup(PyObject *, PyObject *args) {
  PyObject *type, *dev, *raw;
  unsigned long long at[7];
  if (!PyArg_ParseTuple(args, "O!OO(KKKKKKK)", &PyType_Type, &type, &dev, &raw, at, at + 1, at + 2, at + 3, at + 4, at + 5, at + 6)) return nullptr;
  Py_INCREF(type), Py_INCREF(dev), Py_INCREF(raw);
  heads_type = (PyTypeObject *)type;
  get_device = dev;
  get_raw_stream = raw == Py_None ? nullptr : raw;
  static_assert(sizeof(lib) == 7 * sizeof(void *), "an address each");
  void *p[7];
  for (int i = 0; i < 7; ++i) p[i] = (void *)(uintptr_t)at[i];
  memcpy(&lib, p, sizeof(lib));
  Py_RETURN_NONE;
}

// setup_paged(HeadNorm class, PagedCache class, addresses of the entry points in the order of `paged`)
PyObject *setup_paged(PyObject *, PyObject *args) {
  PyObject *norm, *cache;
  unsigned long long at[4];
  if (!PyArg_ParseTuple(args, "O!O!(KKKK)", &PyType_Type, &norm, &PyType_Type, &cache, at, at + 1, at + 2, at + 3)) return nullptr;
  Py_INCREF(norm), Py_INCREF(cache);
  norm_type = (PyTypeObject *)norm;
  cache_type = (PyTypeObject *)cache;
  static_assert(sizeof(paged) == 4 * sizeof(void *), "an address each");
  void *p[4];
  for (int i = 0; i < 4; ++i) p[i] = (void *)(uintptr_t)at[i];
  memcpy(&paged, p, sizeof(paged));
  Py_RETURN_NONE;
}

// setup_long(PageBounds class, addresses of the entry points in the order of `longer`)
PyObject *setup_long(PyObject *, PyObject *args) {
  PyObject *bounds;
  unsigned long long at[5];
  if (!PyArg_ParseTuple(args, "O!(KKKKK)", &PyType_Type, &bounds, at, at + 1, at + 2, at + 3, at + 4)) return nullptr;
  Py_INCREF(bounds);
  bounds_type = (PyTypeObject *)bounds;
  static_assert(sizeof(longer) == 5 * sizeof(void *), "an address each");
  void *p[5];
  for (int i = 0; i < 5; ++i) p[i] = (void *)(uintptr_t)at[i];
  memcpy(&longer, p, sizeof(longer));
  Py_RETURN_NONE;
}

#define FAST(name, fn) {name, (PyCFunction)(void (*)(void))(fn), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, nullptr},
                         {"setup_paged", setup_paged, METH_VARARGS, nullptr},
                         FAST("encode_blocks", encode_blocks),
                         FAST("reencode_positions", reencode_positions),
                         FAST("final_block", final_block<false>),
                         FAST("final_block_static", final_block<true>),
                         FAST("final_block_cached", final_block_cached),
                         FAST("prompts", prompts),
                         FAST("prompts_backward", prompts_backward),
                         FAST("norm_rotate", norm_rotate),
                         FAST("norm_rotate_backward", norm_rotate_backward),
                         FAST("paged_append", paged_append),
                         FAST("paged_attention", paged_attention),
                         {"setup_long", setup_long, METH_VARARGS, nullptr},
                         FAST("key_weights", key_weights),
                         FAST("evict", evict),
                         FAST("page_bounds", page_bounds),
                         FAST("page_select", page_select),
                         FAST("paged_attention_selected", paged_attention_selected),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_face", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__face() {
  import_array();
  name_c = PyUnicode_InternFromString("c");
  name_known = PyUnicode_InternFromString("known");
  name_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  if (!name_c || !name_known || !name_cuda_stream) return nullptr;
  PyObject *m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}
