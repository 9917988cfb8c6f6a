// Host side of an appended token in native code.  A decode loop calls this once per token, and the kernel behind it runs 2 us, so
// what the call costs on the host is what the loop waits for: with the checks, the parameter block and the call through ctypes in
// Python 7.5 us an append (one sequence of 32 layers, DecodeCache.append), now 3.7, 2.6 of them the launch; 128 appends and the
// compression behind them 1200 us, now 710, and over tokens and a cache that were never used before 1370, now 850.
// Directly behind a burst of other launches and a synchronization (a thousand small kernels are enough) both take longer, 1540 and
// 1270: for the next millisecond a thread of the runtime retires what was launched before, and a launch of any kind costs twice as
// much beside it.
//
// rkv_cache_append_rotary, rkv_attend and rkv_attend_shared, called once per layer and decode step, go the same way (append_rotary() and
// attend(), with paged caches too): one token of one sequence 15.9 us a call through ctypes and 5.1 now, its attention 19.2 and 9.7.
//
// append() takes a call whose arguments are all in order and enqueues it; anything else (another type, a subclass of the shape or of a
// tensor, another layout or device, a paged cache, a value out of an int's range) it does not touch
// and answers None, and the Python binding goes through its own checks.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>

#include <ATen/ops/empty.h>

#include "rkv_attend.h"

namespace {

using AppendFn = rkv_status (*)(const rkv_params*, void*, void*, void*, const void*, const void*, const void*, int32_t, int32_t, void*);
AppendFn append_fn = nullptr;
PyObject* shape_type = nullptr;    // rkv.Shape

enum Field { kProblems, kKvHeads, kQHeads, kTokens, kBudget, kAlpha, kHeadDim, kPoolW, kBeta, kThreshold, kLam, kEps, kFlags, kPageSize, kFields };
const char* const kNames[kFields] = {"num_problems", "kv_heads", "q_heads", "n_tokens", "budget", "alpha", "head_dim",
                                     "pool_w", "beta", "sim_threshold", "lam", "eps", "flags", "page_size"};
PyObject* names[kFields];

// One field of the shape as it lies in the parameter block: an int inside its range, or a float.
bool int_field(PyObject* shape, Field f, int64_t lo, int64_t hi, int64_t* out) {
  PyObject* v = PyObject_GetAttr(shape, names[f]);
  if (v == nullptr) return false;
  const bool is_int = PyLong_CheckExact(v);
  int over = 0;
  *out = is_int ? PyLong_AsLongLongAndOverflow(v, &over) : 0;
  Py_DECREF(v);
  return is_int && over == 0 && *out >= lo && *out <= hi;
}
bool float_field(PyObject* shape, Field f, float* out) {
  PyObject* v = PyObject_GetAttr(shape, names[f]);
  if (v == nullptr) return false;
  const bool is_float = PyFloat_CheckExact(v);
  *out = is_float ? (float)PyFloat_AS_DOUBLE(v) : 0.f;
  Py_DECREF(v);
  return is_float;
}

// Strides of 0 in all dimensions but the last say dense to the library, which one row broadcast to all places is not.
bool rows_apart(const at::Tensor& t) { return t.stride(0) != 0 || t.stride(1) != 0 || t.stride(2) != 0 || t.is_contiguous(); }

// A plain strided bf16 tensor in GPU memory with the given sizes; `dense`: contiguous, else only its last dimension.
const at::Tensor* plain(PyObject* o, at::IntArrayRef sizes, bool dense) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.scalar_type() != at::kBFloat16 ||
      t.sizes() != sizes || (dense ? !t.is_contiguous() : t.stride(3) != 1 || !rows_apart(t)))
    return nullptr;
  return &t;
}

PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (count != 9) {
    PyErr_SetString(PyExc_TypeError, "append takes a shape, six tensors, a position and a slot");
    return nullptr;
  }
  try {
    PyObject* shape = args[0];
    constexpr int64_t kMax = INT32_MAX;
    int64_t n[kFields] = {};
    rkv_params p = {};
    // (a subclass may fill the parameter block in its own way)
    bool ok = append_fn != nullptr && (PyObject*)Py_TYPE(shape) == shape_type;
    for (Field f : {kProblems, kKvHeads, kQHeads, kTokens, kBudget, kAlpha, kHeadDim, kPoolW, kBeta}) ok = ok && int_field(shape, f, -kMax - 1, kMax, &n[f]);
    ok = ok && int_field(shape, kFlags, 0, UINT32_MAX, &n[kFlags]) && int_field(shape, kPageSize, 0, 0, &n[kPageSize]);
    ok = ok && float_field(shape, kThreshold, &p.sim_threshold) && float_field(shape, kLam, &p.lambda) && float_field(shape, kEps, &p.eps);
    int over_at = 0, over_slot = 0;
    ok = ok && PyLong_CheckExact(args[7]) && PyLong_CheckExact(args[8]);
    const long long at_row = ok ? PyLong_AsLongLongAndOverflow(args[7], &over_at) : 0, slot = ok ? PyLong_AsLongLongAndOverflow(args[8], &over_slot) : 0;
    ok = ok && over_at == 0 && over_slot == 0 && at_row >= -kMax && at_row <= kMax && slot >= -kMax && slot <= kMax;
    if (PyErr_Occurred()) PyErr_Clear();                 // (a shape without one of the fields: the binding answers that)
    if (!ok) Py_RETURN_NONE;
    const int64_t P = n[kProblems], H = n[kKvHeads], Hq = n[kQHeads], N = n[kTokens], d = n[kHeadDim];
    const at::Tensor* k = plain(args[1], {P, H, N, d}, false);
    const at::Tensor* v = plain(args[2], {P, H, N, d}, false);
    const at::Tensor* q = plain(args[3], {P, Hq, n[kAlpha], d}, false);
    const at::Tensor* k_new = plain(args[4], {P, H, d}, true);
    const at::Tensor* v_new = plain(args[5], {P, H, d}, true);
    const at::Tensor* q_new = plain(args[6], {P, Hq, d}, true);
    if (!k || !v || !q || !k_new || !v_new || !q_new) Py_RETURN_NONE;
    const int device = c10::hip::current_device();       // whose stream is used
    for (const at::Tensor* t : {k, v, q, k_new, v_new, q_new})
      if (t->get_device() != device) Py_RETURN_NONE;
    p.num_problems = (int32_t)P; p.kv_heads = (int32_t)H; p.q_heads = (int32_t)Hq; p.n_tokens = (int32_t)N; p.head_dim = (int32_t)d;
    p.alpha = (int32_t)n[kAlpha]; p.budget = (int32_t)n[kBudget]; p.pool_w = (int32_t)n[kPoolW]; p.beta = (int32_t)n[kBeta];
    p.flags = (uint32_t)n[kFlags];
    p.k_stride_problem = k->stride(0); p.k_stride_head = k->stride(1); p.k_stride_token = k->stride(2);
    p.v_stride_problem = v->stride(0); p.v_stride_head = v->stride(1); p.v_stride_token = v->stride(2);
    if (!q->is_contiguous()) { p.q_stride_problem = q->stride(0); p.q_stride_head = q->stride(1); p.q_stride_token = q->stride(2); }
    void *kp = k->data_ptr(), *vp = v->data_ptr(), *qp = q->data_ptr(), *kn = k_new->data_ptr(), *vn = v_new->data_ptr(), *qn = q_new->data_ptr();
    void* stream = c10::hip::getCurrentHIPStream().stream();
    rkv_status s;
    // (a launch can wait for room in its queue; the caller holds references to all arguments)
    Py_BEGIN_ALLOW_THREADS
    s = append_fn(&p, kp, vp, qp, kn, vn, qn, (int32_t)at_row, (int32_t)slot, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(s);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// ------------------------------------------------------------------------------ the decode loop around the step (rkv_attend.h)
using RotaryFn = rkv_status (*)(const rkv_params*, const rkv_rotary_params*, void*, void*, void*, const void*, const void*, const void*, void*, void*);
using AttendFn = rkv_status (*)(const rkv_params*, const rkv_attend_params*, const void*, const void*, const void*, void*, float*, void*, size_t, void*);
RotaryFn rotary_fn = nullptr;
AttendFn attend_fn = nullptr, shared_fn = nullptr;
PyObject* block_table_name = nullptr;

// A plain strided tensor of the current device, or nullptr.
const at::Tensor* here(PyObject* o, at::ScalarType type, int device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.scalar_type() != type || t.get_device() != device) return nullptr;
  return &t;
}
// (asked before the device: a process without a GPU has none to name)
bool on_gpu(PyObject* o) { return THPVariable_CheckExact(o) && THPVariable_Unpack(o).defined() && THPVariable_Unpack(o).is_cuda(); }
const int32_t* list_of(PyObject* o, int64_t entries, int device) {
  const at::Tensor* t = here(o, at::kInt, device);
  return t != nullptr && t->dim() == 1 && t->size(0) == entries && t->is_contiguous() ? static_cast<const int32_t*>(t->data_ptr()) : nullptr;
}

// The caches that a shape and two tensors describe, as they lie in the parameter block.
struct Caches {
  rkv_params p;
  int64_t P, H, Hq, N, d, alpha;
  int64_t pages;
  const at::Tensor *k, *v;
};
bool caches_of(PyObject* shape, PyObject* k, PyObject* v, int device, Caches* c) {
  c->p = rkv_params{};
  constexpr int64_t kMax = INT32_MAX;
  int64_t page = 0;
  if ((PyObject*)Py_TYPE(shape) != shape_type) return false;
  if (!int_field(shape, kProblems, 1, kMax, &c->P) || !int_field(shape, kKvHeads, 1, kMax, &c->H) || !int_field(shape, kQHeads, 1, kMax, &c->Hq) ||
      !int_field(shape, kTokens, 1, kMax, &c->N) || !int_field(shape, kHeadDim, 1, kMax, &c->d) || !int_field(shape, kAlpha, 1, kMax, &c->alpha) ||
      !int_field(shape, kPageSize, 0, kMax, &page))
    return false;
  c->k = here(k, at::kBFloat16, device);
  c->v = here(v, at::kBFloat16, device);
  if (c->k == nullptr || c->v == nullptr || c->k->dim() != 4 || c->v->dim() != 4 || c->k->stride(3) != 1 || c->v->stride(3) != 1) return false;
  const int64_t rows = page > 0 ? page : c->N;
  for (const at::Tensor* t : {c->k, c->v})
    if ((page == 0 && t->size(0) != c->P) || t->size(1) != c->H || t->size(2) != rows || t->size(3) != c->d || !rows_apart(*t)) return false;
  rkv_params& p = c->p;
  p.num_problems = (int32_t)c->P; p.kv_heads = (int32_t)c->H; p.q_heads = (int32_t)c->Hq; p.n_tokens = (int32_t)c->N; p.head_dim = (int32_t)c->d;
  p.alpha = (int32_t)c->alpha;
  p.k_stride_head = c->k->stride(1); p.k_stride_token = c->k->stride(2);
  p.v_stride_head = c->v->stride(1); p.v_stride_token = c->v->stride(2);
  c->pages = 0;
  if (page == 0) {
    p.k_stride_problem = c->k->stride(0); p.v_stride_problem = c->v->stride(0);
    return true;
  }
  PyObject* table = PyObject_GetAttr(shape, block_table_name);
  const at::Tensor* t = table != nullptr ? here(table, at::kInt, device) : nullptr;
  const bool ok = t != nullptr && t->dim() == 2 && t->size(0) == c->P && t->size(1) <= kMax && t->is_contiguous();
  if (ok) {
    p.page_size = (int32_t)page; p.table_stride = (int32_t)t->size(1); p.block_table = static_cast<const int32_t*>(t->data_ptr());
    p.k_stride_page = c->k->stride(0); p.v_stride_page = c->v->stride(0);
    c->pages = std::min({c->k->size(0), c->v->size(0), kMax});
  }
  Py_XDECREF(table);                                     // (the shape holds it)
  return ok;
}

// bf16 [T, heads, d] with a contiguous last dimension, and its strides: 0, 0 says dense, where there is one token or one head only its
// stride is the dense one, and an array with a broadcast dimension is not taken (its strides of 0 would say dense).
const at::Tensor* tokens_of(PyObject* o, int64_t T, int64_t heads, int64_t d, int device, int64_t* st, int64_t* sh) {
  const at::Tensor* t = here(o, at::kBFloat16, device);
  if (t == nullptr || t->dim() != 3 || t->size(0) != T || t->size(1) != heads || t->size(2) != d || t->stride(2) != 1) return nullptr;
  if (t->is_contiguous()) {
    *st = *sh = 0;
    return t;
  }
  *st = T == 1 ? heads * d : t->stride(0);
  *sh = heads == 1 ? d : t->stride(1);
  return *st != 0 && *sh != 0 ? t : nullptr;
}
bool int_arg(PyObject* o, int64_t* out) {
  int over = 0;
  if (!PyLong_CheckExact(o)) return false;
  *out = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0 && *out >= 0 && *out <= INT32_MAX;
}

PyObject* append_rotary(PyObject*, PyObject* const* args, Py_ssize_t count) {
  // shape, k_cache, v_cache, q_cache, k_new, v_new, q_new, cos, sin, starts, held, seen, interleaved, q_out
  if (count != 14) {
    PyErr_SetString(PyExc_TypeError, "append_rotary takes 14 arguments");
    return nullptr;
  }
  try {
    if (!on_gpu(args[1])) Py_RETURN_NONE;
    const int device = c10::hip::current_device();
    Caches c;
    bool ok = rotary_fn != nullptr && caches_of(args[0], args[1], args[2], device, &c);
    if (PyErr_Occurred()) PyErr_Clear();
    if (!ok) Py_RETURN_NONE;
    rkv_rotary_params r = {};
    const at::Tensor* k0 = here(args[4], at::kBFloat16, device);
    if (k0 == nullptr || k0->dim() != 3 || k0->size(0) > INT32_MAX) Py_RETURN_NONE;
    const int64_t T = k0->size(0);
    const at::Tensor* k = tokens_of(args[4], T, c.H, c.d, device, &r.k_stride_token, &r.k_stride_head);
    const at::Tensor* v = tokens_of(args[5], T, c.H, c.d, device, &r.v_stride_token, &r.v_stride_head);
    const at::Tensor* q = tokens_of(args[6], T, c.Hq, c.d, device, &r.q_stride_token, &r.q_stride_head);
    const at::Tensor *cos = here(args[7], at::kFloat, device), *sin = here(args[8], at::kFloat, device);
    if (!k || !v || !q || !cos || !sin || cos->dim() != 2 || cos->sizes() != sin->sizes() || !cos->is_contiguous() || !sin->is_contiguous() ||
        cos->size(0) > INT32_MAX || cos->size(1) > INT32_MAX / 2 || (args[12] != Py_True && args[12] != Py_False))
      Py_RETURN_NONE;
    void* ring = nullptr;
    if (args[3] != Py_None) {
      const at::Tensor* t = here(args[3], at::kBFloat16, device);
      if (t == nullptr || t->sizes() != at::IntArrayRef({c.P, c.Hq, c.alpha, c.d}) || t->stride(3) != 1 || !rows_apart(*t)) Py_RETURN_NONE;
      if (!t->is_contiguous()) { c.p.q_stride_problem = t->stride(0); c.p.q_stride_head = t->stride(1); c.p.q_stride_token = t->stride(2); }
      ring = t->data_ptr();
    }
    r.tokens = (int32_t)T; r.rotary_dim = (int32_t)(2 * cos->size(1)); r.interleaved = args[12] == Py_True; r.table_rows = (int32_t)cos->size(0);
    r.num_pages = (int32_t)c.pages;
    r.cos = static_cast<const float*>(cos->data_ptr()); r.sin = static_cast<const float*>(sin->data_ptr());
    r.starts = list_of(args[9], c.P + 1, device); r.held = list_of(args[10], c.P, device); r.seen = list_of(args[11], c.P, device);
    if (!r.starts || !r.held || !r.seen) Py_RETURN_NONE;
    at::Tensor made;
    const at::Tensor* out = nullptr;
    if (args[13] == Py_None) {
      made = at::empty(q->sizes(), q->options());
      out = &made;
    } else if ((out = tokens_of(args[13], T, c.Hq, c.d, device, &r.o_stride_token, &r.o_stride_head)) == nullptr) {
      Py_RETURN_NONE;
    }
    void *kc = c.k->data_ptr(), *vc = c.v->data_ptr(), *kn = k->data_ptr(), *vn = v->data_ptr(), *qn = q->data_ptr(), *qo = out->data_ptr();
    void* stream = c10::hip::getCurrentHIPStream().stream();
    rkv_status s;
    Py_BEGIN_ALLOW_THREADS
    s = rotary_fn(&c.p, &r, kc, vc, ring, kn, vn, qn, qo, stream);
    Py_END_ALLOW_THREADS
    PyObject* result = PyTuple_New(2);
    if (result == nullptr) return nullptr;
    PyTuple_SET_ITEM(result, 0, PyLong_FromLong(s));
    PyObject* o = args[13];
    if (o == Py_None) o = THPVariable_Wrap(made);
    else Py_INCREF(o);
    PyTuple_SET_ITEM(result, 1, o);
    return result;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyObject* attend(PyObject*, PyObject* const* args, Py_ssize_t count) {
  // shape, q, k, v, starts, kv_len, group_starts, prefix_len, window, sinks, scale, max_new, ws, out, lse, want_lse
  if (count != 16) {
    PyErr_SetString(PyExc_TypeError, "attend takes 16 arguments");
    return nullptr;
  }
  try {
    if (!on_gpu(args[2])) Py_RETURN_NONE;
    const int device = c10::hip::current_device();
    Caches c;
    bool ok = attend_fn != nullptr && caches_of(args[0], args[2], args[3], device, &c);
    if (PyErr_Occurred()) PyErr_Clear();
    if (!ok) Py_RETURN_NONE;
    rkv_attend_params a = {};
    const at::Tensor* q0 = here(args[1], at::kBFloat16, device);
    if (q0 == nullptr || q0->dim() != 3 || q0->size(0) > INT32_MAX) Py_RETURN_NONE;
    const int64_t T = q0->size(0);
    const at::Tensor* q = tokens_of(args[1], T, c.Hq, c.d, device, &a.q_stride_token, &a.q_stride_head);
    int64_t window, sinks, max_new = T;
    if (q == nullptr || !int_arg(args[8], &window) || !int_arg(args[9], &sinks) || (args[11] != Py_None && !int_arg(args[11], &max_new))) Py_RETURN_NONE;
    a.starts = list_of(args[4], c.P + 1, device);
    a.kv_len = list_of(args[5], c.P, device);
    if (!a.starts || !a.kv_len) Py_RETURN_NONE;
    const bool shared = args[6] != Py_None;
    if (shared) {
      const at::Tensor* t = here(args[7], at::kInt, device);
      if (t == nullptr || t->dim() != 1 || t->size(0) > c.P) Py_RETURN_NONE;
      a.groups = (int32_t)t->size(0);
      a.group_starts = list_of(args[6], a.groups + 1, device);
      a.prefix_len = list_of(args[7], a.groups, device);
      if (a.group_starts == nullptr || (a.prefix_len == nullptr && a.groups > 0)) Py_RETURN_NONE;
    }
    if (args[10] == Py_None) a.scale = (float)std::pow((double)c.d, -0.5);
    else if (PyFloat_CheckExact(args[10])) a.scale = (float)PyFloat_AS_DOUBLE(args[10]);
    else Py_RETURN_NONE;
    a.tokens = (int32_t)T; a.max_new = (int32_t)max_new; a.window = (int32_t)window; a.sinks = (int32_t)sinks; a.num_pages = (int32_t)c.pages;
    // (a workspace that the call allocates by itself is sized and made in Python)
    if (!THPVariable_CheckExact(args[12])) Py_RETURN_NONE;
    const at::Tensor& ws = THPVariable_Unpack(args[12]);
    if (!ws.defined() || !ws.is_cuda() || ws.get_device() != device || ws.scalar_type() != at::kByte || !ws.is_contiguous()) Py_RETURN_NONE;
    at::Tensor made, made_lse;
    const at::Tensor *out = nullptr, *lse = nullptr;
    if (args[13] == Py_None) {
      made = at::empty(q->sizes(), q->options());
      out = &made;
    } else if ((out = tokens_of(args[13], T, c.Hq, c.d, device, &a.o_stride_token, &a.o_stride_head)) == nullptr) {
      Py_RETURN_NONE;
    }
    const int want = PyObject_IsTrue(args[15]);
    if (want < 0) return nullptr;
    if (args[14] != Py_None) {
      lse = here(args[14], at::kFloat, device);
      if (lse == nullptr || lse->sizes() != at::IntArrayRef({T, c.Hq}) || !lse->is_contiguous()) Py_RETURN_NONE;
    } else if (want) {
      made_lse = at::empty({T, c.Hq}, q->options().dtype(at::kFloat));
      lse = &made_lse;
    }
    const uintptr_t base = reinterpret_cast<uintptr_t>(ws.data_ptr()), aligned = (base + 255) & ~(uintptr_t)255;
    const int64_t room = ws.numel() - (int64_t)(aligned - base);
    void *qp = q->data_ptr(), *kp = c.k->data_ptr(), *vp = c.v->data_ptr(), *op = out->data_ptr();
    float* lp = lse != nullptr ? static_cast<float*>(lse->data_ptr()) : nullptr;
    void* stream = c10::hip::getCurrentHIPStream().stream();
    const AttendFn fn = shared ? shared_fn : attend_fn;
    rkv_status s;
    Py_BEGIN_ALLOW_THREADS
    s = fn(&c.p, &a, qp, kp, vp, op, lp, reinterpret_cast<void*>(aligned), room > 0 ? (size_t)room : 0, stream);
    Py_END_ALLOW_THREADS
    PyObject* result = PyTuple_New(3);
    if (result == nullptr) return nullptr;
    PyTuple_SET_ITEM(result, 0, PyLong_FromLong(s));
    PyObject* o = args[13];
    if (o == Py_None) o = THPVariable_Wrap(made);
    else Py_INCREF(o);
    PyTuple_SET_ITEM(result, 1, o);
    PyObject* l = args[14];
    if (l == Py_None && want) l = THPVariable_Wrap(made_lse);
    else Py_INCREF(l);
    PyTuple_SET_ITEM(result, 2, l);
    return result;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// The addresses of rkv_cache_append_rotary, rkv_attend and rkv_attend_shared.
PyObject* bind_attend(PyObject*, PyObject* args) {
  PyObject* address[3];
  if (!PyArg_ParseTuple(args, "OOO", &address[0], &address[1], &address[2])) return nullptr;
  void* p[3];
  for (int i = 0; i < 3; ++i) {
    p[i] = PyLong_AsVoidPtr(address[i]);
    if (p[i] == nullptr && PyErr_Occurred()) return nullptr;
  }
  rotary_fn = reinterpret_cast<RotaryFn>(p[0]);
  attend_fn = reinterpret_cast<AttendFn>(p[1]);
  shared_fn = reinterpret_cast<AttendFn>(p[2]);
  Py_RETURN_NONE;
}

// The address of rkv_cache_append in the loaded library and the class of its shapes.
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *address, *type;
  if (!PyArg_ParseTuple(args, "OO!", &address, &PyType_Type, &type)) return nullptr;
  void* p = PyLong_AsVoidPtr(address);
  if (p == nullptr && PyErr_Occurred()) return nullptr;
  append_fn = reinterpret_cast<AppendFn>(p);
  Py_INCREF(type);
  Py_XDECREF(shape_type);
  shape_type = type;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append)), METH_FASTCALL,
     "append(shape, k_cache, v_cache, q_cache, k_new, v_new, q_new, position, slot) -> status, or None if the call is not taken"},
    {"bind", bind, METH_VARARGS, "bind(address of rkv_cache_append, class of the shapes)"},
    {"append_rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append_rotary)), METH_FASTCALL,
     "append_rotary(the arguments of rkv_cache_append_rotary) -> (status, q_out), or None if the call is not taken"},
    {"attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attend)), METH_FASTCALL,
     "attend(the arguments of rkv_attend_shared) -> (status, out, lse), or None if the call is not taken"},
    {"bind_attend", bind_attend, METH_VARARGS, "bind_attend(addresses of rkv_cache_append_rotary, rkv_attend, rkv_attend_shared)"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() {
  for (int f = 0; f < kFields; ++f)
    if ((names[f] = PyUnicode_InternFromString(kNames[f])) == nullptr) return nullptr;
  if ((block_table_name = PyUnicode_InternFromString("block_table")) == nullptr) return nullptr;
  return PyModule_Create(&module);
}
