// The short way from PyTorch tensors to the C ABI (include/mw_bca.h): checks
// of arguments that need nothing special, output allocation and the call, in
// one native function each.
//
// A call's kernels take from 5 us; the same checks and allocations written in
// Python take 10-40 us of host time a call on the Grace cores (more on the
// autograd thread, whose caches are cold), which is what bounds small windows
// and short streams.  Anything unusual -- another type or layout, buffers the
// caller supplies, a wrapped or fake tensor, sizes that do not fit -- makes a
// function here return None, and the Python binding's full checks then run
// and name what is wrong.  An int is a non-zero mw_status.
//
// The C entry points are handed over as addresses (bind), so that this module
// and the ctypes binding share one loaded library and its options.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <ATen/core/grad_mode.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>

#include <array>
#include <climits>
#include <cmath>
#include <initializer_list>
#include <vector>

#include "mw_bca.h"

namespace {

decltype(&mw_bca_fwd) p_fwd = nullptr;
decltype(&mw_bca_bwd) p_bwd = nullptr;
decltype(&mw_bca_bwd_workspace_size) p_bwd_ws = nullptr;
decltype(&mw_bca_cache_workspace_size) p_cache_ws = nullptr;
decltype(&mw_bca_cache_fwd_rope) p_cache = nullptr;
decltype(&mw_bca_cache_step) p_step = nullptr;
decltype(&mw_qkv_rope_split) p_qkv = nullptr;
decltype(&mw_xattn_workspace_size) p_xattn_ws = nullptr;
decltype(&mw_xattn_fwd) p_xattn = nullptr;
decltype(&mw_xattn_bwd_workspace_size) p_xattn_bwd_ws = nullptr;
decltype(&mw_xattn_bwd) p_xattn_bwd = nullptr;
decltype(&mw_layernorm_fwd) p_norm = nullptr;
decltype(&mw_layernorm_bwd_workspace_size) p_norm_bwd_ws = nullptr;
decltype(&mw_layernorm_bwd) p_norm_bwd = nullptr;
decltype(&mw_last_error) p_last_error = nullptr;
PyObject* error_type = nullptr;  // MWError(code, message)

// A tensor this module may look into: exactly a torch.Tensor or Parameter,
// strided, with storage of its own (no fake, batched or other wrapper).
bool is_real(const at::Tensor& t) {
  return t.unsafeGetTensorImpl()->has_storage() && t.layout() == at::kStrided && t.is_cuda() &&
         !t.unsafeGetTensorImpl()->key_set().has(c10::DispatchKey::Python) && !t.is_neg();
}

// (with a torch function or dispatch mode on, which wants to see every
// allocation, nothing here is taken)
const at::Tensor* tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o) || at::impl::torch_function_mode_enabled() ||
      c10::impl::TorchDispatchModeTLS::any_modes_set())
    return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && is_real(t) && t.is_contiguous() ? &t : nullptr;
}

// The i-th argument as a bf16 tensor of `dims` dimensions, else null.
const at::Tensor* bf16(PyObject* o, int dims) {
  const at::Tensor* t = tensor(o);
  return t && t->scalar_type() == at::kBFloat16 && t->dim() == dims ? t : nullptr;
}

// The device of all tensors (null pointers skipped), if it is one and current.
bool one_device(std::initializer_list<const at::Tensor*> ts, c10::DeviceIndex* dev) {
  *dev = -1;
  for (const at::Tensor* t : ts) {
    if (!t) continue;
    if (*dev < 0)
      *dev = t->get_device();
    else if (t->get_device() != *dev)
      return false;
  }
  return *dev >= 0 && *dev == c10::cuda::current_device();
}

bool small_int(PyObject* o, int* out) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long v = PyLong_AsLongAndOverflow(o, &over);
  if (over || v < INT_MIN || v > INT_MAX) return false;
  *out = static_cast<int>(v);
  return true;
}

bool real_number(PyObject* o, float* out) {
  if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *out = static_cast<float>(v);
  return true;
}

// The softmax scale: None is 1 / sqrt(d).
bool softmax_scale(PyObject* o, int64_t d, float* out) {
  if (o == Py_None) {
    *out = static_cast<float>(1.0 / std::sqrt(static_cast<double>(d)));
    return true;
  }
  return real_number(o, out);
}

bool fits(const at::Tensor& t) {
  for (int64_t s : t.sizes())
    if (s > INT_MAX) return false;
  return true;
}

// Bytes [lo, hi) of a tensor, to see that written buffers stand apart.
struct Span {
  const char* lo;
  const char* hi;
};
Span span(const at::Tensor& t) {
  const char* p = static_cast<const char*>(t.const_data_ptr());
  return {p, p + t.nbytes()};
}

// Sizes of a [B, H, rows, d] tensor, as the outputs are allocated from them.
using Shape = std::array<int64_t, 4>;
Shape shape(const at::Tensor& t) { return {t.size(0), t.size(1), t.size(2), t.size(3)}; }

at::Tensor rows_f32(const Shape& s, const at::TensorOptions& options) {
  return at::empty({s[0], s[1], s[2]}, options.dtype(at::kFloat));
}

at::Tensor scratch(size_t bytes, const at::TensorOptions& options) {
  return at::empty({static_cast<int64_t>(bytes)}, options.dtype(at::kByte));
}

PyObject* none() { Py_RETURN_NONE; }

PyObject* result(std::initializer_list<const at::Tensor*> ts) {
  PyObject* tup = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
  if (!tup) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor* t : ts) {
    PyObject* o = t->defined() ? THPVariable_Wrap(*t) : Py_NewRef(Py_None);
    if (!o) {
      Py_DECREF(tup);
      return nullptr;
    }
    PyTuple_SET_ITEM(tup, i++, o);
  }
  return tup;
}

// Runs f, which allocates the outputs and launches, without the interpreter lock:
// an allocation can wait for the device, a launch for room in the stream's queue,
// and what they wait for can be a callback that needs the lock.  Sizes and data
// pointers of the arguments are taken before, with the lock.  A guard, since f
// may throw (out of memory).  f returns false for outputs that are not real
// tensors (is_real), and sets the status otherwise.
class WithoutLock {
 public:
  WithoutLock() : state_(PyEval_SaveThread()) {}
  ~WithoutLock() { PyEval_RestoreThread(state_); }
  WithoutLock(const WithoutLock&) = delete;
  WithoutLock& operator=(const WithoutLock&) = delete;

 private:
  PyThreadState* state_;
};

template <class F>
auto call(F&& f) {
  WithoutLock unlocked;
  return f();
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int kEntries = 15;
  if (n != kEntries + 1) {
    PyErr_SetString(PyExc_TypeError, "bind takes 15 addresses and the error type");
    return nullptr;
  }
  void* p[kEntries];
  for (int i = 0; i < kEntries; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  p_fwd = reinterpret_cast<decltype(p_fwd)>(p[0]);
  p_bwd = reinterpret_cast<decltype(p_bwd)>(p[1]);
  p_bwd_ws = reinterpret_cast<decltype(p_bwd_ws)>(p[2]);
  p_cache_ws = reinterpret_cast<decltype(p_cache_ws)>(p[3]);
  p_cache = reinterpret_cast<decltype(p_cache)>(p[4]);
  p_step = reinterpret_cast<decltype(p_step)>(p[5]);
  p_qkv = reinterpret_cast<decltype(p_qkv)>(p[6]);
  p_xattn_ws = reinterpret_cast<decltype(p_xattn_ws)>(p[7]);
  p_xattn = reinterpret_cast<decltype(p_xattn)>(p[8]);
  p_xattn_bwd_ws = reinterpret_cast<decltype(p_xattn_bwd_ws)>(p[9]);
  p_xattn_bwd = reinterpret_cast<decltype(p_xattn_bwd)>(p[10]);
  p_norm = reinterpret_cast<decltype(p_norm)>(p[11]);
  p_norm_bwd_ws = reinterpret_cast<decltype(p_norm_bwd_ws)>(p[12]);
  p_norm_bwd = reinterpret_cast<decltype(p_norm_bwd)>(p[13]);
  p_last_error = reinterpret_cast<decltype(p_last_error)>(p[14]);
  Py_XDECREF(error_type);
  error_type = Py_NewRef(a[kEntries]);
  Py_RETURN_NONE;
}

// fwd(q, k, v, T_chunk, scale, need_lse) -> (o, lse or None)
PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6 || !p_fwd) return none();
  const at::Tensor *q = bf16(a[0], 4), *k = bf16(a[1], 4), *v = bf16(a[2], 4);
  c10::DeviceIndex dev;
  int T;
  float scale;
  if (!q || !k || !v || k->sizes() != q->sizes() || v->sizes() != q->sizes() || !fits(*q) ||
      !one_device({q, k, v}, &dev) || !small_int(a[3], &T) || T < 1 || q->size(2) % T ||
      !softmax_scale(a[4], q->size(3), &scale) || !PyBool_Check(a[5]))
    return none();
  const Shape sh = shape(*q);
  const at::TensorOptions options = q->options();
  const void *pq = q->const_data_ptr(), *pk = k->const_data_ptr(), *pv = v->const_data_ptr();
  const bool need_lse = a[5] == Py_True;
  at::Tensor o, lse;
  mw_status s = MW_OK;
  const bool real = call([&] {
    o = at::empty(sh, options);
    if (need_lse) lse = rows_f32(sh, options);
    if (!is_real(o) || (need_lse && !is_real(lse))) return false;
    s = p_fwd(pq, pk, pv, o.mutable_data_ptr(),
              need_lse ? static_cast<float*>(lse.mutable_data_ptr()) : nullptr,
              static_cast<int>(sh[0]), static_cast<int>(sh[1]), static_cast<int>(sh[2] / T), T,
              static_cast<int>(sh[3]), scale, c10::cuda::getCurrentCUDAStream(dev).stream());
    return true;
  });
  if (!real) return none();
  if (s != MW_OK) return PyLong_FromLong(s);
  return result({&o, &lse});
  END_HANDLE_TH_ERRORS
}

// bwd(q, k, v, o, lse, dout, T_chunk, scale) -> (dq, dk, dv)
PyObject* bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8 || !p_bwd) return none();
  const at::Tensor *q = bf16(a[0], 4), *k = bf16(a[1], 4), *v = bf16(a[2], 4), *o = bf16(a[3], 4);
  const at::Tensor *lse = tensor(a[4]), *dout = bf16(a[5], 4);
  c10::DeviceIndex dev;
  int T;
  float scale;
  if (!q || !k || !v || !o || !lse || !dout || k->sizes() != q->sizes() ||
      v->sizes() != q->sizes() || o->sizes() != q->sizes() || dout->sizes() != q->sizes() ||
      !fits(*q) || lse->scalar_type() != at::kFloat || lse->sizes() != q->sizes().slice(0, 3) ||
      !one_device({q, k, v, o, lse, dout}, &dev) || !small_int(a[6], &T) || T < 1 ||
      q->size(2) % T || !softmax_scale(a[7], q->size(3), &scale))
    return none();
  const Shape sh = shape(*q);
  const at::TensorOptions options = q->options();
  const int B = static_cast<int>(sh[0]), H = static_cast<int>(sh[1]);
  const int nc = static_cast<int>(sh[2] / T), d = static_cast<int>(sh[3]);
  const size_t bytes = p_bwd_ws(B, H, nc, T, d);
  const void *pq = q->const_data_ptr(), *pk = k->const_data_ptr(), *pv = v->const_data_ptr();
  const void *po = o->const_data_ptr(), *pdo = dout->const_data_ptr();
  const float* pl = static_cast<const float*>(lse->const_data_ptr());
  at::Tensor ws, dq, dk, dv;
  mw_status s = MW_OK;
  const bool real = call([&] {
    ws = scratch(bytes, options);
    dq = at::empty(sh, options);
    dk = at::empty(sh, options);
    dv = at::empty(sh, options);
    if (!is_real(ws) || !is_real(dq) || !is_real(dk) || !is_real(dv)) return false;
    s = p_bwd(pq, pk, pv, po, pl, pdo, dq.mutable_data_ptr(), dk.mutable_data_ptr(),
              dv.mutable_data_ptr(), bytes ? ws.mutable_data_ptr() : nullptr, bytes, B, H, nc, T, d,
              scale, c10::cuda::getCurrentCUDAStream(dev).stream());
    return true;
  });
  if (!real) return none();
  if (s != MW_OK) return PyLong_FromLong(s);
  return result({&dq, &dk, &dv});
  END_HANDLE_TH_ERRORS
}

// cache(q, k_new, v_new, k_sink, v_sink, k_cache, v_cache, head, len, T_chunk,
//       scale, need_lse, workspace, rope, commit) -> (o, lse or None)
// rope: None or (dims, base, shift); commit: None or (slot, rows)
PyObject* cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 15 || !p_cache) return none();
  const at::Tensor *q = bf16(a[0], 4), *kn = bf16(a[1], 4), *vn = bf16(a[2], 4);
  const at::Tensor *kc = bf16(a[5], 4), *vc = bf16(a[6], 4), *ks = nullptr, *vs = nullptr;
  const bool sink = a[3] != Py_None || a[4] != Py_None;
  if (sink) {
    ks = bf16(a[3], 4);
    vs = bf16(a[4], 4);
    if (!ks || !vs || ks->sizes() != vs->sizes() || !fits(*ks)) return none();
  }
  const at::Tensor* given = a[12] == Py_None ? nullptr : tensor(a[12]);
  c10::DeviceIndex dev;
  int head, len, T;
  float scale;
  if (!q || !kn || !vn || !kc || !vc || kn->sizes() != q->sizes() || vn->sizes() != q->sizes() ||
      vc->sizes() != kc->sizes() || !fits(*q) || !fits(*kc) || (a[12] != Py_None && !given) ||
      !one_device({q, kn, vn, kc, vc, ks, vs, given}, &dev) || !small_int(a[7], &head) ||
      !small_int(a[8], &len) || !small_int(a[9], &T) || T < 1 || q->size(2) % T ||
      !softmax_scale(a[10], q->size(3), &scale) || !PyBool_Check(a[11]))
    return none();
  for (const at::Tensor* t : {kc, ks})
    if (t && (t->size(0) != q->size(0) || t->size(1) != q->size(1) || t->size(3) != q->size(3)))
      return none();
  int rope_dims = 0, shift = 0, slot = 0, rows = 0;
  float base = 0.f;
  const bool rope = a[13] != Py_None, commit = a[14] != Py_None;
  if (rope && (!PyTuple_CheckExact(a[13]) || PyTuple_GET_SIZE(a[13]) != 3 ||
               !small_int(PyTuple_GET_ITEM(a[13], 0), &rope_dims) ||
               !real_number(PyTuple_GET_ITEM(a[13], 1), &base) ||
               !small_int(PyTuple_GET_ITEM(a[13], 2), &shift)))
    return none();
  if (commit && (rope || sink || !PyTuple_CheckExact(a[14]) || PyTuple_GET_SIZE(a[14]) != 2 ||
                 !small_int(PyTuple_GET_ITEM(a[14], 0), &slot) ||
                 !small_int(PyTuple_GET_ITEM(a[14], 1), &rows)))
    return none();
  const int sink_len = ks ? static_cast<int>(ks->size(2)) : 0;
  const int64_t keys = static_cast<int64_t>(sink_len) + len;
  if (keys > INT_MAX || keys < 0) return none();
  const Shape sh = shape(*q);
  const at::TensorOptions options = q->options();
  const int B = static_cast<int>(sh[0]), H = static_cast<int>(sh[1]);
  const int W = static_cast<int>(sh[2] / T), d = static_cast<int>(sh[3]);
  const size_t bytes = p_cache_ws(B, H, W, T, d, static_cast<int>(keys));
  // what the call writes shares no byte with anything else of the caller's
  Span spans[8];
  int n_spans = 0, n_written = 0;
  if (given) spans[n_spans++] = span(*given), ++n_written;
  spans[n_spans++] = span(*kc);
  spans[n_spans++] = span(*vc);
  if (commit) n_written += 2;
  for (const at::Tensor* t : {q, kn, vn, ks, vs})
    if (t) spans[n_spans++] = span(*t);
  for (int i = 0; i < n_written; ++i)
    for (int j = i + 1; j < n_spans; ++j)
      if (spans[i].lo < spans[j].hi && spans[j].lo < spans[i].hi) return none();
  const void *pq = q->const_data_ptr(), *pkn = kn->const_data_ptr(), *pvn = vn->const_data_ptr();
  const void *pks = ks ? ks->const_data_ptr() : nullptr, *pvs = vs ? vs->const_data_ptr() : nullptr;
  // (a commit writes the ring; without one it is only read)
  void* const pkc = commit ? kc->mutable_data_ptr() : const_cast<void*>(kc->const_data_ptr());
  void* const pvc = commit ? vc->mutable_data_ptr() : const_cast<void*>(vc->const_data_ptr());
  const int cap = static_cast<int>(kc->size(2));
  const bool need_lse = a[11] == Py_True;
  const bool use_given = bytes > 0 && given && given->nbytes() >= bytes;
  void* const pgiven = use_given ? given->mutable_data_ptr() : nullptr;
  at::Tensor ws, o, lse;
  mw_status s = MW_OK;
  const bool real = call([&] {
    if (bytes > 0 && !use_given) ws = scratch(bytes, options);
    o = at::empty(sh, options);
    if (need_lse) lse = rows_f32(sh, options);
    if (!is_real(o) || (need_lse && !is_real(lse)) || (ws.defined() && !is_real(ws))) return false;
    void* w = ws.defined() ? ws.mutable_data_ptr() : pgiven;
    float* l = need_lse ? static_cast<float*>(lse.mutable_data_ptr()) : nullptr;
    cudaStream_t st = c10::cuda::getCurrentCUDAStream(dev).stream();
    if (commit)
      s = p_step(pq, pkn, pvn, pkc, pvc, cap, head, len, slot, rows, o.mutable_data_ptr(), l, w,
                 bytes, B, H, W, T, d, scale, st);
    else
      s = p_cache(pq, pkn, pvn, pks, pvs, sink_len, pkc, pvc, cap, head, len, rope_dims, base,
                  shift, o.mutable_data_ptr(), l, w, bytes, B, H, W, T, d, scale, st);
    return true;
  });
  if (!real) return none();
  if (s != MW_OK) return PyLong_FromLong(s);
  return result({&o, &lse});
  END_HANDLE_TH_ERRORS
}

// qkv(qkv, rope_dims, rope_base, tokens_per_frame, first_frame) -> (q, k, v)
PyObject* qkv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 5 || !p_qkv) return none();
  const at::Tensor* x = bf16(a[0], 5);
  c10::DeviceIndex dev;
  int dims, per_frame, first;
  float base;
  if (!x || x->size(2) != 3 || !fits(*x) || !one_device({x}, &dev) || !small_int(a[1], &dims) ||
      !real_number(a[2], &base) || !small_int(a[3], &per_frame) || !small_int(a[4], &first))
    return none();
  const int64_t B = x->size(0), N = x->size(1), H = x->size(3), d = x->size(4);
  const at::TensorOptions options = x->options();
  const void* px = x->const_data_ptr();
  at::Tensor q, k, v;
  mw_status s = MW_OK;
  const bool real = call([&] {
    q = at::empty({B, H, N, d}, options);
    k = at::empty({B, H, N, d}, options);
    v = at::empty({B, H, N, d}, options);
    if (!is_real(q) || !is_real(k) || !is_real(v)) return false;
    s = p_qkv(px, q.mutable_data_ptr(), k.mutable_data_ptr(), v.mutable_data_ptr(),
              static_cast<int>(B), static_cast<int>(N), static_cast<int>(H), static_cast<int>(d),
              dims, base, per_frame, first, c10::cuda::getCurrentCUDAStream(dev).stream());
    return true;
  });
  if (!real) return none();
  if (s != MW_OK) return PyLong_FromLong(s);
  return result({&q, &k, &v});
  END_HANDLE_TH_ERRORS
}

// K and V of a cross attention and the valid states of its samples (null: all).
struct States {
  const at::Tensor *k = nullptr, *v = nullptr, *len = nullptr;
  bool read(const at::Tensor* q, PyObject* ko, PyObject* vo, PyObject* lo) {
    k = bf16(ko, 4);
    v = bf16(vo, 4);
    if (!q || !k || !v || k->sizes() != v->sizes() || !fits(*q) || !fits(*k) ||
        k->size(0) != q->size(0) || k->size(3) != q->size(3) || k->size(1) < 1 ||
        q->size(1) % k->size(1))
      return false;
    if (lo == Py_None) return true;
    len = tensor(lo);
    return len && len->scalar_type() == at::kInt && len->dim() == 1 && len->size(0) == q->size(0);
  }
  const int* lens() const { return len ? static_cast<const int*>(len->const_data_ptr()) : nullptr; }
};

// A cross attention call: its tensors and sizes, and the results of its forward.
struct Xattn {
  const at::Tensor* q = nullptr;
  States st;
  c10::DeviceIndex dev = -1;
  float scale = 0.f;
  at::Tensor o, lse;
  bool read(PyObject* qo, PyObject* ko, PyObject* vo, PyObject* lo, PyObject* so) {
    q = bf16(qo, 4);
    return st.read(q, ko, vo, lo) && one_device({q, st.k, st.v, st.len}, &dev) &&
           softmax_scale(so, q->size(3), &scale);
  }
  // false: outputs that are not real tensors
  bool forward(bool need_lse, mw_status* s) {
    const Shape sh = shape(*q);
    const at::TensorOptions options = q->options();
    const int B = static_cast<int>(sh[0]), H = static_cast<int>(sh[1]), M = static_cast<int>(sh[2]);
    const int Hkv = static_cast<int>(st.k->size(1)), S = static_cast<int>(st.k->size(2));
    const int d = static_cast<int>(sh[3]);
    const size_t bytes = p_xattn_ws(B, H, Hkv, M, S, d);
    const void *pq = q->const_data_ptr(), *pk = st.k->const_data_ptr(), *pv = st.v->const_data_ptr();
    const int* lens = st.lens();
    return call([&] {
      at::Tensor ws;
      o = at::empty(sh, options);
      if (need_lse) lse = rows_f32(sh, options);
      if (bytes) ws = scratch(bytes, options);
      if (!is_real(o) || (need_lse && !is_real(lse)) || (bytes && !is_real(ws))) return false;
      *s = p_xattn(pq, pk, pv, lens, o.mutable_data_ptr(),
                   need_lse ? static_cast<float*>(lse.mutable_data_ptr()) : nullptr,
                   bytes ? ws.mutable_data_ptr() : nullptr, bytes, B, H, Hkv, M, S, d, scale,
                   c10::cuda::getCurrentCUDAStream(dev).stream());
      return true;
    });
  }
};

// xattn_fwd(q, k, v, kv_len, scale, need_lse, workspace) -> (o, lse or None)
PyObject* xattn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Xattn x;
  if (n != 7 || !p_xattn || a[6] != Py_None || !PyBool_Check(a[5]) || !x.read(a[0], a[1], a[2], a[3], a[4]))
    return none();
  mw_status s = MW_OK;
  if (!x.forward(a[5] == Py_True, &s)) return none();
  if (s != MW_OK) return PyLong_FromLong(s);
  return result({&x.o, &x.lse});
  END_HANDLE_TH_ERRORS
}

// The gradients of a cross attention into new tensors; false: not real ones.  Called
// without the interpreter lock.
bool xattn_gradients(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const int* lens,
                     const at::Tensor& o, const at::Tensor& lse, const at::Tensor& dout, float scale,
                     c10::DeviceIndex dev, std::array<at::Tensor, 3>* grads, mw_status* s) {
  const Shape sh = shape(q), ks = shape(k);
  const at::TensorOptions options = q.options();
  const int B = static_cast<int>(sh[0]), H = static_cast<int>(sh[1]), M = static_cast<int>(sh[2]);
  const int Hkv = static_cast<int>(ks[1]), S = static_cast<int>(ks[2]), d = static_cast<int>(sh[3]);
  const size_t bytes = p_xattn_bwd_ws(B, H, Hkv, M, S, d);
  at::Tensor ws;
  if (bytes) ws = scratch(bytes, options);
  (*grads)[0] = at::empty(sh, options);
  (*grads)[1] = at::empty(ks, options);
  (*grads)[2] = at::empty(ks, options);
  if (bytes && !is_real(ws)) return false;
  for (const at::Tensor& t : *grads)
    if (!is_real(t)) return false;
  *s = p_xattn_bwd(q.const_data_ptr(), k.const_data_ptr(), v.const_data_ptr(), lens, o.const_data_ptr(),
                   static_cast<const float*>(lse.const_data_ptr()), dout.const_data_ptr(),
                   (*grads)[0].mutable_data_ptr(), (*grads)[1].mutable_data_ptr(),
                   (*grads)[2].mutable_data_ptr(), bytes ? ws.mutable_data_ptr() : nullptr, bytes, B, H,
                   Hkv, M, S, d, scale, c10::cuda::getCurrentCUDAStream(dev).stream());
  return true;
}

// xattn_bwd(q, k, v, o, lse, dout, kv_len, scale) -> (dq, dk, dv)
PyObject* xattn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8 || !p_xattn_bwd) return none();
  Xattn x;
  const at::Tensor *o = bf16(a[3], 4), *lse = tensor(a[4]), *dout = bf16(a[5], 4);
  c10::DeviceIndex dev;
  if (!x.read(a[0], a[1], a[2], a[6], a[7]) || !o || !lse || !dout || o->sizes() != x.q->sizes() ||
      dout->sizes() != x.q->sizes() || lse->scalar_type() != at::kFloat ||
      lse->sizes() != x.q->sizes().slice(0, 3) || !one_device({x.q, o, lse, dout}, &dev))
    return none();
  std::array<at::Tensor, 3> g;
  mw_status s = MW_OK;
  const int* lens = x.st.lens();
  const bool real =
      call([&] { return xattn_gradients(*x.q, *x.st.k, *x.st.v, lens, *o, *lse, *dout, x.scale, dev, &g, &s); });
  if (!real) return none();
  if (s != MW_OK) return PyLong_FromLong(s);
  return result({&g[0], &g[1], &g[2]});
  END_HANDLE_TH_ERRORS
}

// Type codes of the layer norm's arrays (-1: another type).
int norm_type(at::ScalarType t) { return t == at::kBFloat16 ? MW_BF16 : t == at::kFloat ? MW_F32 : -1; }
at::ScalarType torch_type(int t) { return t == MW_F32 ? at::kFloat : at::kBFloat16; }

// A layer norm call: its tensors and sizes, and the results of its forward.
struct Norm {
  const at::Tensor *x = nullptr, *w = nullptr, *b = nullptr;
  int xt = -1, pt = MW_F32, C = 0, groups = 1;
  int64_t rows = 0;
  c10::DeviceIndex dev = -1;
  at::Tensor y, mean, rstd;
  bool read(PyObject* xo, PyObject* wo, PyObject* bo) {
    x = tensor(xo);
    if (!x || x->dim() < 1 || (xt = norm_type(x->scalar_type())) < 0) return false;
    const int64_t c = x->size(-1);
    if (c < 1 || c > INT_MAX) return false;
    C = static_cast<int>(c);
    rows = x->numel() / c;
    if (wo != Py_None && !(w = tensor(wo))) return false;
    if (bo != Py_None && !(b = tensor(bo))) return false;
    for (const at::Tensor* t : {w, b}) {
      if (!t) continue;
      pt = norm_type(t->scalar_type());
      if (pt < 0 || t->dim() < 1 || t->dim() > 2 || t->size(-1) != c) return false;
      const int64_t g = t->dim() == 2 ? t->size(0) : 1;
      if (g < 1 || g > INT_MAX) return false;
      groups = static_cast<int>(g);
    }
    if (w && b && (w->scalar_type() != b->scalar_type() || w->sizes() != b->sizes())) return false;
    return rows % groups == 0 && one_device({x, w, b}, &dev);
  }
  bool out_type(PyObject* o, int* yt) const {
    *yt = xt;
    if (o == Py_None) return true;
    if (!THPDtype_Check(o)) return false;
    *yt = norm_type(reinterpret_cast<THPDtype*>(o)->scalar_type);
    return *yt >= 0;
  }
  bool forward(float eps, int yt, bool stats, mw_status* s) {
    const at::TensorOptions options = x->options();
    const std::vector<int64_t> full = x->sizes().vec();
    const at::IntArrayRef lead(full.data(), full.size() - 1);
    const void* px = x->const_data_ptr();
    const void *pw = w ? w->const_data_ptr() : nullptr, *pb = b ? b->const_data_ptr() : nullptr;
    return call([&] {
      y = at::empty(full, options.dtype(yt == MW_F32 ? at::kFloat : at::kBFloat16));
      if (stats) {
        mean = at::empty(lead, options.dtype(at::kFloat));
        rstd = at::empty(lead, options.dtype(at::kFloat));
      }
      if (!is_real(y) || (stats && (!is_real(mean) || !is_real(rstd)))) return false;
      *s = p_norm(px, pw, pb, y.mutable_data_ptr(),
                  stats ? static_cast<float*>(mean.mutable_data_ptr()) : nullptr,
                  stats ? static_cast<float*>(rstd.mutable_data_ptr()) : nullptr, rows, C, groups, eps, xt,
                  yt, pt, c10::cuda::getCurrentCUDAStream(dev).stream());
      return true;
    });
  }
};

// norm_fwd(x, weight, bias, eps, out_dtype, need_stats) -> (y, mean or None, rstd or None)
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Norm t;
  float eps;
  int yt;
  if (n != 6 || !p_norm || !t.read(a[0], a[1], a[2]) || !real_number(a[3], &eps) || !t.out_type(a[4], &yt) ||
      !PyBool_Check(a[5]))
    return none();
  mw_status s = MW_OK;
  if (!t.forward(eps, yt, a[5] == Py_True, &s)) return none();
  if (s != MW_OK) return PyLong_FromLong(s);
  return result({&t.y, &t.mean, &t.rstd});
  END_HANDLE_TH_ERRORS
}

// The gradients of a layer norm into new tensors (of x, weight, bias; the latter two
// where `w` and `b` say so); false: not real ones.  Called without the interpreter lock.
struct NormSizes {
  int64_t rows;
  int C, groups, xt, yt, pt;
  bool w, b;
  std::vector<int64_t> params;  // shape of weight and bias
};
bool norm_gradients(const at::Tensor& dy, const at::Tensor& x, const at::Tensor& mean, const at::Tensor& rstd,
                    const void* weight, const NormSizes& z, c10::DeviceIndex dev,
                    std::array<at::Tensor, 3>* grads, mw_status* s) {
  const size_t bytes = z.w || z.b ? p_norm_bwd_ws(z.rows, z.C, z.groups) : 0;
  const at::TensorOptions options = x.options();
  const at::TensorOptions poptions = options.dtype(z.pt == MW_F32 ? at::kFloat : at::kBFloat16);
  at::Tensor ws;
  if (bytes) ws = scratch(bytes, options);
  (*grads)[0] = at::empty(x.sizes(), options);
  if (z.w) (*grads)[1] = at::empty(z.params, poptions);
  if (z.b) (*grads)[2] = at::empty(z.params, poptions);
  if (bytes && !is_real(ws)) return false;
  for (const at::Tensor& t : *grads)
    if (t.defined() && !is_real(t)) return false;
  *s = p_norm_bwd(dy.const_data_ptr(), x.const_data_ptr(), static_cast<const float*>(mean.const_data_ptr()),
                  static_cast<const float*>(rstd.const_data_ptr()), weight, (*grads)[0].mutable_data_ptr(),
                  z.w ? (*grads)[1].mutable_data_ptr() : nullptr,
                  z.b ? (*grads)[2].mutable_data_ptr() : nullptr, bytes ? ws.mutable_data_ptr() : nullptr,
                  bytes, z.rows, z.C, z.groups, z.xt, z.yt, z.pt,
                  c10::cuda::getCurrentCUDAStream(dev).stream());
  return true;
}

NormSizes norm_sizes(const Norm& t, int yt) {
  const at::Tensor* some = t.w ? t.w : t.b;
  return {t.rows, t.C, t.groups, t.xt, yt, t.pt, t.w != nullptr, t.b != nullptr,
          some ? some->sizes().vec() : std::vector<int64_t>()};
}

// norm_bwd(dy, x, mean, rstd, weight, bias) -> (dx, dweight or None, dbias or None)
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6 || !p_norm_bwd) return none();
  Norm t;
  const at::Tensor *dy = tensor(a[0]), *mean = tensor(a[2]), *rstd = tensor(a[3]);
  c10::DeviceIndex dev;
  if (!t.read(a[1], a[4], a[5]) || !dy || !mean || !rstd || dy->sizes() != t.x->sizes() ||
      !one_device({t.x, dy, mean, rstd}, &dev))
    return none();
  const int yt = norm_type(dy->scalar_type());
  const at::IntArrayRef lead = t.x->sizes().slice(0, t.x->dim() - 1);
  if (yt < 0 || mean->scalar_type() != at::kFloat || rstd->scalar_type() != at::kFloat ||
      mean->sizes() != lead || rstd->sizes() != lead)
    return none();
  const NormSizes z = norm_sizes(t, yt);
  const void* pw = t.w ? t.w->const_data_ptr() : nullptr;
  std::array<at::Tensor, 3> g;
  mw_status s = MW_OK;
  if (!call([&] { return norm_gradients(*dy, *t.x, *mean, *rstd, pw, z, dev, &g, &s); })) return none();
  if (s != MW_OK) return PyLong_FromLong(s);
  return result({&g[0], &g[1], &g[2]});
  END_HANDLE_TH_ERRORS
}

// ---- the same with gradients: nodes of PyTorch's graph, whose backward pass runs
// without the interpreter (a Python function's takes 60 us on the autograd thread,
// more than the kernels of many layers).

using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

// A failed call on the autograd thread, as the Python binding raises it.
[[noreturn]] void raise(mw_status s) {
  const std::string what = p_last_error();
  const PyGILState_STATE gil = PyGILState_Ensure();
  PyObject* e = PyObject_CallFunction(error_type, "is", static_cast<int>(s), what.c_str());
  if (e) PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(e)), e);
  Py_XDECREF(e);
  python_error err;
  err.persist();
  PyGILState_Release(gil);
  throw err;  // NOLINT
}

// The gradient of an output as the kernels read it.
at::Tensor plain_gradient(const at::Tensor& g, const at::Tensor& like, at::ScalarType type) {
  TORCH_CHECK(is_real(g) && g.scalar_type() == type && g.sizes() == like.sizes() && g.device() == like.device(),
              "the gradient must be a plain CUDA tensor like the output");
  return g.contiguous();
}

// A saved tensor as the forward left it: a hook may have put another in its place, and the
// kernels get its address.
void check_saved(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef sizes,
                 c10::DeviceIndex dev) {
  TORCH_CHECK(t.defined() && is_real(t) && t.is_contiguous() && t.scalar_type() == type && t.sizes() == sizes &&
                  t.get_device() == dev,
              "the saved ", name, " is not the plain CUDA tensor that was saved");
}

// Stands behind first derivatives that were asked for with a graph of their own: there is
// no second one, and a gradient without a graph would leave it out silently.
struct NoSecondDerivative : public torch::autograd::Node {
  std::string what;
  std::string name() const override { return "NoSecondDerivative"; }
  variable_list apply(variable_list&&) override { TORCH_CHECK(false, what, " has no second derivative"); }
};

// For gradients that depend on `inputs`, with grad mode as the engine set it.
template <class... T>
void first_only(const char* what, const variable_list& grads, const T&... inputs) {
  if (!torch::autograd::compute_requires_grad(inputs...)) return;
  auto node = std::shared_ptr<NoSecondDerivative>(new NoSecondDerivative(), torch::autograd::deleteNode);
  node->what = what;
  node->set_next_edges(torch::autograd::collect_next_edges(inputs...));
  for (const at::Tensor& g : grads)
    if (g.defined()) torch::autograd::set_history(g, node);
}

struct CrossAttentionBackward : public torch::autograd::Node {
  SavedVariable q, k, v, o, lse, len;
  Shape q_sizes{}, k_sizes{};
  bool lengths = false;
  float scale = 0.f;
  c10::DeviceIndex dev = 0;

  std::string name() const override { return "CrossAttentionBackward"; }
  void release_variables() override {
    for (SavedVariable* s : {&q, &k, &v, &o, &lse, &len}) s->reset_data();
  }
  variable_list apply(variable_list&& grads) override {
    variable_list out(3);
    if (!grads[0].defined()) return out;
    const at::Tensor tq = q.unpack(), tk = k.unpack(), tv = v.unpack(), to = o.unpack(shared_from_this());
    const at::Tensor tl = lse.unpack(), tn = len.unpack();
    gradients(grads[0], tq, tk, tv, to, tl, tn, &out);
    first_only("CrossAttention", out, tq, tk, tv, grads[0]);
    return out;
  }

 private:
  void gradients(const at::Tensor& grad, const at::Tensor& tq, const at::Tensor& tk, const at::Tensor& tv,
                 const at::Tensor& to, const at::Tensor& tl, const at::Tensor& tn, variable_list* out) {
    const at::NoGradGuard no_grad;
    check_saved(tq, "q", at::kBFloat16, q_sizes, dev);
    check_saved(tk, "k", at::kBFloat16, k_sizes, dev);
    check_saved(tv, "v", at::kBFloat16, k_sizes, dev);
    check_saved(to, "o", at::kBFloat16, q_sizes, dev);
    check_saved(tl, "lse", at::kFloat, at::IntArrayRef(q_sizes.data(), 3), dev);
    if (lengths) check_saved(tn, "kv_len", at::kInt, at::IntArrayRef(q_sizes.data(), 1), dev);
    const at::Tensor dout = plain_gradient(grad, tq, at::kBFloat16);
    const int* lens = lengths ? static_cast<const int*>(tn.const_data_ptr()) : nullptr;
    std::array<at::Tensor, 3> g;
    mw_status s = MW_OK;
    TORCH_CHECK(xattn_gradients(tq, tk, tv, lens, to, tl, dout, scale, dev, &g, &s), "no plain CUDA tensors");
    if (s != MW_OK) raise(s);
    for (size_t i = 0; i < 3; ++i)
      if (task_should_compute_output(i)) (*out)[i] = g[i];
  }
};

// A tensor with a forward-mode gradient, which only the Python function refuses.
bool dual(const at::Tensor* t) { return t && t->_fw_grad(0).defined(); }

// xattn_apply(q, k, v, kv_len, scale) -> o
PyObject* xattn_apply(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Xattn x;
  if (n != 5 || !p_xattn || !x.read(a[0], a[1], a[2], a[3], a[4]) || dual(x.q) || dual(x.st.k) || dual(x.st.v))
    return none();
  const at::Tensor &q = *x.q, &k = *x.st.k, &v = *x.st.v;
  mw_status s = MW_OK;
  const bool graph = torch::autograd::compute_requires_grad(q, k, v);
  {
    const at::NoGradGuard no_grad;
    if (!x.forward(graph, &s)) return none();
  }
  if (s != MW_OK) return PyLong_FromLong(s);
  if (graph) {
    auto node = std::shared_ptr<CrossAttentionBackward>(new CrossAttentionBackward(), torch::autograd::deleteNode);
    node->set_next_edges(torch::autograd::collect_next_edges(q, k, v));
    node->q = SavedVariable(q, false);
    node->k = SavedVariable(k, false);
    node->v = SavedVariable(v, false);
    node->lse = SavedVariable(x.lse, false);
    if (x.st.len) node->len = SavedVariable(*x.st.len, false);
    node->lengths = x.st.len != nullptr;
    node->q_sizes = shape(q);
    node->k_sizes = shape(k);
    node->scale = x.scale;
    node->dev = x.dev;
    torch::autograd::set_history(x.o, node);
    node->o = SavedVariable(x.o, true);
  }
  return THPVariable_Wrap(x.o);
  END_HANDLE_TH_ERRORS
}

struct LayerNormBackward : public torch::autograd::Node {
  SavedVariable x, weight, mean, rstd;
  NormSizes z{};
  std::vector<int64_t> sizes;  // of x
  c10::DeviceIndex dev = 0;

  std::string name() const override { return "LayerNormBackward"; }
  void release_variables() override {
    for (SavedVariable* s : {&x, &weight, &mean, &rstd}) s->reset_data();
  }
  variable_list apply(variable_list&& grads) override {
    variable_list out(3);
    if (!grads[0].defined()) return out;
    const at::Tensor tx = x.unpack(), tw = weight.unpack(), tm = mean.unpack(), tr = rstd.unpack();
    gradients(grads[0], tx, tw, tm, tr, &out);
    first_only("LayerNorm", out, tx, tw, grads[0]);
    return out;
  }

 private:
  void gradients(const at::Tensor& grad, const at::Tensor& tx, const at::Tensor& tw, const at::Tensor& tm,
                 const at::Tensor& tr, variable_list* out) {
    const at::NoGradGuard no_grad;
    const at::IntArrayRef lead(sizes.data(), sizes.size() - 1);
    check_saved(tx, "x", torch_type(z.xt), sizes, dev);
    check_saved(tm, "mean", at::kFloat, lead, dev);
    check_saved(tr, "rstd", at::kFloat, lead, dev);
    if (z.w) check_saved(tw, "weight", torch_type(z.pt), z.params, dev);
    const at::Tensor dy = plain_gradient(grad, tx, torch_type(z.yt));
    // (gradients of parameters that nothing asks for are left out)
    NormSizes need = z;
    need.w = z.w && task_should_compute_output(1);
    need.b = z.b && task_should_compute_output(2);
    std::array<at::Tensor, 3> g;
    mw_status s = MW_OK;
    TORCH_CHECK(norm_gradients(dy, tx, tm, tr, z.w ? tw.const_data_ptr() : nullptr, need, dev, &g, &s),
                "no plain CUDA tensors");
    if (s != MW_OK) raise(s);
    for (size_t i = 0; i < 3; ++i)
      if (g[i].defined() && task_should_compute_output(i)) (*out)[i] = g[i];
  }
};

// norm_apply(x, weight, bias, eps, out_dtype) -> y
PyObject* norm_apply(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Norm t;
  float eps;
  int yt;
  if (n != 5 || !p_norm || !t.read(a[0], a[1], a[2]) || !real_number(a[3], &eps) || !t.out_type(a[4], &yt) ||
      dual(t.x) || dual(t.w) || dual(t.b))
    return none();
  const at::Tensor none_given;
  const at::Tensor &x = *t.x, &w = t.w ? *t.w : none_given, &b = t.b ? *t.b : none_given;
  const bool graph = torch::autograd::compute_requires_grad(x, w, b);
  mw_status s = MW_OK;
  {
    const at::NoGradGuard no_grad;
    if (!t.forward(eps, yt, graph, &s)) return none();
  }
  if (s != MW_OK) return PyLong_FromLong(s);
  if (graph) {
    auto node = std::shared_ptr<LayerNormBackward>(new LayerNormBackward(), torch::autograd::deleteNode);
    node->set_next_edges(torch::autograd::collect_next_edges(x, w, b));
    node->x = SavedVariable(x, false);
    if (t.w) node->weight = SavedVariable(w, false);
    node->mean = SavedVariable(t.mean, false);
    node->rstd = SavedVariable(t.rstd, false);
    node->z = norm_sizes(t, yt);
    node->sizes = x.sizes().vec();
    node->dev = t.dev;
    torch::autograd::set_history(t.y, node);
  }
  return THPVariable_Wrap(t.y);
  END_HANDLE_TH_ERRORS
}

#define MW_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef methods[] = {
    {"bind", MW_FAST(bind), "addresses of the C entry points"},
    {"fwd", MW_FAST(fwd), "mw_bca_fwd"},
    {"bwd", MW_FAST(bwd), "mw_bca_bwd"},
    {"cache", MW_FAST(cache), "mw_bca_cache_fwd in its forms, mw_bca_cache_step"},
    {"qkv", MW_FAST(qkv), "mw_qkv_rope_split"},
    {"xattn_fwd", MW_FAST(xattn_fwd), "mw_xattn_fwd"},
    {"xattn_bwd", MW_FAST(xattn_bwd), "mw_xattn_bwd"},
    {"norm_fwd", MW_FAST(norm_fwd), "mw_layernorm_fwd"},
    {"norm_bwd", MW_FAST(norm_bwd), "mw_layernorm_bwd"},
    {"xattn_apply", MW_FAST(xattn_apply), "CrossAttention.apply"},
    {"norm_apply", MW_FAST(norm_apply), "LayerNorm.apply"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mw_torch", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The PyTorch and Python it was built for: it reads their objects' fields through
// their headers, and another version's symbols may resolve all the same.
PyMODINIT_FUNC PyInit__mw_torch(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && (PyModule_AddStringConstant(m, "torch_version", MW_TORCH_VERSION) < 0 ||
            PyModule_AddIntConstant(m, "python_hexversion", PY_VERSION_HEX) < 0)) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
