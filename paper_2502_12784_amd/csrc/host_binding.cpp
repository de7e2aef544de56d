// The host path of the Python entry points for the calls that need nothing unusual: argument checks,
// output allocation and the C-ABI call in one native function per direction (CPython extension
// `_spark_host`, used by binding.py).
//
// Small problems are bound by the host: a training step of 2 heads x 128 tokens took 33 us a pass with its
// marshalling in Python through ctypes (nine tensors checked and six allocated in the interpreter, arguments
// converted one by one), here 18 us with the same three launches, 14.4 us with two and 13.8 us with the allocations
// below (10.7 us of kernels).
//
// Nothing is refused or reported here.  Whatever is not an ordinary call (a wrong shape, type, device or
// layout, a tensor subclass or transform wrapper, an active dispatch mode, a number that is not a plain
// float or int) returns None before anything has been allocated or launched, and binding.py's general
// path, which accepts or raises as documented there, takes the call.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ExpandUtils.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>

#include <limits.h>

#include "../../include/spark_mha.h"

namespace {

enum Kind { SELF = 0, CROSS = 1, STRIDED = 2 };

constexpr c10::DispatchKeySet kWrappers({c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot,
                                         c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                         c10::DispatchKey::Functionalize, c10::DispatchKey::Conjugate,
                                         c10::DispatchKey::Negative, c10::DispatchKey::ZeroTensor});

// An ordinary dense device tensor of dtype `st` and rank `rank`, or nullptr.
const at::Tensor* plain(PyObject* o, int rank) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.dim() != rank) return nullptr;
  if (t.key_set().has_any(kWrappers) || !t.has_storage() || t.unsafeGetTensorImpl()->has_symbolic_sizes_strides())
    return nullptr;
  return &t;
}

bool shaped(const at::Tensor& t, at::ScalarType st, int64_t B, int64_t H, int64_t N, int64_t d, int kind) {
  return t.scalar_type() == st && t.size(0) == B && t.size(1) == H && t.size(2) == N && t.size(3) == d &&
         (kind == STRIDED ? t.stride(3) == 1 : t.is_contiguous());
}

bool stats_shaped(const at::Tensor& t, int64_t B, int64_t H, int64_t N) {
  return t.scalar_type() == at::kFloat && t.size(0) == B && t.size(1) == H && t.size(2) == N && t.is_contiguous();
}

// A contiguous tensor may have any stride in a dimension of size one: those of its sizes are passed then.
spark_strides_t strides(const at::Tensor& t, int kind) {
  if (kind == STRIDED) return spark_strides_t{t.stride(0), t.stride(1), t.stride(2)};
  return spark_strides_t{t.size(1) * t.size(2) * t.size(3), t.size(2) * t.size(3), t.size(3)};
}

// torch._C._cuda_getDevice and torch._C._cuda_getCurrentRawStream, handed over once by bind()
PyObject *get_device = nullptr, *get_raw_stream = nullptr;

// The current stream of the current device; false with a Python error set if torch cannot say.
bool current_stream(void** out) {
  PyObject* dev = PyObject_CallNoArgs(get_device);
  if (!dev) return false;
  PyObject* raw = PyObject_CallOneArg(get_raw_stream, dev);
  Py_DECREF(dev);
  if (!raw) return false;
  *out = PyLong_AsVoidPtr(raw);
  Py_DECREF(raw);
  return !PyErr_Occurred();
}

struct Numbers {
  float scale, p_drop;
  int causal, kind;
  unsigned long long seed;
  unsigned offset;
};

// scale, causal, p_drop, seed, offset, kind
bool numbers(PyObject* const* a, Numbers* n) {
  if (!PyFloat_Check(a[0]) || !PyBool_Check(a[1]) || !PyFloat_Check(a[2]) || !PyLong_Check(a[3]) ||
      !PyLong_Check(a[4]) || !PyLong_Check(a[5]))
    return false;
  n->scale = (float)PyFloat_AS_DOUBLE(a[0]);
  n->causal = a[1] == Py_True;
  n->p_drop = (float)PyFloat_AS_DOUBLE(a[2]);
  n->seed = PyLong_AsUnsignedLongLongMask(a[3]);  // modulo 2^64 and 2^32, as ctypes converts them
  n->offset = (unsigned)PyLong_AsUnsignedLongLongMask(a[4]);
  n->kind = (int)PyLong_AsLong(a[5]);
  return true;
}

bool modes_active() {
  return c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::torch_function_mode_enabled();
}

// Allocations of a call.  With nothing in the thread's dispatch state that wants to see them (a tracer, a transform, a
// profiler) they go to the device's kernel directly: a step of 2 heads x 128 tokens makes six of them, and the way there
// through the dispatcher, and through empty_like's choice of a layout, took 0.6 of its 14.4 us (both ways in alternating
// blocks of one process, whose medians vary by 0.1 us; from process to process a pass varies by 1 us).
class Allocator {
 public:
  explicit Allocator(const at::Tensor& like)
      : direct_((c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty() &&
                !at::hasCallbacks()),
        like_(like) {}
  at::Tensor contiguous(at::IntArrayRef sizes, at::ScalarType st) const {
    if (!direct_) return at::empty(sizes, like_.options().dtype(st));
    return at::_ops::empty_memory_format::redispatch(c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                     c10::fromIntArrayRefSlow(sizes), st, c10::Layout::Strided,
                                                     like_.device(), std::nullopt, std::nullopt);
  }
  // sizes, type, layout and names of `t`, as torch.empty_like
  at::Tensor same(const at::Tensor& t) const {
    if (t.has_names()) return at::empty_like(t);
    int64_t stride = 1;
    for (int i = 3; i >= 0; stride *= t.size(i--))
      if (t.stride(i) != stride || t.size(i) < 1) return at::empty_like(t);
    return contiguous(t.sizes(), t.scalar_type());
  }

  // the same for views, whose layouts empty_like works out in Python-visible steps: its order of the dimensions, without gaps
  // (slices of a packed projection: norm and rotation of one token in eight sequences 6.7 -> 5.9 us a call)
  at::Tensor like(const at::Tensor& t) const {
    if (!direct_ || t.has_names()) return at::empty_like(t);
    const at::IntArrayRef sizes = t.sizes();
    const auto dense = [&](at::IntArrayRef strides) {
      return at::_ops::empty_strided::redispatch(c10::DispatchKeySet(c10::DispatchKey::CUDA), c10::fromIntArrayRefSlow(sizes),
                                                 c10::fromIntArrayRefSlow(strides), t.scalar_type(), c10::Layout::Strided,
                                                 like_.device(), std::nullopt);
    };
    if (t.is_non_overlapping_and_dense()) return dense(t.strides());
    return dense(at::infer_dense_strides(sizes, t.strides()));
  }

 private:
  const bool direct_;
  const at::Tensor& like_;
};

// Sizes of the problem as ints and its dtype; false if they do not fit.
struct Sizes {
  int B, H, Nq, Nk, d;
  spark_dtype_t code;
};
bool sizes(const at::Tensor& Q, const at::Tensor& K, int kind, Sizes* s) {
  for (int i = 0; i < 4; ++i)
    if (Q.size(i) > INT_MAX) return false;
  if (K.size(2) > INT_MAX || (kind == SELF && K.size(2) != Q.size(2))) return false;
  if (Q.scalar_type() != at::kHalf && Q.scalar_type() != at::kBFloat16) return false;
  *s = Sizes{(int)Q.size(0), (int)Q.size(1), (int)Q.size(2), (int)K.size(2), (int)Q.size(3),
             Q.scalar_type() == at::kHalf ? SPARK_F16 : SPARK_BF16};
  return true;
}

// fwd(Q, K, V, O | None, LSE | None, scale, causal, p_drop, seed, offset, kind)
//   -> (O, LSE), a status other than 0, or None (not taken)
PyObject* host_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Numbers x;
  Sizes s;
  if (n != 11 || !get_device || !numbers(a + 5, &x) || modes_active()) Py_RETURN_NONE;
  const at::Tensor *Q = plain(a[0], 4), *K = plain(a[1], 4), *V = plain(a[2], 4);
  if (!Q || !K || !V || !sizes(*Q, *K, x.kind, &s)) Py_RETURN_NONE;
  const at::ScalarType st = Q->scalar_type();
  if (!shaped(*Q, st, s.B, s.H, s.Nq, s.d, x.kind) || !shaped(*K, st, s.B, s.H, s.Nk, s.d, x.kind) ||
      !shaped(*V, st, s.B, s.H, s.Nk, s.d, x.kind))
    Py_RETURN_NONE;
  const at::Tensor* Og = a[3] == Py_None ? nullptr : plain(a[3], 4);
  const at::Tensor* Lg = a[4] == Py_None ? nullptr : plain(a[4], 3);
  if ((a[3] != Py_None && (!Og || !shaped(*Og, st, s.B, s.H, s.Nq, s.d, x.kind))) ||
      (a[4] != Py_None && (!Lg || !stats_shaped(*Lg, s.B, s.H, s.Nq))))
    Py_RETURN_NONE;
  const Allocator fresh(*Q);
  const at::Tensor O = Og ? *Og : fresh.same(*Q);
  const at::Tensor L = Lg ? *Lg : fresh.contiguous({s.B, s.H, s.Nq}, at::kFloat);
  const size_t need = spark_mha_fwd_workspace_bytes(s.B, s.H, s.Nq, s.Nk, s.d, x.causal, s.code);
  at::Tensor ws;
  if (need) ws = fresh.contiguous({(int64_t)need}, at::kByte);
  const void *q = Q->data_ptr(), *k = K->data_ptr(), *v = V->data_ptr();
  void *o = O.data_ptr(), *work = need ? ws.data_ptr() : nullptr;
  float* lse = static_cast<float*>(L.data_ptr());
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  const spark_strides_t sq = strides(*Q, x.kind), sk = strides(*K, x.kind), sv = strides(*V, x.kind),
                        so = strides(O, x.kind);
  rc = spark_mha_workspace_fwd(q, k, v, o, lse, &sq, &sk, &sv, &so, work, need, s.B, s.H, s.Nq, s.Nk, s.d, x.scale,
                               x.causal, x.p_drop, x.seed, x.offset, s.code, stream);
  Py_END_ALLOW_THREADS;
  if (rc != SPARK_OK) return PyLong_FromLong(rc);
  PyObject* out = PyTuple_New(2);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(O));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(L));
  return out;
  END_HANDLE_TH_ERRORS
}

// bwd(Q, K, V, O, LSE, dO, dQ | None, dK | None, dV | None, scale, causal, p_drop, seed, offset, kind)
//   -> (dQ, dK, dV), a status other than 0, or None (not taken)
PyObject* host_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Numbers x;
  Sizes s;
  if (n != 15 || !get_device || !numbers(a + 9, &x) || modes_active()) Py_RETURN_NONE;
  const at::Tensor *Q = plain(a[0], 4), *K = plain(a[1], 4), *V = plain(a[2], 4), *O = plain(a[3], 4),
                   *L = plain(a[4], 3), *dO = plain(a[5], 4);
  if (!Q || !K || !V || !O || !L || !dO || !sizes(*Q, *K, x.kind, &s)) Py_RETURN_NONE;
  const at::ScalarType st = Q->scalar_type();
  auto q_like = [&](const at::Tensor& t) { return shaped(t, st, s.B, s.H, s.Nq, s.d, x.kind); };
  auto k_like = [&](const at::Tensor& t) { return shaped(t, st, s.B, s.H, s.Nk, s.d, x.kind); };
  if (!q_like(*Q) || !q_like(*O) || !q_like(*dO) || !k_like(*K) || !k_like(*V) || !stats_shaped(*L, s.B, s.H, s.Nq))
    Py_RETURN_NONE;
  const at::Tensor* given[3];
  for (int i = 0; i < 3; ++i) {
    given[i] = a[6 + i] == Py_None ? nullptr : plain(a[6 + i], 4);
    if (a[6 + i] != Py_None && (!given[i] || !(i == 0 ? q_like(*given[i]) : k_like(*given[i])))) Py_RETURN_NONE;
  }
  const size_t need = spark_mha_cross_bwd_workspace_bytes(s.B, s.H, s.Nq, s.Nk, s.d, s.code);
  const Allocator fresh(*Q);
  const at::Tensor dQ = given[0] ? *given[0] : fresh.same(*Q), dK = given[1] ? *given[1] : fresh.same(*K),
                   dV = given[2] ? *given[2] : fresh.same(*V);
  const int64_t wbytes = need > 16 ? (int64_t)need : 16;
  const at::Tensor ws = fresh.contiguous({wbytes}, at::kByte);
  const void *q = Q->data_ptr(), *k = K->data_ptr(), *v = V->data_ptr(), *o = O->data_ptr(), *dout = dO->data_ptr();
  const float* lse = static_cast<const float*>(L->data_ptr());
  void *dq = dQ.data_ptr(), *dk = dK.data_ptr(), *dv = dV.data_ptr(), *work = ws.data_ptr();
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  if (x.kind == STRIDED) {
    const int st4 = STRIDED;
    const spark_strides_t sq = strides(*Q, st4), sk = strides(*K, st4), sv = strides(*V, st4), so = strides(*O, st4),
                          sdo = strides(*dO, st4), sdq = strides(dQ, st4), sdk = strides(dK, st4),
                          sdv = strides(dV, st4);
    rc = spark_mha_strided_bwd(q, k, v, o, lse, dout, dq, dk, dv, &sq, &sk, &sv, &so, &sdo, &sdq, &sdk, &sdv, work,
                               (size_t)wbytes, s.B, s.H, s.Nq, s.Nk, s.d, x.scale, x.causal, x.p_drop, x.seed, x.offset,
                               s.code, stream);
  } else {
    rc = spark_mha_dropout_bwd(q, k, v, o, lse, dout, dq, dk, dv, work, (size_t)wbytes, s.B, s.H, s.Nq, s.Nk, s.d,
                               x.scale, x.causal, x.p_drop, x.seed, x.offset, s.code, stream);
  }
  Py_END_ALLOW_THREADS;
  if (rc != SPARK_OK) return PyLong_FromLong(rc);
  PyObject* out = PyTuple_New(3);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(dQ));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(dK));
  PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(dV));
  return out;
  END_HANDLE_TH_ERRORS
}

// ---- the operators around a decoder's attention ----

// The current device and its stream; false with a Python error set if torch cannot say.
struct Here {
  void* stream;
  long device;
};
bool here(Here* h) {
  PyObject* dev = PyObject_CallNoArgs(get_device);
  if (!dev) return false;
  h->device = PyLong_AsLong(dev);
  PyObject* raw = PyObject_CallOneArg(get_raw_stream, dev);
  Py_DECREF(dev);
  if (!raw) return false;
  h->stream = PyLong_AsVoidPtr(raw);
  Py_DECREF(raw);
  return !PyErr_Occurred();
}

// Arguments of one call as they are checked: everything ordinary, on the current device, so far.
class Arguments {
 public:
  explicit Arguments(long device) : device_(device) {}
  bool ok = true;
  // a tensor of this rank, or nullptr
  const at::Tensor* tensor(PyObject* o, int rank) {
    const at::Tensor* t = plain(o, rank);
    if (!t || t->device().index() != device_) ok = false;
    return ok ? t : nullptr;
  }
  const at::Tensor* view(PyObject* o, at::ScalarType st, int64_t a, int64_t b, int64_t n, int64_t d) {
    const at::Tensor* t = tensor(o, 4);
    if (ok && !(t->scalar_type() == st && t->size(0) == a && t->size(1) == b && t->size(2) == n && t->size(3) == d &&
                t->stride(3) == 1))
      ok = false;
    return ok ? t : nullptr;
  }
  const at::Tensor* dense(PyObject* o, at::ScalarType st, at::IntArrayRef sizes) {
    const at::Tensor* t = tensor(o, (int)sizes.size());
    if (ok && !(t->scalar_type() == st && t->sizes() == sizes && t->is_contiguous())) ok = false;
    return ok ? t : nullptr;
  }
  const at::Tensor* given(PyObject* o, at::ScalarType st, int64_t a, int64_t b, int64_t n, int64_t d) {
    return o == Py_None ? nullptr : view(o, st, a, b, n, d);
  }
  // address of an optional [a] or [a, b] tensor of int32
  const int* lengths(PyObject* o, at::IntArrayRef sizes) {
    if (o == Py_None) return nullptr;
    const at::Tensor* t = dense(o, at::kInt, sizes);
    return ok ? static_cast<const int*>(t->data_ptr()) : nullptr;
  }

 private:
  const long device_;
};
spark_strides_t of(const at::Tensor& t) { return spark_strides_t{t.stride(0), t.stride(1), t.stride(2)}; }
bool fits(const at::Tensor& t) {
  for (int i = 0; i < (int)t.dim(); ++i)
    if (t.size(i) > INT_MAX) return false;
  return true;
}
PyObject* result(std::initializer_list<at::Tensor> list) {
  PyObject* out = PyTuple_New((Py_ssize_t)list.size());
  if (!out) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& t : list) PyTuple_SET_ITEM(out, i++, THPVariable_Wrap(t));
  return out;
}
bool half_type(at::ScalarType st) { return st == at::kHalf || st == at::kBFloat16; }

// What both directions of the norm and rotation share: Q, K, wq | None, wk | None, cos | None, sin | None,
// positions | None, eps, interleaved (in two places of the argument list).
struct QkCall {
  const at::Tensor *Q, *K;
  const void *wq = nullptr, *wk = nullptr;
  const float *cos = nullptr, *sin = nullptr;
  const int* positions;
  at::ScalarType st;
  spark_dtype_t code;
  int B, H, N, d, Hkv, rd = 0, table = 0, fp32 = 0, interleaved;
  float eps;
};
bool qk_call(Arguments& args, PyObject* const* a, PyObject* positions, PyObject* eps, PyObject* interleaved, QkCall* c) {
  if (!PyFloat_Check(eps) || !PyBool_Check(interleaved)) return false;
  c->Q = args.tensor(a[0], 4);
  c->K = args.tensor(a[1], 4);
  if (!args.ok || !fits(*c->Q) || !fits(*c->K) || !half_type(c->Q->scalar_type())) return false;
  c->st = c->Q->scalar_type();
  c->code = c->st == at::kHalf ? SPARK_F16 : SPARK_BF16;
  c->B = (int)c->Q->size(0); c->H = (int)c->Q->size(1); c->N = (int)c->Q->size(2); c->d = (int)c->Q->size(3);
  c->Hkv = (int)c->K->size(1);
  args.view(a[0], c->st, c->B, c->H, c->N, c->d);
  args.view(a[1], c->st, c->B, c->Hkv, c->N, c->d);
  const at::ScalarType wt[2] = {at::kFloat, c->st};
  at::ScalarType seen = at::kFloat;
  for (int i = 0; i < 2 && args.ok; ++i) {
    if (a[2 + i] == Py_None) continue;
    const at::Tensor* w = args.tensor(a[2 + i], 1);
    if (!args.ok || w->size(0) != c->d || !w->is_contiguous()) return false;
    if (w->scalar_type() != wt[0] && w->scalar_type() != wt[1]) return false;
    if ((c->wq || c->wk) && w->scalar_type() != seen) return false;
    seen = w->scalar_type();
    c->fp32 = seen == at::kFloat;
    (i ? c->wk : c->wq) = w->data_ptr();
  }
  if (!args.ok || (a[4] == Py_None) != (a[5] == Py_None)) return false;
  if (a[4] != Py_None) {
    const at::Tensor *x = args.tensor(a[4], 2), *y = args.tensor(a[5], 2);
    if (!args.ok || x->scalar_type() != at::kFloat || y->scalar_type() != at::kFloat || !x->is_contiguous() ||
        !y->is_contiguous() || x->sizes() != y->sizes() || !fits(*x) || x->size(1) > 64)
      return false;
    c->table = (int)x->size(0);
    c->rd = 2 * (int)x->size(1);
    c->cos = static_cast<const float*>(x->data_ptr());
    c->sin = static_cast<const float*>(y->data_ptr());
  }
  c->positions = args.lengths(positions, {c->B, c->N});
  c->eps = (float)PyFloat_AS_DOUBLE(eps);
  c->interleaved = interleaved == Py_True;
  return args.ok;
}

// qk_fwd(Q, K, wq, wk, cos, sin, positions, eps, interleaved, Qr | None, Kr | None)
PyObject* host_qk_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Here h;
  QkCall c;
  if (n != 11 || !get_device || modes_active() || !plain(a[0], 4)) Py_RETURN_NONE;
  if (!here(&h)) return nullptr;
  Arguments args(h.device);
  if (!qk_call(args, a, a[6], a[7], a[8], &c)) Py_RETURN_NONE;
  const at::Tensor *Qr = args.given(a[9], c.st, c.B, c.H, c.N, c.d), *Kr = args.given(a[10], c.st, c.B, c.Hkv, c.N, c.d);
  if (!args.ok) Py_RETURN_NONE;
  const Allocator fresh(*c.Q);
  const at::Tensor q = Qr ? *Qr : fresh.like(*c.Q), k = Kr ? *Kr : fresh.like(*c.K);
  void *qp = q.data_ptr(), *kp = k.data_ptr();
  const void *Qp = c.Q->data_ptr(), *Kp = c.K->data_ptr();
  const spark_strides_t sQ = of(*c.Q), sK = of(*c.K), sq = of(q), sk = of(k);
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = spark_qk_norm_rope_fwd(Qp, Kp, c.wq, c.wk, c.cos, c.sin, c.positions, qp, kp, &sQ, &sK, &sq, &sk, c.B, c.N, c.H, c.Hkv,
                              c.d, c.rd, c.table, c.eps, c.interleaved, c.fp32, c.code, h.stream);
  Py_END_ALLOW_THREADS;
  if (rc != SPARK_OK) return PyLong_FromLong(rc);
  return result({q, k});
  END_HANDLE_TH_ERRORS
}

// qk_bwd(Q, K, wq, wk, cos, sin, dQr, dKr, positions, eps, interleaved, dQ | None, dK | None, dwq | None, dwk | None)
PyObject* host_qk_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Here h;
  QkCall c;
  if (n != 15 || !get_device || modes_active() || !plain(a[0], 4)) Py_RETURN_NONE;
  if (!here(&h)) return nullptr;
  Arguments args(h.device);
  if (!qk_call(args, a, a[8], a[9], a[10], &c)) Py_RETURN_NONE;
  const at::Tensor *gq = args.view(a[6], c.st, c.B, c.H, c.N, c.d), *gk = args.view(a[7], c.st, c.B, c.Hkv, c.N, c.d);
  const at::Tensor *dQg = args.given(a[11], c.st, c.B, c.H, c.N, c.d), *dKg = args.given(a[12], c.st, c.B, c.Hkv, c.N, c.d);
  const at::Tensor* dwg[2];
  for (int i = 0; i < 2; ++i) dwg[i] = a[13 + i] == Py_None ? nullptr : args.dense(a[13 + i], at::kFloat, {c.d});
  if (!args.ok) Py_RETURN_NONE;
  const Allocator fresh(*c.Q);
  const at::Tensor dQ = dQg ? *dQg : fresh.like(*c.Q), dK = dKg ? *dKg : fresh.like(*c.K);
  const at::Tensor dwq = dwg[0] ? *dwg[0] : fresh.contiguous({c.d}, at::kFloat),
                   dwk = dwg[1] ? *dwg[1] : fresh.contiguous({c.d}, at::kFloat);
  const size_t need = spark_qk_norm_rope_bwd_workspace_bytes(c.B, c.N, c.H, c.Hkv, c.d, c.rd, c.code);
  const at::Tensor ws = fresh.contiguous({(int64_t)(need > 16 ? need : 16)}, at::kByte);
  const void *Qp = c.Q->data_ptr(), *Kp = c.K->data_ptr(), *gqp = gq->data_ptr(), *gkp = gk->data_ptr();
  void *dQp = dQ.data_ptr(), *dKp = dK.data_ptr(), *wsp = ws.data_ptr();
  float *dwqp = static_cast<float*>(dwq.data_ptr()), *dwkp = static_cast<float*>(dwk.data_ptr());
  const spark_strides_t sQ = of(*c.Q), sK = of(*c.K), sgq = of(*gq), sgk = of(*gk), sdq = of(dQ), sdk = of(dK);
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = spark_qk_norm_rope_bwd(Qp, Kp, c.wq, c.wk, c.cos, c.sin, c.positions, gqp, gkp, dQp, dKp, dwqp, dwkp, &sQ, &sK, &sgq,
                              &sgk, &sdq, &sdk, wsp, need, c.B, c.N, c.H, c.Hkv, c.d, c.rd, c.table, c.eps, c.interleaved,
                              c.fp32, c.code, h.stream);
  Py_END_ALLOW_THREADS;
  if (rc != SPARK_OK) return PyLong_FromLong(rc);
  return result({dQ, dK, dwq, dwk});
  END_HANDLE_TH_ERRORS
}

// What both directions of the attention behind a prefix share.
struct PrefixCall {
  const at::Tensor* x[5];  // Q, Kp, Vp, Ks, Vs
  at::ScalarType st;
  spark_dtype_t code;
  int G, B, H, Hkv, Nq, P, S, d, causal;
  float scale;
  const int *prefix_lens, *q_lens, *s_lens;
  spark_strides_t s[5];
  const void* p[5];
};
// x: Q, Kp, Vp, Ks, Vs;  how: scale, causal, prefix_lens | None, q_lens | None, s_lens | None
bool prefix_call(Arguments& args, PyObject* const* x, PyObject* const* how, PrefixCall* c) {
  if (!PyFloat_Check(how[0]) || !PyBool_Check(how[1])) return false;
  for (int i = 0; i < 5; ++i) {
    c->x[i] = args.tensor(x[i], 4);
    if (!args.ok || !fits(*c->x[i])) return false;
  }
  c->st = c->x[0]->scalar_type();
  if (!half_type(c->st)) return false;
  c->code = c->st == at::kHalf ? SPARK_F16 : SPARK_BF16;
  c->B = (int)c->x[0]->size(0); c->H = (int)c->x[0]->size(1); c->Nq = (int)c->x[0]->size(2); c->d = (int)c->x[0]->size(3);
  c->G = (int)c->x[1]->size(0); c->Hkv = (int)c->x[1]->size(1); c->P = (int)c->x[1]->size(2); c->S = (int)c->x[3]->size(2);
  args.view(x[0], c->st, c->B, c->H, c->Nq, c->d);
  args.view(x[1], c->st, c->G, c->Hkv, c->P, c->d);
  args.view(x[2], c->st, c->G, c->Hkv, c->P, c->d);
  args.view(x[3], c->st, c->B, c->Hkv, c->S, c->d);
  args.view(x[4], c->st, c->B, c->Hkv, c->S, c->d);
  c->prefix_lens = args.lengths(how[2], {c->G});
  c->q_lens = args.lengths(how[3], {c->B});
  c->s_lens = args.lengths(how[4], {c->B});
  if (!args.ok) return false;
  c->scale = (float)PyFloat_AS_DOUBLE(how[0]);
  c->causal = how[1] == Py_True;
  for (int i = 0; i < 5; ++i) {
    c->s[i] = of(*c->x[i]);
    c->p[i] = c->x[i]->data_ptr();
  }
  return true;
}

// prefix_fwd(Q, Kp, Vp, Ks, Vs, scale, causal, prefix_lens, q_lens, s_lens, O | None, LSE | None)
PyObject* host_prefix_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Here h;
  PrefixCall c;
  if (n != 12 || !get_device || modes_active() || !plain(a[0], 4)) Py_RETURN_NONE;
  if (!here(&h)) return nullptr;
  Arguments args(h.device);
  if (!prefix_call(args, a, a + 5, &c)) Py_RETURN_NONE;
  const at::Tensor* Og = args.given(a[10], c.st, c.B, c.H, c.Nq, c.d);
  const at::Tensor* Lg = a[11] == Py_None ? nullptr : args.dense(a[11], at::kFloat, {c.B, c.H, c.Nq});
  if (!args.ok) Py_RETURN_NONE;
  const Allocator fresh(*c.x[0]);
  const at::Tensor O = Og ? *Og : fresh.like(*c.x[0]), L = Lg ? *Lg : fresh.contiguous({c.B, c.H, c.Nq}, at::kFloat);
  const size_t need = spark_mha_prefix_fwd_workspace_bytes(c.G, c.B, c.H, c.Hkv, c.Nq, c.P, c.S, c.d, c.code);
  at::Tensor ws;
  if (need) ws = fresh.contiguous({(int64_t)need}, at::kByte);
  void *o = O.data_ptr(), *wsp = need ? ws.data_ptr() : nullptr;
  float* lse = static_cast<float*>(L.data_ptr());
  const spark_strides_t sO = of(O);
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = spark_mha_prefix_fwd(c.p[0], c.p[1], c.p[2], c.p[3], c.p[4], o, lse, &c.s[0], &c.s[1], &c.s[2], &c.s[3], &c.s[4], &sO,
                            c.prefix_lens, c.q_lens, c.s_lens, wsp, need, c.G, c.B, c.H, c.Hkv, c.Nq, c.P, c.S, c.d, c.scale,
                            c.causal, c.code, h.stream);
  Py_END_ALLOW_THREADS;
  if (rc != SPARK_OK) return PyLong_FromLong(rc);
  return result({O, L});
  END_HANDLE_TH_ERRORS
}

// prefix_bwd(Q, Kp, Vp, Ks, Vs, O, LSE, dO, scale, causal, prefix_lens, q_lens, s_lens, dQ | None, dKp | None, dVp | None,
//            dKs | None, dVs | None)
PyObject* host_prefix_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Here h;
  PrefixCall c;
  if (n != 18 || !get_device || modes_active() || !plain(a[0], 4)) Py_RETURN_NONE;
  if (!here(&h)) return nullptr;
  Arguments args(h.device);
  if (!prefix_call(args, a, a + 8, &c)) Py_RETURN_NONE;
  const at::Tensor *O = args.view(a[5], c.st, c.B, c.H, c.Nq, c.d), *dO = args.view(a[7], c.st, c.B, c.H, c.Nq, c.d);
  const at::Tensor* L = args.dense(a[6], at::kFloat, {c.B, c.H, c.Nq});
  const at::Tensor* given[5];
  for (int i = 0; i < 5; ++i)
    given[i] = !args.ok ? nullptr : args.given(a[13 + i], c.st, c.x[i]->size(0), c.x[i]->size(1), c.x[i]->size(2), c.d);
  if (!args.ok) Py_RETURN_NONE;
  const Allocator fresh(*c.x[0]);
  at::Tensor g[5];
  void* gp[5];
  spark_strides_t gs[5];
  for (int i = 0; i < 5; ++i) {
    g[i] = given[i] ? *given[i] : fresh.like(*c.x[i]);
    gp[i] = g[i].data_ptr();
    gs[i] = of(g[i]);
  }
  const size_t need = spark_mha_prefix_bwd_workspace_bytes(c.G, c.B, c.H, c.Hkv, c.Nq, c.P, c.S, c.d, c.causal, c.code);
  const at::Tensor ws = fresh.contiguous({(int64_t)(need > 16 ? need : 16)}, at::kByte);
  const void *o = O->data_ptr(), *dout = dO->data_ptr();
  const float* lse = static_cast<const float*>(L->data_ptr());
  void* wsp = ws.data_ptr();
  const spark_strides_t sO = of(*O), sdO = of(*dO);
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = spark_mha_prefix_bwd(c.p[0], c.p[1], c.p[2], c.p[3], c.p[4], o, lse, dout, gp[0], gp[1], gp[2], gp[3], gp[4], &c.s[0],
                            &c.s[1], &c.s[2], &c.s[3], &c.s[4], &sO, &sdO, &gs[0], &gs[1], &gs[2], &gs[3], &gs[4],
                            c.prefix_lens, c.q_lens, c.s_lens, wsp, need, c.G, c.B, c.H, c.Hkv, c.Nq, c.P, c.S, c.d, c.scale,
                            c.causal, c.code, h.stream);
  Py_END_ALLOW_THREADS;
  if (rc != SPARK_OK) return PyLong_FromLong(rc);
  return result({g[0], g[1], g[2], g[3], g[4]});
  END_HANDLE_TH_ERRORS
}

// bind(get_device, get_raw_stream)
PyObject* host_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 2 || !PyCallable_Check(a[0]) || !PyCallable_Check(a[1])) {
    PyErr_SetString(PyExc_TypeError, "bind(get_device, get_raw_stream)");
    return nullptr;
  }
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(get_device, a[0]);
  Py_XSETREF(get_raw_stream, a[1]);
  Py_RETURN_NONE;
}

#define SPARK_FASTCALL(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)), METH_FASTCALL
PyMethodDef methods[] = {
    {"bind", SPARK_FASTCALL(host_bind), "the two torch functions that name the current stream"},
    {"fwd", SPARK_FASTCALL(host_fwd), "forward"},
    {"bwd", SPARK_FASTCALL(host_bwd), "backward"},
    {"qk_fwd", SPARK_FASTCALL(host_qk_fwd), "norm and rotation of queries and keys"},
    {"qk_bwd", SPARK_FASTCALL(host_qk_bwd), "its backward"},
    {"prefix_fwd", SPARK_FASTCALL(host_prefix_fwd), "attention behind a shared prefix"},
    {"prefix_bwd", SPARK_FASTCALL(host_prefix_bwd), "its backward"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_spark_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__spark_host() { return PyModule_Create(&module); }
