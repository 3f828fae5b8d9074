// Calls of the block operators from Python without the interpreter's share: a token's rows take the GPU 3 us, and attribute
// by attribute through Python and ctypes a call cost the host 8 to 13 (q/k norms 8.2 and 12.5, row dropout 12, now 2.9, 4.5
// and 3.1). The checks are those of the holders (block.py), made on the tensors themselves. A call that is not exactly in
// order returns None: the holder then goes its ordinary way, which says what is wrong. Otherwise the library's status
// comes back, or the output.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <new>

#include "psppo.h"

namespace {

decltype(&ps_dropout_rows) dropout_rows_fn = nullptr;
decltype(&ps_qk_norm_rope_fwd) qk_fwd_fn = nullptr;
decltype(&ps_qk_norm_rope_bwd) qk_bwd_fn = nullptr;
decltype(&ps_gated_ffn_fwd) ffn_fwd_fn = nullptr;
decltype(&ps_gated_ffn_bwd) ffn_bwd_fn = nullptr;

ps_stream_t stream() { return reinterpret_cast<ps_stream_t>(c10::cuda::getCurrentCUDAStream().stream()); }

// `device`: the one that the call launches on, the current one; a plan's buffers are on it, and so has every tensor to be.
const at::Tensor* tensor(PyObject* o, int device) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.layout() == at::kStrided && t.is_cuda() && t.get_device() == device ? &t : nullptr;
}
int current_device() { return static_cast<int>(c10::cuda::current_device()); }

struct Rows {
  void* at = nullptr;
  int64_t ld = 0;
};
// N rows of cols elements that lie side by side.
bool rows(PyObject* o, int device, int64_t N, int64_t cols, at::ScalarType type, Rows& r) {
  const at::Tensor* t = tensor(o, device);
  if (!t || t->dim() != 2 || t->size(0) != N || t->size(1) != cols || t->scalar_type() != type) return false;
  if (t->stride(1) != 1 && cols > 1 && N > 0) return false;
  r.at = t->data_ptr();
  r.ld = N > 1 ? t->stride(0) : cols;   // (a single row's stride says nothing)
  return true;
}
// n contiguous elements.
bool whole(PyObject* o, int device, int64_t n, at::ScalarType type, const void** at) {
  const at::Tensor* t = tensor(o, device);
  if (!t || t->dim() != 1 || t->size(0) != n || t->scalar_type() != type || !t->is_contiguous()) return false;
  *at = t->data_ptr();
  return true;
}
bool integer(PyObject* o, int64_t& v) {
  if (!PyLong_Check(o)) return false;
  v = PyLong_AsLongLong(o);
  return v != -1 || !PyErr_Occurred();
}

PyObject* ordinary() {
  PyErr_Clear();
  Py_RETURN_NONE;
}
template <class F>
PyObject* guarded(F&& f) {   // (no C++ exception passes into the interpreter)
  try {
    return f();
  } catch (...) {
    return ordinary();
  }
}

// (x, row_traj, row_pos, seed, step, res or None, traj_base, out or None, p, site) -> output, status or None
PyObject* dropout_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10 || !THPVariable_Check(a[0])) return ordinary();
    const int dev = current_device();
    const at::Tensor* x = tensor(a[0], dev);
    if (!x || x->dim() != 2) return ordinary();
    const at::ScalarType type = x->scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat) return ordinary();
    const int64_t N = x->size(0), d = x->size(1);
    Rows rx, rr, ry;
    const void *traj, *pos;
    int64_t step, base, site;
    if (d > INT32_MAX || !rows(a[0], dev, N, d, type, rx) || !whole(a[1], dev, N, at::kInt, &traj) ||
        !whole(a[2], dev, N, at::kInt, &pos) || (a[5] != Py_None && !rows(a[5], dev, N, d, type, rr)) ||
        (a[7] != Py_None && !rows(a[7], dev, N, d, type, ry)) ||
        !PyLong_Check(a[3]) || !integer(a[4], step) || !integer(a[6], base) || !integer(a[9], site) ||
        site != static_cast<int>(site) || step < 0 || !PyFloat_Check(a[8]))
      return ordinary();
    const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[3]);
    PyObject* y = a[7];
    if (y == Py_None) {
      at::Tensor out = at::detail::empty_cuda({N, d}, type, x->device(), std::nullopt);
      ry.at = out.data_ptr();
      ry.ld = d;
      y = THPVariable_Wrap(std::move(out));
      if (!y) return ordinary();
    } else {
      Py_INCREF(y);
    }
    const int rc = dropout_rows_fn(N, static_cast<int>(d), type == at::kFloat ? PS_DTYPE_F32 : PS_DTYPE_BF16, rx.at, rx.ld, rr.at,
                                   rr.ld, static_cast<const int32_t*>(traj), static_cast<const int32_t*>(pos), base,
                                   PyFloat_AS_DOUBLE(a[8]), seed, static_cast<uint64_t>(step), static_cast<int>(site), ry.at, ry.ld,
                                   stream());
    if (rc == PS_OK) return y;
    Py_DECREF(y);
    return PyLong_FromLong(rc);
  });
}

// A plan in a capsule: what stays the same over a holder's calls (the holder keeps the buffers). device: theirs; a plan made
// without one takes no call.
template <class P>
PyObject* capsule(const P& p) {
  P* own = new (std::nothrow) P(p);
  if (!own) return PyErr_NoMemory();
  PyObject* c = PyCapsule_New(own, P::kName, [](PyObject* o) { delete static_cast<P*>(PyCapsule_GetPointer(o, P::kName)); });
  if (!c) delete own;
  return c;
}
// The plan of a call that launches on its device.
template <class P>
const P* plan_of(PyObject* o) {
  const P* p = static_cast<const P*>(PyCapsule_GetPointer(o, P::kName));
  return p && p->device >= 0 && p->device == current_device() ? p : nullptr;
}

struct QkPlan {
  static constexpr char kName[] = "psppo.qk_plan";
  int64_t rows;
  int Hq, Hk, D, R, dtype, layout, T;
  double eps;
  const float* table;
  void *q, *k, *ws, *dq, *dk;
  float *dgq, *dgk;
  size_t ws_bytes;
  int device = -1;
  at::ScalarType type() const { return dtype == PS_DTYPE_F32 ? at::kFloat : at::kBFloat16; }
  int64_t wq() const { return static_cast<int64_t>(Hq) * D; }
  int64_t wk() const { return static_cast<int64_t>(Hk) * D; }
};

PyObject* qk_plan(PyObject*, PyObject* args) {
  QkPlan p;
  unsigned long long ptr[8], ws_bytes;
  long long rows_;
  if (!PyArg_ParseTuple(args, "LiiiiiiidKKKKKKKKK|i", &rows_, &p.Hq, &p.Hk, &p.D, &p.R, &p.dtype, &p.layout, &p.T, &p.eps,
                        &ptr[0], &ptr[1], &ptr[2], &ptr[3], &ws_bytes, &ptr[4], &ptr[5], &ptr[6], &ptr[7], &p.device))
    return nullptr;
  p.rows = rows_;
  p.ws_bytes = static_cast<size_t>(ws_bytes);
  p.table = reinterpret_cast<const float*>(ptr[0]);
  p.q = reinterpret_cast<void*>(ptr[1]);
  p.k = reinterpret_cast<void*>(ptr[2]);
  p.ws = reinterpret_cast<void*>(ptr[3]);
  p.dq = reinterpret_cast<void*>(ptr[4]);
  p.dk = reinterpret_cast<void*>(ptr[5]);
  p.dgq = reinterpret_cast<float*>(ptr[6]);
  p.dgk = reinterpret_cast<float*>(ptr[7]);
  return capsule(p);
}

// The forward's inputs: a[0..5] = q, k, gq, gk (None: 1), pos (None without a rotation), pos_base.
struct QkIn {
  int64_t N;
  Rows q, k;
  const void *gq = nullptr, *gk = nullptr, *pos = nullptr;
  int64_t base;
};
bool qk_inputs(const QkPlan& p, PyObject* const* a, QkIn& in) {
  const int dev = p.device;
  const at::Tensor* q = tensor(a[0], dev);
  if (!q || q->dim() != 2) return false;
  in.N = q->size(0);
  return in.N <= p.rows && rows(a[0], dev, in.N, p.wq(), p.type(), in.q) && rows(a[1], dev, in.N, p.wk(), p.type(), in.k) &&
         (a[2] == Py_None || whole(a[2], dev, p.D, p.type(), &in.gq)) &&
         (a[3] == Py_None || whole(a[3], dev, p.D, p.type(), &in.gk)) &&
         (p.R == 0 || whole(a[4], dev, in.N, at::kInt, &in.pos)) && integer(a[5], in.base) &&
         in.base == static_cast<int>(in.base);
}

// (plan, q, k, gq, gk, pos, pos_base, in_place) -> status or None
PyObject* qk_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const QkPlan* p = n == 8 ? plan_of<QkPlan>(a[0]) : nullptr;
    QkIn in;
    if (!p || !qk_inputs(*p, a + 1, in) || !PyBool_Check(a[7])) return ordinary();
    const bool over = a[7] == Py_True;
    return PyLong_FromLong(qk_fwd_fn(in.N, p->Hq, p->Hk, p->D, p->R, p->dtype, p->layout, in.q.at, in.q.ld, in.k.at, in.k.ld, in.gq,
                                     in.gk, p->eps, static_cast<const int32_t*>(in.pos), static_cast<int>(in.base), p->T, p->table,
                                     over ? in.q.at : p->q, over ? in.q.ld : p->wq(), over ? in.k.at : p->k,
                                     over ? in.k.ld : p->wk(), p->ws, p->ws_bytes, stream()));
  });
}

// (plan, dq_out, dk_out, q, k, gq, gk, pos, pos_base, dw_accumulate) -> status or None
PyObject* qk_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const QkPlan* p = n == 10 ? plan_of<QkPlan>(a[0]) : nullptr;
    QkIn in;
    Rows dq, dk;
    if (!p || !p->dgq || !qk_inputs(*p, a + 3, in) || !rows(a[1], p->device, in.N, p->wq(), p->type(), dq) ||
        !rows(a[2], p->device, in.N, p->wk(), p->type(), dk) || !PyBool_Check(a[9]))
      return ordinary();
    return PyLong_FromLong(qk_bwd_fn(in.N, p->Hq, p->Hk, p->D, p->R, p->dtype, p->layout, dq.at, dq.ld, dk.at, dk.ld, in.q.at, in.q.ld,
                                     in.k.at, in.k.ld, in.gq, in.gk, p->eps, static_cast<const int32_t*>(in.pos),
                                     static_cast<int>(in.base), p->T, p->table, p->dq, p->wq(), p->dk, p->wk(), p->dgq, p->dgk,
                                     a[9] == Py_True ? PS_DW_ACCUMULATE : 0, p->ws, p->ws_bytes, stream()));
  });
}

struct FfnPlan {
  static constexpr char kName[] = "psppo.ffn_plan";
  int64_t rows;
  int d, F, act, dx_dtype, dw_dtype;
  void *Y, *store, *ws_fwd, *ws_bwd, *dX, *dWg, *dWu, *dWd;
  size_t store_bytes, ws_fwd_bytes, ws_bwd_bytes;
  int device = -1;
};

PyObject* ffn_plan(PyObject*, PyObject* args) {
  FfnPlan p;
  unsigned long long v[11];
  long long rows_;
  if (!PyArg_ParseTuple(args, "LiiiiiKKKKKKKKKKK|i", &rows_, &p.d, &p.F, &p.act, &p.dx_dtype, &p.dw_dtype, &v[0], &v[1], &v[2],
                        &v[3], &v[4], &v[5], &v[6], &v[7], &v[8], &v[9], &v[10], &p.device))
    return nullptr;
  p.rows = rows_;
  void** const to[8] = {&p.Y, &p.store, &p.ws_fwd, &p.ws_bwd, &p.dX, &p.dWg, &p.dWu, &p.dWd};
  for (int i = 0; i < 8; ++i) *to[i] = reinterpret_cast<void*>(v[i]);
  p.store_bytes = static_cast<size_t>(v[8]);
  p.ws_fwd_bytes = static_cast<size_t>(v[9]);
  p.ws_bwd_bytes = static_cast<size_t>(v[10]);
  return capsule(p);
}

// a[0..3] = X, Wg, Wu, Wd.
struct FfnIn {
  int64_t N;
  Rows X;
  const void* w[3];
};
bool ffn_inputs(const FfnPlan& p, PyObject* const* a, FfnIn& in) {
  const at::Tensor* X = tensor(a[0], p.device);
  if (!X || X->dim() != 2) return false;
  in.N = X->size(0);
  if (in.N > p.rows || !rows(a[0], p.device, in.N, p.d, at::kBFloat16, in.X)) return false;
  for (int i = 0; i < 3; ++i) {
    const at::Tensor* w = tensor(a[1 + i], p.device);
    if (!w || w->dim() != 2 || w->size(0) != (i < 2 ? p.F : p.d) || w->size(1) != (i < 2 ? p.d : p.F) ||
        w->scalar_type() != at::kBFloat16 || !w->is_contiguous())
      return false;
    in.w[i] = w->data_ptr();
  }
  return true;
}

// (plan, X, Wg, Wu, Wd, out or None) -> status or None
PyObject* ffn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const FfnPlan* p = n == 6 ? plan_of<FfnPlan>(a[0]) : nullptr;
    FfnIn in;
    Rows Y;
    if (!p || !ffn_inputs(*p, a + 1, in)) return ordinary();
    if (a[5] == Py_None) {
      Y.at = p->Y;
      Y.ld = p->d;
    } else if (!rows(a[5], p->device, in.N, p->d, at::kBFloat16, Y)) {
      return ordinary();
    }
    return PyLong_FromLong(ffn_fwd_fn(in.N, p->d, p->F, PS_DTYPE_BF16, p->act, in.X.at, in.X.ld, in.w[0], in.w[1], in.w[2], Y.at,
                                      Y.ld, p->store, p->store_bytes, p->ws_fwd, p->ws_fwd_bytes, stream()));
  });
}

// (plan, dY, X, Wg, Wu, Wd, dw_accumulate) -> status or None
PyObject* ffn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const FfnPlan* p = n == 7 ? plan_of<FfnPlan>(a[0]) : nullptr;
    FfnIn in;
    Rows dY;
    if (!p || !p->store || !ffn_inputs(*p, a + 2, in) || !rows(a[1], p->device, in.N, p->d, at::kBFloat16, dY) ||
        !PyBool_Check(a[6]))
      return ordinary();
    return PyLong_FromLong(ffn_bwd_fn(in.N, p->d, p->F, PS_DTYPE_BF16, dY.at, dY.ld, in.X.at, in.X.ld, in.w[0], in.w[1], in.w[2],
                                      p->store, p->store_bytes, p->dX, p->d, p->dx_dtype, p->dWg, p->dWu, p->dWd, p->dw_dtype,
                                      a[6] == Py_True ? PS_DW_ACCUMULATE : 0, p->ws_bwd, p->ws_bwd_bytes, stream()));
  });
}

// The library's entries (addresses): ps_dropout_rows, ps_qk_norm_rope_fwd and _bwd, ps_gated_ffn_fwd and _bwd.
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long f[5];
  if (!PyArg_ParseTuple(args, "KKKKK", &f[0], &f[1], &f[2], &f[3], &f[4])) return nullptr;
  dropout_rows_fn = reinterpret_cast<decltype(dropout_rows_fn)>(f[0]);
  qk_fwd_fn = reinterpret_cast<decltype(qk_fwd_fn)>(f[1]);
  qk_bwd_fn = reinterpret_cast<decltype(qk_bwd_fn)>(f[2]);
  ffn_fwd_fn = reinterpret_cast<decltype(ffn_fwd_fn)>(f[3]);
  ffn_bwd_fn = reinterpret_cast<decltype(ffn_bwd_fn)>(f[4]);
  Py_RETURN_NONE;
}

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  static PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                                  {"dropout_rows", fast(dropout_rows), METH_FASTCALL, nullptr},
                                  {"qk_plan", qk_plan, METH_VARARGS, nullptr},
                                  {"qk_fwd", fast(qk_fwd), METH_FASTCALL, nullptr},
                                  {"qk_bwd", fast(qk_bwd), METH_FASTCALL, nullptr},
                                  {"ffn_plan", ffn_plan, METH_VARARGS, nullptr},
                                  {"ffn_fwd", fast(ffn_fwd), METH_FASTCALL, nullptr},
                                  {"ffn_bwd", fast(ffn_bwd), METH_FASTCALL, nullptr},
                                  {nullptr, nullptr, 0, nullptr}};
  static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods};
  return PyModule_Create(&module);
}
