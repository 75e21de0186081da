// The binding's ordinary calls as native functions: what a call needs from its tensors is read and its outputs are allocated
// here, without a Python object per step.  A call that spends 2 to 10 us in kernels took 10 to 18 us of host time through
// ctypes and torch.empty (about 1 us per output and 2 to 3 us of argument conversion).  In a loop, us per call, ctypes / so:
// quantizer 64 x 1024 14.1 / 8.4, with a given scale 11.8 / 6.1; one-sided 64 x 512 -> 512 W16A16 10.0 / 6.7, W16A4 14.6 / 11.4;
// dense 16 x 512 -> 512 11.1 / 7.9; host time of a MoE layer's call at one token 16.4 / 12.7.
//
// Every function takes the arguments of the binding's function of that name and returns what it returns, or None for
// arguments that it does not know (tensor subclasses, other types and ranks), which the binding then handles itself.
// The library's status becomes the binding's QuadsError.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/quads.h"

namespace {

// The torch and Python whose inline code this object holds; the binding looks for it in the file before it loads it.
__attribute__((used)) const char g_tag[] = "built for " QUADS_NATIVE_TAG;

PyObject* g_error = nullptr;                               // the binding's exception class
PyObject *s_q, *s_sf, *s_gs, *s_atoms, *s_out, *s_workspace, *s_softmax, *s_sigmoid, *s_dx, *s_dw;

// A plain tensor on a CUDA device, or null.
const at::Tensor* cuda_tensor(PyObject* o) {
  if (!o || !THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() ? &t : nullptr;
}
// The same, or None (`*t` = null).  False: neither.
bool cuda_tensor_or_none(PyObject* o, const at::Tensor** t) {
  *t = nullptr;
  if (o == Py_None) return true;
  *t = cuda_tensor(o);
  return *t != nullptr;
}
const at::Tensor* entry(PyObject* dict, PyObject* key) { return PyDict_CheckExact(dict) ? cuda_tensor(PyDict_GetItem(dict, key)) : nullptr; }
bool small_int(PyObject* o, int32_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long long x = PyLong_AsLongLongAndOverflow(o, &over);
  if (over || x > INT32_MAX || x < INT32_MIN) return false;
  *v = (int32_t)x;
  return true;
}
void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
// Whether somebody wants to know of an allocation, or to fill it: a dispatch mode, a functional transform, a profiler, deterministic algorithms.
bool allocation_is_watched() {
  if (!(c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty() || at::hasCallbacks()) return true;
  const at::Context& c = at::globalContext();
  return c.deterministicAlgorithms() && c.deterministicFillUninitializedMemory();
}
// (where nobody does, without the dispatcher: at::empty takes 0.3 us longer)
at::Tensor alloc(at::IntArrayRef sizes, const at::Tensor& like, at::ScalarType type) {
  if (allocation_is_watched()) return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
  return at::Tensor(at::detail::empty_cuda(sizes, type, like.device(), std::nullopt));
}
at::Tensor alloc_workspace(size_t bytes, const at::Tensor& like) { return alloc({(int64_t)std::max<size_t>(bytes, 256)}, like, at::kByte); }
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// Null, with the binding's exception set, unless `s` is QUADS_OK.
bool passed(quads_status s) {
  if (s == QUADS_OK) return true;
  PyObject* e = PyObject_CallFunction(g_error, "i", (int)s);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return false;
}
template <typename F>
quads_status unlocked(F f) {
  quads_status s;
  Py_BEGIN_ALLOW_THREADS
  s = f();
  Py_END_ALLOW_THREADS
  return s;
}
PyObject* out_and_workspace(PyObject* out, PyObject* ws) {             // takes both references
  PyObject* d = out && ws ? PyDict_New() : nullptr;
  if (d && (PyDict_SetItem(d, s_out, out) < 0 || PyDict_SetItem(d, s_workspace, ws) < 0)) Py_CLEAR(d);
  Py_XDECREF(out);
  Py_XDECREF(ws);
  return d;
}
PyObject* wrapped(const at::Tensor& made, PyObject* given) {           // a new reference to the caller's object, or to a new one
  if (given != Py_None) return Py_NewRef(given);
  return THPVariable_Wrap(made);
}

// (x, gs, sf_layout, out, workspace) -> (q, sf, gs)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int32_t layout;
  const at::Tensor *x, *gs, *ws, *given[3];
  if (n != 5 || !(x = cuda_tensor(a[0])) || !cuda_tensor_or_none(a[1], &gs) || !small_int(a[2], &layout) || !cuda_tensor_or_none(a[4], &ws))
    Py_RETURN_NONE;
  if (x->scalar_type() != at::kBFloat16 || x->dim() != 2 || x->stride(1) != 1 || (layout != QUADS_SF_LINEAR && layout != QUADS_SF_TILED))
    Py_RETURN_NONE;
  const int64_t rows = x->size(0), K = x->size(1);
  at::Tensor made[3], made_ws;
  if (a[3] == Py_None) {
    made[0] = alloc({rows, K / 2}, *x, at::kByte);
    made[1] = layout == QUADS_SF_LINEAR ? alloc({rows, K / 16}, *x, at::kByte) : alloc({(int64_t)quads_sf_tiled_bytes(rows, K)}, *x, at::kByte);
    made[2] = alloc({1}, *x, at::kFloat);
    for (int i = 0; i < 3; ++i) given[i] = &made[i];
  } else {
    if (!PyTuple_CheckExact(a[3]) || PyTuple_GET_SIZE(a[3]) != 3) Py_RETURN_NONE;
    for (int i = 0; i < 3; ++i)
      if (!(given[i] = cuda_tensor(PyTuple_GET_ITEM(a[3], i)))) Py_RETURN_NONE;
  }
  if (!ws) { made_ws = alloc_workspace(quads_quantize_workspace_bytes(), *x); ws = &made_ws; }
  const int64_t ld = rows > 1 ? x->stride(0) : std::max(K, x->stride(0));
  uint8_t *q = (uint8_t*)ptr(given[0]), *sf = (uint8_t*)ptr(given[1]);
  float* g = (float*)ptr(given[2]);
  const void *xp = ptr(x), *gp = ptr(gs);
  void *wp = ptr(ws), *st = stream();
  if (!passed(unlocked([&] { return quads_quantize_nvfp4(xp, rows, K, ld, (const float*)gp, q, sf, g, layout, wp, (size_t)ws->numel(), st); })))
    return nullptr;
  PyObject* r = PyTuple_New(3);
  for (int i = 0; r && i < 3; ++i) {
    PyObject* o = a[3] == Py_None ? THPVariable_Wrap(made[i]) : Py_NewRef(PyTuple_GET_ITEM(a[3], i));
    if (!o) Py_CLEAR(r);
    else PyTuple_SET_ITEM(r, i, o);
  }
  return r;
  END_HANDLE_TH_ERRORS
}

// One dense projection; the arguments of the tensors are in `m` already.
PyObject* run_dense(quads_moe_args& m, const at::Tensor& x, PyObject* ws_obj, const at::Tensor* ws) {
  at::Tensor out = alloc({m.T, m.N}, x, at::kBFloat16), made_ws;
  if (!ws) { made_ws = alloc_workspace(quads_moe_workspace_bytes(m.T, m.H, 0, 1, 1, m.N), x); ws = &made_ws; }
  m.out = out.data_ptr();
  m.workspace = ptr(ws);
  m.workspace_bytes = (size_t)ws->numel();
  void* st = stream();
  if (!passed(unlocked([&] { return quads_moe_w4a4_rac(&m, st); }))) return nullptr;
  return out_and_workspace(THPVariable_Wrap(out), wrapped(made_ws, ws_obj));
}
bool rows_and_width(const at::Tensor& x, quads_moe_args* m) {
  if (x.dim() != 2 || x.size(0) > INT32_MAX || x.size(1) > INT32_MAX) return false;
  m->T = (int32_t)x.size(0);
  m->H = (int32_t)x.size(1);
  m->x = x.data_ptr();
  return true;
}
bool dense_weight(PyObject* w, quads_moe_args* m) {
  const at::Tensor *q = entry(w, s_q), *sf = entry(w, s_sf), *gs = entry(w, s_gs);
  if (!q || !sf || !gs || q->dim() < 2 || q->size(-2) > INT32_MAX) return false;
  m->w13_q = (const uint8_t*)ptr(q); m->w13_sf = (const uint8_t*)ptr(sf); m->w13_gs = (const float*)ptr(gs);
  m->N = (int32_t)q->size(-2);
  return true;
}

// (x, w, nsel, a_gs, workspace) -> dict(out, workspace)
PyObject* dense(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  quads_moe_args m{};
  const at::Tensor *x, *gs, *ws;
  if (n != 5 || !(x = cuda_tensor(a[0])) || !small_int(a[2], &m.rac_nsel_13) || !cuda_tensor_or_none(a[3], &gs) || !cuda_tensor_or_none(a[4], &ws) ||
      !rows_and_width(*x, &m) || !dense_weight(a[1], &m))
    Py_RETURN_NONE;
  m.E = m.topk = 1;
  m.a13_gs = (const float*)ptr(gs);
  return run_dense(m, *x, a[4], ws);
  END_HANDLE_TH_ERRORS
}

// (x, mode, w, w_bf16, a_gs, workspace) -> dict(out, workspace)
PyObject* one_sided(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  quads_moe_args m{};
  const at::Tensor *x, *gs, *ws;
  if (n != 6 || !(x = cuda_tensor(a[0])) || !small_int(a[1], &m.operand_mode) || !cuda_tensor_or_none(a[4], &gs) || !cuda_tensor_or_none(a[5], &ws) ||
      !rows_and_width(*x, &m))
    Py_RETURN_NONE;
  if (m.operand_mode == QUADS_W4A16) {
    if (!dense_weight(a[2], &m)) Py_RETURN_NONE;
  } else if (m.operand_mode == QUADS_W16A4 || m.operand_mode == QUADS_W16A16) {
    const at::Tensor* w = cuda_tensor(a[3]);
    if (!w || w->dim() < 1 || w->size(0) > INT32_MAX) Py_RETURN_NONE;
    m.N = (int32_t)w->size(0);
    m.w13_bf16 = ptr(w);
    if (m.operand_mode == QUADS_W16A4) m.a13_gs = (const float*)ptr(gs);
  } else {
    Py_RETURN_NONE;
  }
  m.E = m.topk = 1;
  return run_dense(m, *x, a[5], ws);
  END_HANDLE_TH_ERRORS
}

// On the current device, whose stream takes the launch; of this type, rank and shape; rows contiguous.
bool is_here(const at::Tensor& t) { return t.device().index() == c10::cuda::current_device(); }
bool is_matrix(const at::Tensor& t, at::ScalarType type, int64_t rows, int64_t cols) {
  return t.dim() == 2 && t.scalar_type() == type && t.size(0) == rows && t.size(1) == cols && (cols <= 1 || t.stride(1) == 1) && is_here(t);
}
bool is_plain_matrix(const at::Tensor& t, at::ScalarType type, int64_t rows, int64_t cols) {
  return is_matrix(t, type, rows, cols) && t.is_contiguous();
}
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
// Logits [T, E] or, with None in their place, a tuple (ids, weights) [T, topk]; E of the logits or of the weights `q`.
struct Routing { int32_t E; const float *logits, *w; const int32_t* ids; };
bool read_routing(PyObject* logits, PyObject* routing, const at::Tensor* q, int64_t T, int32_t topk, Routing* r) {
  *r = Routing{};
  if (routing == Py_None) {
    const at::Tensor* lg = cuda_tensor(logits);
    if (!lg || lg->dim() < 2 || lg->size(1) > INT32_MAX || !is_here(*lg)) return false;
    r->E = (int32_t)lg->size(1);
    r->logits = (const float*)ptr(lg);
    return true;
  }
  if (logits != Py_None || !PyTuple_CheckExact(routing) || PyTuple_GET_SIZE(routing) != 2 || !q || q->dim() < 3 || q->size(0) > INT32_MAX) return false;
  const at::Tensor *ids = cuda_tensor(PyTuple_GET_ITEM(routing, 0)), *w = cuda_tensor(PyTuple_GET_ITEM(routing, 1));
  if (!ids || !w || !is_plain_matrix(*ids, at::kInt, T, topk) || !is_plain_matrix(*w, at::kFloat, T, topk)) return false;
  r->E = (int32_t)q->size(0);
  r->ids = (const int32_t*)ptr(ids);
  r->w = (const float*)ptr(w);
  return true;
}

// (x, logits, w13, w2, topk, nsel13, nsel2, a2_gs, a13_gs, renormalize, workspace, out, routing) -> dict(out, workspace)
PyObject* moe(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  quads_moe_args m{};
  const at::Tensor *x, *a2, *a13, *ws, *out;
  if (n != 13 || !(x = cuda_tensor(a[0])) || !small_int(a[4], &m.topk) || !small_int(a[5], &m.rac_nsel_13) ||
      !small_int(a[6], &m.rac_nsel_2) || !cuda_tensor_or_none(a[7], &a2) || !cuda_tensor_or_none(a[8], &a13) || !cuda_tensor_or_none(a[10], &ws) ||
      !cuda_tensor_or_none(a[11], &out) || !rows_and_width(*x, &m))
    Py_RETURN_NONE;
  const at::Tensor *q1 = entry(a[2], s_q), *f1 = entry(a[2], s_sf), *g1 = entry(a[2], s_gs);
  const at::Tensor *q2 = entry(a[3], s_q), *f2 = entry(a[3], s_sf), *g2 = entry(a[3], s_gs);
  Routing rt;
  if (!q1 || !f1 || !g1 || !q2 || !f2 || !g2 || q2->dim() < 3 || q2->size(2) > INT32_MAX / 2 || !read_routing(a[1], a[12], q1, m.T, m.topk, &rt) ||
      !is_here(*x) || !is_here(*q1) || !is_here(*q2))
    Py_RETURN_NONE;
  const int renorm = PyObject_IsTrue(a[9]);
  if (renorm < 0) return nullptr;
  m.E = rt.E;
  m.I = (int32_t)q2->size(2) * 2;
  m.router_logits = rt.logits; m.topk_ids_in = rt.ids; m.topk_w_in = rt.w;
  m.w13_q = (const uint8_t*)ptr(q1); m.w13_sf = (const uint8_t*)ptr(f1); m.w13_gs = (const float*)ptr(g1);
  m.w2_q = (const uint8_t*)ptr(q2); m.w2_sf = (const uint8_t*)ptr(f2); m.w2_gs = (const float*)ptr(g2);
  m.a13_gs = (const float*)ptr(a13); m.a2_gs = (const float*)ptr(a2);
  m.renormalize = renorm;
  at::Tensor made_out, made_ws;
  if (!out) { made_out = alloc({m.T, m.H}, *x, at::kBFloat16); out = &made_out; }
  if (!ws) { made_ws = alloc_workspace(quads_moe_workspace_bytes(m.T, m.H, m.I, m.E, m.topk, 0), *x); ws = &made_ws; }
  m.out = ptr(out);
  m.workspace = ptr(ws);
  m.workspace_bytes = (size_t)ws->numel();
  void* st = stream();
  if (!passed(unlocked([&] { return quads_moe_w4a4_rac(&m, st); }))) return nullptr;
  return out_and_workspace(wrapped(made_out, a[11]), wrapped(made_ws, a[10]));
  END_HANDLE_TH_ERRORS
}

// (x, logits, w13, w2, topk, renormalize, workspace, out, routing) -> dict(out, workspace)
PyObject* moe_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  quads_moe_fp8_args m{};
  const at::Tensor *x, *ws, *out;
  if (n != 9 || !(x = cuda_tensor(a[0])) || !small_int(a[4], &m.topk) || !cuda_tensor_or_none(a[6], &ws) ||
      !cuda_tensor_or_none(a[7], &out) || x->dim() != 2 || x->size(0) > INT32_MAX || x->size(1) > INT32_MAX)
    Py_RETURN_NONE;
  const at::Tensor *q1 = entry(a[2], s_q), *t1 = entry(a[2], s_atoms), *q2 = entry(a[3], s_q), *t2 = entry(a[3], s_atoms);
  Routing rt;
  if (!q1 || !t1 || !q2 || !t2 || q2->dim() < 3 || q2->size(2) > INT32_MAX || !read_routing(a[1], a[8], q1, x->size(0), m.topk, &rt) || !is_here(*x) ||
      !is_here(*q1) || !is_here(*q2))
    Py_RETURN_NONE;
  const int renorm = PyObject_IsTrue(a[5]);
  if (renorm < 0) return nullptr;
  m.T = (int32_t)x->size(0); m.H = (int32_t)x->size(1); m.I = (int32_t)q2->size(2); m.E = rt.E;
  m.x = ptr(x);
  m.router_logits = rt.logits; m.topk_ids_in = rt.ids; m.topk_w_in = rt.w;
  m.w13_q = (const uint8_t*)ptr(q1); m.w13_atoms = (const uint8_t*)ptr(t1);
  m.w2_q = (const uint8_t*)ptr(q2); m.w2_atoms = (const uint8_t*)ptr(t2);
  m.renormalize = renorm;
  at::Tensor made_out, made_ws;
  if (!out) { made_out = alloc({m.T, m.H}, *x, at::kBFloat16); out = &made_out; }
  if (!ws) { made_ws = alloc_workspace(quads_moe_fp8_workspace_bytes(m.T, m.H, m.I, m.E, m.topk), *x); ws = &made_ws; }
  m.out = ptr(out);
  m.workspace = ptr(ws);
  m.workspace_bytes = (size_t)ws->numel();
  void* st = stream();
  if (!passed(unlocked([&] { return quads_moe_fp8_w8a8(&m, st); }))) return nullptr;
  return out_and_workspace(wrapped(made_out, a[7]), wrapped(made_ws, a[6]));
  END_HANDLE_TH_ERRORS
}

bool float_or_int(PyObject* o, float* v) {
  if (PyFloat_CheckExact(o)) *v = (float)PyFloat_AS_DOUBLE(o);
  else if (PyLong_CheckExact(o)) *v = (float)PyLong_AsDouble(o);
  else return false;
  return !PyErr_Occurred();
}
// logits, topk, score, renormalize and scale into `r`; false: not known here (or, with an exception set, an error)
bool route_args(PyObject* logits, PyObject* score, PyObject* renorm, PyObject* scale, const at::Tensor** lg, quads_route_args* r) {
  if (!(*lg = cuda_tensor(logits)) || !float_or_int(scale, &r->scale)) return false;
  const at::Tensor& l = **lg;
  if (l.dim() != 2 || (l.scalar_type() != at::kFloat && l.scalar_type() != at::kBFloat16) || l.size(0) > INT32_MAX || l.size(1) > INT32_MAX ||
      !is_matrix(l, l.scalar_type(), l.size(0), l.size(1)) || !PyUnicode_CheckExact(score))
    return false;
  if (PyUnicode_Compare(score, s_softmax) == 0) r->score = QUADS_SCORE_SOFTMAX;
  else if (PyUnicode_Compare(score, s_sigmoid) == 0) r->score = QUADS_SCORE_SIGMOID;
  else return false;
  r->renormalize = PyObject_IsTrue(renorm);
  if (r->renormalize < 0) return false;
  r->T = (int32_t)l.size(0); r->E = (int32_t)l.size(1);
  r->logits_bf16 = l.scalar_type() == at::kBFloat16;
  r->logits = l.data_ptr();
  r->ld = row_stride(l);
  return true;
}

// (logits, topk, score, bias, n_group, topk_group, group_top, renormalize, scale) -> (ids, weights)
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  quads_route_args r{};
  const at::Tensor *lg, *bias;
  if (n != 9 || !small_int(a[1], &r.topk) || !cuda_tensor_or_none(a[3], &bias) || !small_int(a[4], &r.n_group) || !small_int(a[5], &r.topk_group) ||
      !small_int(a[6], &r.group_top) || r.topk < 1 || !route_args(a[0], a[2], a[7], a[8], &lg, &r)) {
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
  if (bias && (bias->scalar_type() != at::kFloat || bias->dim() != 1 || bias->size(0) != r.E || !bias->is_contiguous() || !is_here(*bias))) Py_RETURN_NONE;
  r.bias = (const float*)ptr(bias);
  // (a storage each: one that both types share can't be saved together with the other, and keeps both alive)
  at::Tensor ids = alloc({r.T, r.topk}, *lg, at::kInt), w = alloc({r.T, r.topk}, *lg, at::kFloat);
  r.topk_ids = (int32_t*)ids.data_ptr();
  r.topk_w = (float*)w.data_ptr();
  void* st = stream();
  if (!passed(unlocked([&] { return quads_route_experts(&r, st); }))) return nullptr;
  PyObject *o0 = THPVariable_Wrap(ids), *o1 = THPVariable_Wrap(w), *t = o0 && o1 ? PyTuple_Pack(2, o0, o1) : nullptr;
  Py_XDECREF(o0);
  Py_XDECREF(o1);
  return t;
  END_HANDLE_TH_ERRORS
}

// (logits, ids, dweights, score, renormalize, scale) -> dlogits
PyObject* route_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  quads_route_args r{};
  const at::Tensor *lg, *ids, *dw;
  if (n != 6 || !(ids = cuda_tensor(a[1])) || !(dw = cuda_tensor(a[2])) || !route_args(a[0], a[3], a[4], a[5], &lg, &r)) {
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
  if (ids->dim() != 2 || ids->size(1) > INT32_MAX || !is_plain_matrix(*ids, at::kInt, r.T, ids->size(1)) || !is_plain_matrix(*dw, at::kFloat, r.T, ids->size(1)))
    Py_RETURN_NONE;
  r.topk = (int32_t)ids->size(1);
  at::Tensor out = alloc({r.T, r.E}, *lg, lg->scalar_type());
  const int32_t* ip = (const int32_t*)ids->data_ptr();
  const float* dp = (const float*)dw->data_ptr();
  void *op = out.data_ptr(), *st = stream();
  if (!passed(unlocked([&] { return quads_route_experts_backward(&r, ip, dp, op, r.E, st); }))) return nullptr;
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// One weight of fp8_quantize_weights.
struct Fp8Weight { const uint8_t *q, *atoms; int64_t N, K; };
bool fp8_weight(PyObject* w, Fp8Weight* f) {
  const at::Tensor *q = entry(w, s_q), *t = entry(w, s_atoms);
  if (!q || !t || q->dim() < 2 || q->scalar_type() != at::kByte || t->scalar_type() != at::kByte || !q->is_contiguous() || !t->is_contiguous() ||
      !is_here(*q) || !is_here(*t))
    return false;
  f->N = q->size(-2); f->K = q->size(-1);
  if (q->numel() != f->N * f->K || t->numel() != ((f->N + 127) / 128) * ((f->K + 127) / 128) * 512) return false;
  f->q = (const uint8_t*)q->data_ptr(); f->atoms = (const uint8_t*)t->data_ptr();
  return true;
}

// (x, w, workspace, out) -> dict(out, workspace)
PyObject* fp8_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *x, *ws, *out;
  Fp8Weight f;
  if (n != 4 || !(x = cuda_tensor(a[0])) || !fp8_weight(a[1], &f) || !cuda_tensor_or_none(a[2], &ws) || !cuda_tensor_or_none(a[3], &out) || x->dim() != 2 ||
      !is_matrix(*x, at::kBFloat16, x->size(0), f.K) || (ws && !is_here(*ws)) || (out && !is_plain_matrix(*out, at::kBFloat16, x->size(0), f.N)))
    Py_RETURN_NONE;
  const int64_t T = x->size(0), ld = row_stride(*x);
  at::Tensor made_out, made_ws;
  if (!out) { made_out = alloc({T, f.N}, *x, at::kBFloat16); out = &made_out; }
  if (!ws) { made_ws = alloc_workspace(quads_fp8_linear_workspace_bytes(T, f.N, f.K), *x); ws = &made_ws; }
  const void* xp = ptr(x);
  void *op = ptr(out), *wp = ptr(ws), *st = stream();
  const size_t bytes = (size_t)ws->nbytes();
  if (!passed(unlocked([&] { return quads_fp8_linear(xp, T, f.K, ld, f.q, f.atoms, f.N, op, wp, bytes, st); }))) return nullptr;
  return out_and_workspace(wrapped(made_out, a[3]), wrapped(made_ws, a[2]));
  END_HANDLE_TH_ERRORS
}

// (dy, x, w, dw, accumulate, workspace, dx) -> dict(dx, dw, workspace): both gradients
PyObject* fp8_linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *dy, *x, *dw, *ws, *dx;
  Fp8Weight f;
  if (n != 7 || !(dy = cuda_tensor(a[0])) || !(x = cuda_tensor(a[1])) || !fp8_weight(a[2], &f) || !cuda_tensor_or_none(a[3], &dw) ||
      !cuda_tensor_or_none(a[5], &ws) || !cuda_tensor_or_none(a[6], &dx) || dy->dim() != 2)
    Py_RETURN_NONE;
  const int64_t T = dy->size(0);
  const int add = PyObject_IsTrue(a[4]);
  if (add < 0) return nullptr;
  if (!is_matrix(*dy, at::kBFloat16, T, f.N) || !is_matrix(*x, at::kBFloat16, T, f.K) || (dw && !is_plain_matrix(*dw, at::kFloat, f.N, f.K)) || (add && !dw) ||
      (dx && !is_plain_matrix(*dx, at::kBFloat16, T, f.K)) || (ws && !is_here(*ws)))
    Py_RETURN_NONE;
  at::Tensor made_dx, made_dw, made_ws;
  if (!dx) { made_dx = alloc({T, f.K}, *dy, at::kBFloat16); dx = &made_dx; }
  if (!dw) { made_dw = alloc({f.N, f.K}, *dy, at::kFloat); dw = &made_dw; }
  if (!ws) { made_ws = alloc_workspace(quads_fp8_linear_backward_workspace_bytes(T, f.N, f.K), *dy); ws = &made_ws; }
  const int64_t ldy = row_stride(*dy), ldx = row_stride(*x);
  const void *yp = ptr(dy), *xp = ptr(x);
  void *dxp = ptr(dx), *dwp = ptr(dw), *wp = ptr(ws), *st = stream();
  const size_t bytes = (size_t)ws->nbytes();
  if (!passed(unlocked([&] {
        return quads_fp8_linear_backward(yp, ldy, xp, ldx, T, f.N, f.K, f.q, f.atoms, dxp, (float*)dwp, add, wp, bytes, st);
      })))
    return nullptr;
  PyObject *o[3] = {wrapped(made_dx, a[6]), wrapped(made_dw, a[3]), wrapped(made_ws, a[5])}, *keys[3] = {s_dx, s_dw, s_workspace};
  PyObject* d = o[0] && o[1] && o[2] ? PyDict_New() : nullptr;
  for (int i = 0; i < 3; ++i) {
    if (d && PyDict_SetItem(d, keys[i], o[i]) < 0) Py_CLEAR(d);
    Py_XDECREF(o[i]);
  }
  return d;
  END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_XSETREF(g_error, Py_NewRef(cls));
  Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {
    {"set_error", set_error, METH_O, "The exception class raised for a status other than QUADS_OK."},
    {"quantize_nvfp4", (PyCFunction)(void (*)(void))quantize, METH_FASTCALL, nullptr},
    {"dense_w4a4_rac", (PyCFunction)(void (*)(void))dense, METH_FASTCALL, nullptr},
    {"dense_one_sided", (PyCFunction)(void (*)(void))one_sided, METH_FASTCALL, nullptr},
    {"moe_w4a4_rac", (PyCFunction)(void (*)(void))moe, METH_FASTCALL, nullptr},
    {"moe_fp8_w8a8", (PyCFunction)(void (*)(void))moe_fp8, METH_FASTCALL, nullptr},
    {"route_experts", (PyCFunction)(void (*)(void))route, METH_FASTCALL, nullptr},
    {"route_experts_backward", (PyCFunction)(void (*)(void))route_backward, METH_FASTCALL, nullptr},
    {"fp8_linear", (PyCFunction)(void (*)(void))fp8_linear, METH_FASTCALL, nullptr},
    {"fp8_linear_backward", (PyCFunction)(void (*)(void))fp8_linear_backward, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
  s_q = PyUnicode_InternFromString("q"); s_sf = PyUnicode_InternFromString("sf"); s_gs = PyUnicode_InternFromString("gs");
  s_atoms = PyUnicode_InternFromString("atoms"); s_out = PyUnicode_InternFromString("out");
  s_workspace = PyUnicode_InternFromString("workspace");
  s_softmax = PyUnicode_InternFromString("softmax"); s_sigmoid = PyUnicode_InternFromString("sigmoid");
  s_dx = PyUnicode_InternFromString("dx"); s_dw = PyUnicode_InternFromString("dw");
  if (!s_q || !s_sf || !s_gs || !s_atoms || !s_out || !s_workspace || !s_softmax || !s_sigmoid || !s_dx || !s_dw) return nullptr;
  return PyModule_Create(&g_module);
}
