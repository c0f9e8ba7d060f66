// Native argument marshalling for the short calls of api.py: layer norm, its gradient,
// the 8-bit layers, the gated layer, the layers' gradients and a block's end take a few
// microseconds on the device, less than Python needs to check their arguments and
// allocate their outputs.
//
// Each function takes what its namesake in api.py takes, for the ordinary form alone:
// plain tensors on the current device, on the current stream, outputs allocated here.
// Anything else, and any status but GL_OK (nothing was enqueued then), returns None: the
// caller goes through api.py's own checks, which name what is wrong.  No computation
// and no allocation but the outputs' and the workspace's happens here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <dlfcn.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "graphleap.h"

namespace {

decltype(&gl_layer_norm) p_layer_norm;
decltype(&gl_layer_norm_backward) p_layer_norm_backward;
decltype(&gl_layer_norm_backward_workspace_bytes) p_layer_norm_backward_ws;
decltype(&gl_quantize_rows) p_quantize_rows;
decltype(&gl_layer_norm_q8) p_layer_norm_q8;
decltype(&gl_linear_q8) p_linear_q8;
decltype(&gl_gated_linear) p_gated_linear;
decltype(&gl_gated_linear_workspace_bytes) p_gated_linear_ws;
decltype(&gl_linear_backward) p_linear_backward;
decltype(&gl_linear_backward_workspace_bytes) p_linear_backward_ws;
decltype(&gl_gated_linear_backward) p_gated_linear_backward;
decltype(&gl_gated_linear_backward_workspace_bytes) p_gated_linear_backward_ws;
decltype(&gl_residual_norm) p_residual_norm;
decltype(&gl_residual_norm_backward) p_residual_norm_backward;
decltype(&gl_residual_norm_backward_workspace_bytes) p_residual_norm_backward_ws;

// A plain device tensor of the current device; null for anything else.
const at::Tensor* tensor(PyObject* o, int device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.layout() != c10::kStrided || t.get_device() != device || t.is_conj() || t.is_neg())
    return nullptr;
  return &t;
}

bool float_type(const at::Tensor& t, gl_dtype* dt) {
  *dt = t.scalar_type() == at::kBFloat16 ? GL_BF16 : GL_F32;
  return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat;
}

struct Rows {
  const at::Tensor* t;
  long long R, C, ld;
  gl_dtype dt;
};

// Rows over the last axis, a uniform stride apart.
bool rows(PyObject* o, int device, Rows* r) {
  r->t = tensor(o, device);
  if (!r->t || !float_type(*r->t, &r->dt) || r->t->dim() < 1) return false;
  const at::Tensor& t = *r->t;
  r->C = t.size(-1);
  if (r->C < 1 || t.numel() < 1 || t.numel() / r->C > INT_MAX || r->C > INT_MAX) return false;
  r->R = t.numel() / r->C;
  r->ld = r->C;
  if (t.is_contiguous()) return true;
  if (r->C > 1 && t.stride(-1) != 1) return false;
  long long n = 0;  // rows that lie r->ld apart
  for (long long d = t.dim() - 2; d >= 0; --d) {
    if (t.size(d) == 1) continue;
    if (n == 0) {
      r->ld = t.stride(d);
      n = t.size(d);
    } else if (t.stride(d) == r->ld * n) {
      n *= t.size(d);
    } else {
      return false;
    }
  }
  return r->ld >= r->C;
}

// None, or a contiguous tensor of `n` elements of this type in one axis; false otherwise.
bool vec(PyObject* o, int device, at::ScalarType type, long long n, void** p) {
  *p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o, device);
  if (!t || t->scalar_type() != type || t->dim() != 1 || t->size(0) != n || !t->is_contiguous()) return false;
  *p = t->data_ptr();
  return true;
}

// A contiguous tensor of this type whose shape is x's without its last axis.
bool stats(PyObject* o, int device, const at::Tensor& x, const float** p) {
  const at::Tensor* t = tensor(o, device);
  if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous() ||
      t->sizes() != x.sizes().slice(0, x.dim() - 1))
    return false;
  *p = static_cast<const float*>(t->data_ptr());
  return true;
}

int device_now() {
  c10::DeviceIndex d = -1;
  return c10::hip::GetDevice(&d) == hipSuccess ? d : -1;
}
hipStream_t stream_now(int device) { return c10::hip::getCurrentHIPStream(device).stream(); }

at::Tensor empty(at::IntArrayRef shape, const at::Tensor& like, at::ScalarType type) {
  return at::empty(shape, like.options().dtype(type).requires_grad(false));
}

// One of several small outputs: empty(), made by the allocator that `like` came from without
// the dispatcher between.
at::Tensor small(at::IntArrayRef shape, const at::Tensor& like) {
  c10::Allocator* from = like.storage().allocator();
  if (!from) return empty(shape, like, at::kFloat);
  return at::Tensor(at::detail::empty_generic(shape, from, c10::DispatchKeySet(c10::DispatchKey::CUDA), at::kFloat, std::nullopt));
}

// Runs f; a C++ exception becomes torch's Python one.
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

PyObject* none() { Py_RETURN_NONE; }

// An activation or a norm: what does not fit 32 bits is not cut short to one that there is.
bool choice(long v) { return v == (int)v; }

// layer_norm(x, gamma, beta, eps, stats) -> out or (out, mean, rstd)
PyObject* py_layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 5 || !p_layer_norm) return none();
    const int dev = device_now();
    Rows x;
    void *gamma, *beta;
    if (!rows(a[0], dev, &x) || !vec(a[1], dev, x.t->scalar_type(), x.C, &gamma) ||
        !vec(a[2], dev, x.t->scalar_type(), x.C, &beta))
      return none();
    const double eps = PyFloat_AsDouble(a[3]);
    const int want = PyObject_IsTrue(a[4]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out = empty(x.t->sizes(), *x.t, x.t->scalar_type()), mean, rstd;
    if (want) {
      const auto lead = x.t->sizes().slice(0, x.t->dim() - 1);
      mean = empty(lead, *x.t, at::kFloat);
      rstd = empty(lead, *x.t, at::kFloat);
    }
    if (p_layer_norm(x.t->data_ptr(), (int)x.R, (int)x.C, x.ld, gamma, beta, (float)eps, x.dt, out.data_ptr(),
                     want ? static_cast<float*>(mean.data_ptr()) : nullptr,
                     want ? static_cast<float*>(rstd.data_ptr()) : nullptr, stream_now(dev)) != GL_OK)
      return none();
    if (!want) return THPVariable_Wrap(std::move(out));
    return Py_BuildValue("(NNN)", THPVariable_Wrap(std::move(out)), THPVariable_Wrap(std::move(mean)),
                         THPVariable_Wrap(std::move(rstd)));
  });
}

// layer_norm_backward(dy, x, mean, rstd, gamma) -> (dx, dgamma, dbeta)
PyObject* py_layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 5 || !p_layer_norm_backward) return none();
    const int dev = device_now();
    Rows dy, x;
    const float *mean, *rstd;
    void* gamma;
    if (!rows(a[1], dev, &x) || !rows(a[0], dev, &dy) || dy.t->sizes() != x.t->sizes() || dy.dt != x.dt ||
        !stats(a[2], dev, *x.t, &mean) || !stats(a[3], dev, *x.t, &rstd) ||
        !vec(a[4], dev, x.t->scalar_type(), x.C, &gamma))
      return none();
    const size_t bytes = p_layer_norm_backward_ws((int)x.R, (int)x.C, x.dt);
    at::Tensor dx = empty(x.t->sizes(), *x.t, x.t->scalar_type()), dgamma = empty({x.C}, *x.t, at::kFloat),
               dbeta = empty({x.C}, *x.t, at::kFloat), ws;
    if (bytes) ws = empty({(long long)bytes}, *x.t, at::kByte);
    if (p_layer_norm_backward(dy.t->data_ptr(), dy.ld, x.t->data_ptr(), x.ld, (int)x.R, (int)x.C, mean, rstd, gamma,
                              x.dt, dx.data_ptr(), static_cast<float*>(dgamma.data_ptr()),
                              static_cast<float*>(dbeta.data_ptr()), bytes ? ws.data_ptr() : nullptr, bytes,
                              stream_now(dev)) != GL_OK)
      return none();
    return Py_BuildValue("(NNN)", THPVariable_Wrap(std::move(dx)), THPVariable_Wrap(std::move(dgamma)),
                         THPVariable_Wrap(std::move(dbeta)));
  });
}

// The 8-bit rows' tensors (q, scale) of rows x, after `call` wrote them.
template <class F>
PyObject* rows_q8(const Rows& x, F call) {
  if (x.C > GL_MAX_Q8_K) return none();
  const long long kp = (x.C + 15) / 16 * 16;
  c10::SmallVector<int64_t, 5> shape(x.t->sizes().begin(), x.t->sizes().end());
  shape.back() = kp;
  at::Tensor q = empty(shape, *x.t, at::kChar),
             scale = empty(x.t->sizes().slice(0, x.t->dim() - 1), *x.t, at::kFloat);
  if (call(static_cast<int8_t*>(q.data_ptr()), static_cast<float*>(scale.data_ptr())) != GL_OK) return none();
  return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(q)), THPVariable_Wrap(std::move(scale)));
}

// quantize_rows(x) -> (q, scale)
PyObject* py_quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 1 || !p_quantize_rows) return none();
    const int dev = device_now();
    Rows x;
    if (!rows(a[0], dev, &x)) return none();
    return rows_q8(x, [&](int8_t* q, float* s) {
      return p_quantize_rows(x.t->data_ptr(), (int)x.R, (int)x.C, x.ld, x.dt, q, s, stream_now(dev));
    });
  });
}

// layer_norm_q8(x, gamma, beta, eps) -> (q, scale)
PyObject* py_layer_norm_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 4 || !p_layer_norm_q8) return none();
    const int dev = device_now();
    Rows x;
    void *gamma, *beta;
    if (!rows(a[0], dev, &x) || !vec(a[1], dev, x.t->scalar_type(), x.C, &gamma) ||
        !vec(a[2], dev, x.t->scalar_type(), x.C, &beta))
      return none();
    const double eps = PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) return nullptr;
    return rows_q8(x, [&](int8_t* q, float* s) {
      return p_layer_norm_q8(x.t->data_ptr(), (int)x.R, (int)x.C, x.ld, gamma, beta, (float)eps, x.dt, q, s,
                             stream_now(dev));
    });
  });
}

// linear_q8(x.q, x.scale, K, W.q, W.scale, W.K, bias, act_out, residual, bf16) -> out
PyObject* py_linear_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10 || !p_linear_q8) return none();
    const int dev = device_now();
    const at::Tensor *q = tensor(a[0], dev), *w = tensor(a[3], dev);
    const long long K = PyLong_AsLongLong(a[2]), WK = PyLong_AsLongLong(a[5]), act = PyLong_AsLongLong(a[7]);
    const int bf16 = PyObject_IsTrue(a[9]);
    if (PyErr_Occurred()) return nullptr;
    if (!q || !w || K < 1 || K > GL_MAX_Q8_K || K != WK) return none();
    const long long kp = (K + 15) / 16 * 16;
    for (const at::Tensor* t : {q, w})
      if (t->scalar_type() != at::kChar || t->dim() < 1 || !t->is_contiguous() || t->size(-1) != kp || t->numel() < 1 ||
          t->numel() / kp > INT_MAX)
        return none();
    if (w->dim() != 2) return none();
    const long long R = q->numel() / kp, cout = w->size(0);
    const at::ScalarType type = bf16 ? at::kBFloat16 : at::kFloat;
    const float* scale;
    void *w_scale, *bias;
    if (!stats(a[1], dev, *q, &scale) || a[4] == Py_None || !vec(a[4], dev, at::kFloat, cout, &w_scale) ||
        !vec(a[6], dev, type, cout, &bias))
      return none();
    c10::SmallVector<int64_t, 5> shape(q->sizes().begin(), q->sizes().end());
    shape.back() = cout;
    const void* residual = nullptr;
    if (a[8] != Py_None) {
      const at::Tensor* r = tensor(a[8], dev);
      if (!r || r->scalar_type() != type || !r->is_contiguous() || r->sizes() != at::IntArrayRef(shape)) return none();
      residual = r->data_ptr();
    }
    at::Tensor out = empty(shape, *q, type);
    if (p_linear_q8(static_cast<const int8_t*>(q->data_ptr()), scale, (int)R, (int)K,
                    static_cast<const int8_t*>(w->data_ptr()), static_cast<const float*>(w_scale), bias, (int)cout,
                    (gl_act)act, residual, bf16 ? GL_BF16 : GL_F32, out.data_ptr(), stream_now(dev)) != GL_OK)
      return none();
    return THPVariable_Wrap(std::move(out));
  });
}

// x's shape with another last axis
c10::SmallVector<int64_t, 5> with_last(const at::Tensor& x, long long n) {
  c10::SmallVector<int64_t, 5> shape(x.sizes().begin(), x.sizes().end());
  shape.back() = n;
  return shape;
}

// A contiguous tensor of this type and shape.
const at::Tensor* shaped(PyObject* o, int device, at::ScalarType type, at::IntArrayRef shape) {
  const at::Tensor* t = tensor(o, device);
  return t && t->scalar_type() == type && t->sizes() == shape && t->is_contiguous() ? t : nullptr;
}

// A layer's contiguous input rows x and weight W [N, K].
struct Layer {
  const at::Tensor *x, *W;
  int R, K, N;
  gl_dtype dt;
};

bool layer(PyObject* x, PyObject* W, int device, Layer* l) {
  l->x = tensor(x, device), l->W = tensor(W, device);
  if (!l->x || !l->W || !float_type(*l->x, &l->dt) || l->W->scalar_type() != l->x->scalar_type() || l->x->dim() < 1 ||
      l->W->dim() != 2 || !l->x->is_contiguous() || !l->W->is_contiguous() || l->x->numel() < 1 || l->W->numel() < 1)
    return false;
  const long long K = l->x->size(-1), R = l->x->numel() / K, N = l->W->size(0);
  if (l->W->size(1) != K || K > INT_MAX || R > INT_MAX || N > INT_MAX) return false;
  l->R = (int)R, l->K = (int)K, l->N = (int)N;
  return true;
}

PyObject* wrap_or_none(at::Tensor&& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(std::move(t));
}
template <class T = void>
T* ptr(const at::Tensor& t) {
  return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr;
}

// gated_linear(x, W, bias, act, keep) -> h or (h, pre)
PyObject* py_gated_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 5 || !p_gated_linear) return none();
    const int dev = device_now();
    Layer l;
    void* bias;
    if (!layer(a[0], a[1], dev, &l) || l.N % 2 || !vec(a[2], dev, l.x->scalar_type(), l.N, &bias)) return none();
    const long act = PyLong_AsLong(a[3]);
    const int keep = PyObject_IsTrue(a[4]), F = l.N / 2;
    if (PyErr_Occurred()) return nullptr;
    if (!choice(act)) return none();
    const size_t bytes = p_gated_linear_ws(l.R, l.K, F, l.dt);
    at::Tensor h = empty(with_last(*l.x, F), *l.x, l.x->scalar_type()), pre, ws;
    if (keep) pre = empty(with_last(*l.x, l.N), *l.x, l.x->scalar_type());
    if (bytes) ws = empty({(long long)bytes}, *l.x, at::kByte);
    if (p_gated_linear(l.x->data_ptr(), l.R, l.K, l.W->data_ptr(), bias, F, (gl_act)act, l.dt, h.data_ptr(), ptr(pre), ptr(ws),
                       bytes, stream_now(dev)) != GL_OK)
      return none();
    if (!keep) return THPVariable_Wrap(std::move(h));
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(h)), THPVariable_Wrap(std::move(pre)));
  });
}

// linear_backward(dy, x, W, dx, dW, dbias) and gated_linear_backward(dh, x, W, pre, act, dx, dW,
// dbias), the last three whether each is wanted -> (dx, dW, dbias)
PyObject* layer_backward(PyObject* const* a, bool gated) {
  const int dev = device_now();
  Layer l;
  if (!layer(a[1], a[2], dev, &l) || (gated && l.N % 2)) return none();
  const int F = gated ? l.N / 2 : l.N;
  const at::ScalarType type = l.x->scalar_type();
  const at::Tensor* dy = shaped(a[0], dev, type, with_last(*l.x, F));
  const at::Tensor* pre = gated ? shaped(a[3], dev, type, with_last(*l.x, l.N)) : nullptr;
  if (!dy || (gated && !pre)) return none();
  const long act = gated ? PyLong_AsLong(a[4]) : 0;
  PyObject* const* need = a + (gated ? 5 : 3);
  const int wx = PyObject_IsTrue(need[0]), ww = PyObject_IsTrue(need[1]), wb = PyObject_IsTrue(need[2]);
  if (PyErr_Occurred()) return nullptr;
  if (!choice(act)) return none();
  const size_t bytes = gated ? p_gated_linear_backward_ws(l.R, l.K, F, l.dt) : p_linear_backward_ws(l.R, l.K, F, l.dt);
  at::Tensor dx, dW, db, ws;
  if (wx) dx = empty(l.x->sizes(), *l.x, type);
  if (ww) dW = empty(l.W->sizes(), *l.x, type);
  if (wb) db = empty({l.N}, *l.x, at::kFloat);
  if (bytes) ws = empty({(long long)bytes}, *l.x, at::kByte);
  const gl_status s =
      gated ? p_gated_linear_backward(dy->data_ptr(), l.x->data_ptr(), l.R, l.K, l.W->data_ptr(), pre->data_ptr(), F, (gl_act)act,
                                      l.dt, ptr(dx), ptr(dW), ptr<float>(db), ptr(ws), bytes, stream_now(dev))
            : p_linear_backward(dy->data_ptr(), l.x->data_ptr(), l.R, l.K, l.W->data_ptr(), F, l.dt, ptr(dx), ptr(dW),
                                ptr<float>(db), ptr(ws), bytes, stream_now(dev));
  if (s != GL_OK) return none();
  return Py_BuildValue("(NNN)", wrap_or_none(std::move(dx)), wrap_or_none(std::move(dW)), wrap_or_none(std::move(db)));
}

PyObject* py_linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* { return n != 6 || !p_linear_backward ? none() : layer_backward(a, false); });
}
PyObject* py_gated_linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* { return n != 8 || !p_gated_linear_backward ? none() : layer_backward(a, true); });
}

// What residual_norm and its backward pass share: post and norm (a pair or None), scale, gate.
struct Join {
  void *g1 = nullptr, *b1 = nullptr, *g2 = nullptr, *b2 = nullptr, *scale = nullptr;
  const at::Tensor* gate = nullptr;
  bool post, norm;
  int per = 1;
};

bool norm_pair(PyObject* o, int dev, at::ScalarType type, long long C, bool* on, void** gamma, void** beta) {
  *on = o != Py_None;
  if (!*on) return true;
  return PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 2 && vec(PyTuple_GET_ITEM(o, 0), dev, type, C, gamma) &&
         vec(PyTuple_GET_ITEM(o, 1), dev, type, C, beta);
}

bool join_args(const Rows& x, int dev, PyObject* post, PyObject* scale, PyObject* gate, PyObject* norm, Join* j) {
  const at::ScalarType type = x.t->scalar_type();
  if (!norm_pair(post, dev, type, x.C, &j->post, &j->g1, &j->b1) || !norm_pair(norm, dev, type, x.C, &j->norm, &j->g2, &j->b2) ||
      !vec(scale, dev, type, x.C, &j->scale))
    return false;
  if (gate == Py_None) return true;
  j->gate = tensor(gate, dev);
  if (!j->gate || j->gate->scalar_type() != at::kFloat || !j->gate->is_contiguous() || j->gate->dim() < 1 ||
      j->gate->dim() >= x.t->dim() || j->gate->sizes() != x.t->sizes().slice(0, j->gate->dim()))
    return false;
  j->per = (int)(x.R / j->gate->numel());
  return true;
}

const float* gate_of(const Join& j) { return j.gate ? static_cast<const float*>(j.gate->data_ptr()) : nullptr; }

bool same(const Rows& a, const Rows& b) { return a.t->sizes() == b.t->sizes() && a.dt == b.dt; }

// residual_norm(x, b, post, scale, gate, norm, kind, eps, stats) -> (s, y) or (s, y, (the four
// statistics)), None for what there is not
PyObject* py_residual_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 9 || !p_residual_norm) return none();
    const int dev = device_now();
    Rows x, b;
    Join j;
    if (!rows(a[0], dev, &x) || !rows(a[1], dev, &b) || !same(x, b) || !join_args(x, dev, a[2], a[3], a[4], a[5], &j))
      return none();
    const long kind = PyLong_AsLong(a[6]);
    const double eps = PyFloat_AsDouble(a[7]);
    const int want = PyObject_IsTrue(a[8]);
    if (PyErr_Occurred()) return nullptr;
    if (!choice(kind)) return none();
    const at::ScalarType type = x.t->scalar_type();
    at::Tensor s = empty(x.t->sizes(), *x.t, type), y, st[4];
    if (j.norm) y = empty(x.t->sizes(), *x.t, type);
    const bool means = kind == GL_NORM_LAYER, on[4] = {j.post && means, j.post, j.norm && means, j.norm};
    for (int i = 0; i < 4; ++i)
      if (want && on[i]) st[i] = empty(x.t->sizes().slice(0, x.t->dim() - 1), *x.t, at::kFloat);
    if (p_residual_norm(x.t->data_ptr(), x.ld, b.t->data_ptr(), b.ld, (int)x.R, (int)x.C, (gl_norm)kind, (float)eps, j.post, j.g1,
                        j.b1, j.scale, gate_of(j), j.per, j.g2, j.b2, x.dt, s.data_ptr(), ptr(y), ptr<float>(st[0]),
                        ptr<float>(st[1]), ptr<float>(st[2]), ptr<float>(st[3]), stream_now(dev)) != GL_OK)
      return none();
    PyObject *ps = THPVariable_Wrap(std::move(s)), *py = wrap_or_none(std::move(y));
    if (!want) return Py_BuildValue("(NN)", ps, py);
    return Py_BuildValue("(NN(NNNN))", ps, py, wrap_or_none(std::move(st[0])), wrap_or_none(std::move(st[1])),
                         wrap_or_none(std::move(st[2])), wrap_or_none(std::move(st[3])));
  });
}

// residual_norm_backward(ds, dy, b, s, stats, post, scale, gate, norm, kind)
//   -> (dx, db, dgate, dscale, (dpost's two) or None, (dnorm's two) or None)
PyObject* py_residual_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10 || !p_residual_norm_backward) return none();
    const int dev = device_now();
    const bool has_ds = a[0] != Py_None, has_dy = a[1] != Py_None;
    Rows ds{}, dy{}, b, s{};
    Join j;
    if ((!has_ds && !has_dy) || !rows(a[2], dev, &b) || (has_ds && (!rows(a[0], dev, &ds) || !same(ds, b))) ||
        (has_dy && (!rows(a[1], dev, &dy) || !same(dy, b) || !rows(a[3], dev, &s) || !same(s, b))) ||
        !join_args(b, dev, a[5], a[6], a[7], a[8], &j) || j.norm != has_dy)
      return none();
    const long kind = PyLong_AsLong(a[9]);
    if (PyErr_Occurred()) return nullptr;
    if (!choice(kind)) return none();
    const float* st[4] = {};
    const bool means = kind == GL_NORM_LAYER, on[4] = {j.post && means, j.post, j.norm && means, j.norm};
    // (an iterator's tensors would be gone, and their memory the outputs', before the kernel
    // reads them: a tuple or a list holds what it is asked for)
    if (!PyTuple_Check(a[4]) && !PyList_Check(a[4])) return none();
    bool ok = PySequence_Fast_GET_SIZE(a[4]) == 4;
    for (int i = 0; ok && i < 4; ++i)
      if (on[i]) ok = stats(PySequence_Fast_GET_ITEM(a[4], i), dev, *b.t, &st[i]);
    if (!ok) return none();
    const at::ScalarType type = b.t->scalar_type();
    at::Tensor dx = empty(b.t->sizes(), *b.t, type), db = empty(b.t->sizes(), *b.t, type), dgate, v[5], ws;
    // scale, post's gamma and beta, norm's: a tensor each, as the Python path has them (what
    // shared a storage would be kept or saved whole with any of them, and grow into the next).
    // us a call, 196 x 192 fp32 with all six: 14.2, by empty() 16.3, in one storage 13.2
    const void* given[5] = {j.scale, j.g1, j.b1, j.g2, j.b2};
    bool sums = j.gate;
    if (j.gate) dgate = small(j.gate->sizes(), *b.t);
    for (int i = 0; i < 5; ++i)
      if (given[i]) v[i] = small({b.C}, *b.t), sums = true;
    const size_t bytes = sums ? p_residual_norm_backward_ws((int)b.R, (int)b.C, b.dt) : 0;
    if (bytes) ws = empty({(long long)bytes}, *b.t, at::kByte);
    if (p_residual_norm_backward(has_ds ? ds.t->data_ptr() : nullptr, ds.ld, has_dy ? dy.t->data_ptr() : nullptr, dy.ld,
                                 b.t->data_ptr(), b.ld, has_dy ? s.t->data_ptr() : nullptr, s.ld, (int)b.R, (int)b.C,
                                 (gl_norm)kind, j.post, st[0], st[1], st[2], st[3], j.g1, j.b1, j.scale, gate_of(j), j.per, j.g2,
                                 b.dt, dx.data_ptr(), db.data_ptr(), ptr<float>(dgate), ptr<float>(v[0]), ptr<float>(v[1]),
                                 ptr<float>(v[2]), ptr<float>(v[3]), ptr<float>(v[4]), ptr(ws), bytes, stream_now(dev)) != GL_OK)
      return none();
    auto pair = [](bool is, at::Tensor& g, at::Tensor& o) -> PyObject* {
      if (!is) Py_RETURN_NONE;
      return Py_BuildValue("(NN)", wrap_or_none(std::move(g)), wrap_or_none(std::move(o)));
    };
    return Py_BuildValue("(NNNNNN)", THPVariable_Wrap(std::move(dx)), THPVariable_Wrap(std::move(db)),
                         wrap_or_none(std::move(dgate)), wrap_or_none(std::move(v[0])), pair(j.post, v[1], v[2]),
                         pair(j.norm, v[3], v[4]));
  });
}

// open(path of libgraphleap.so)
PyObject* py_open(PyObject*, PyObject* arg) {
  const char* path = PyUnicode_AsUTF8(arg);
  if (!path) return nullptr;
  void* h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
  if (!h) {
    PyErr_SetString(PyExc_RuntimeError, dlerror());
    return nullptr;
  }
#define GL_SYM(name, p)                                                       \
  if (!((p) = reinterpret_cast<decltype(p)>(dlsym(h, #name)))) {              \
    PyErr_SetString(PyExc_RuntimeError, "libgraphleap.so does not have " #name); \
    return nullptr;                                                           \
  }
  GL_SYM(gl_layer_norm, p_layer_norm)
  GL_SYM(gl_layer_norm_backward, p_layer_norm_backward)
  GL_SYM(gl_layer_norm_backward_workspace_bytes, p_layer_norm_backward_ws)
  GL_SYM(gl_quantize_rows, p_quantize_rows)
  GL_SYM(gl_layer_norm_q8, p_layer_norm_q8)
  GL_SYM(gl_linear_q8, p_linear_q8)
  GL_SYM(gl_gated_linear, p_gated_linear)
  GL_SYM(gl_gated_linear_workspace_bytes, p_gated_linear_ws)
  GL_SYM(gl_linear_backward, p_linear_backward)
  GL_SYM(gl_linear_backward_workspace_bytes, p_linear_backward_ws)
  GL_SYM(gl_gated_linear_backward, p_gated_linear_backward)
  GL_SYM(gl_gated_linear_backward_workspace_bytes, p_gated_linear_backward_ws)
  GL_SYM(gl_residual_norm, p_residual_norm)
  GL_SYM(gl_residual_norm_backward, p_residual_norm_backward)
  GL_SYM(gl_residual_norm_backward_workspace_bytes, p_residual_norm_backward_ws)
#undef GL_SYM
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"open", py_open, METH_O, "Take the entry points from this library."},
    {"layer_norm", (PyCFunction)(void (*)(void))py_layer_norm, METH_FASTCALL, nullptr},
    {"layer_norm_backward", (PyCFunction)(void (*)(void))py_layer_norm_backward, METH_FASTCALL, nullptr},
    {"quantize_rows", (PyCFunction)(void (*)(void))py_quantize_rows, METH_FASTCALL, nullptr},
    {"layer_norm_q8", (PyCFunction)(void (*)(void))py_layer_norm_q8, METH_FASTCALL, nullptr},
    {"linear_q8", (PyCFunction)(void (*)(void))py_linear_q8, METH_FASTCALL, nullptr},
    {"gated_linear", (PyCFunction)(void (*)(void))py_gated_linear, METH_FASTCALL, nullptr},
    {"linear_backward", (PyCFunction)(void (*)(void))py_linear_backward, METH_FASTCALL, nullptr},
    {"gated_linear_backward", (PyCFunction)(void (*)(void))py_gated_linear_backward, METH_FASTCALL, nullptr},
    {"residual_norm", (PyCFunction)(void (*)(void))py_residual_norm, METH_FASTCALL, nullptr},
    {"residual_norm_backward", (PyCFunction)(void (*)(void))py_residual_norm_backward, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&kModule); }
