// Native argument marshalling for the short calls of api.py: layer norm, its gradient
// and the 8-bit layers take a few microseconds on the device, less than Python needs to
// check their arguments and allocate their outputs.
//
// Each function takes what its namesake in api.py takes, for the ordinary form alone:
// plain tensors on the current device, on the current stream, outputs allocated here.
// Anything else, and any status but GL_OK (nothing was enqueued then), returns None: the
// caller goes through api.py's own checks, which name what is wrong.  No computation
// and no allocation but the outputs' and the workspace's happens here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

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

// Contiguous rows over the last axis, or a matrix of strided ones.
bool rows(PyObject* o, int device, Rows* r) {
  r->t = tensor(o, device);
  if (!r->t || !float_type(*r->t, &r->dt) || r->t->dim() < 1) return false;
  const at::Tensor& t = *r->t;
  r->C = t.size(-1);
  if (r->C < 1 || t.numel() < 1 || t.numel() / r->C > INT_MAX || r->C > INT_MAX) return false;
  r->R = t.numel() / r->C;
  r->ld = r->C;
  if (t.is_contiguous()) return true;
  if (t.dim() != 2 || t.stride(1) != 1 || t.stride(0) < r->C) return false;
  r->ld = t.stride(0);
  return true;
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
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&kModule); }
