// whtmix_torch.cpp -- the Python binding's quick path for the layer operators: a call whose tensors are plain (of torch's own
// classes, on the current device, rows at one stride) and whose results are to be allocated is checked, given its results and passed
// to the C ABI here.  A call of one token is bound by its way to the GPU: on a Grace core, in a loop over the same inputs, a norm takes
// 5.0 us this way and 12.3 step by step in Python, a product 4.9 and 12.0.  Every function returns None for any other call: whtmix.py then takes it step by step, with
// its own checks and messages.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include "whtmix.h"

namespace {

PyObject* g_check = nullptr;  // whtmix._check(status, what), which raises

struct Rows {
  void* p = nullptr;
  int64_t rows = 0, cols = 0, stride = 0;
};

// a plain tensor, or null
const at::Tensor* tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }
bool placed(const at::Tensor& t, int device, at::ScalarType type) {
  return t.is_cuda() && t.layout() == at::kStrided && t.get_device() == device && t.scalar_type() == type;
}
// t [..., C] with contiguous channels and its rows at one stride
bool rows_of(const at::Tensor& t, int device, at::ScalarType type, Rows* r) {
  if (t.dim() < 1 || !placed(t, device, type)) return false;
  r->cols = t.sizes().back();
  if (r->cols < 1) return false;
  r->p = t.data_ptr();
  if (t.is_contiguous()) {
    r->rows = t.numel() / r->cols, r->stride = r->cols;
    return true;
  }
  if (t.dim() != 2 || t.stride(1) != 1 || t.size(0) < 2 || t.stride(0) < r->cols) return false;
  r->rows = t.size(0), r->stride = t.stride(0);
  return true;
}
bool rows_like(PyObject* o, at::IntArrayRef shape, int device, at::ScalarType type, Rows* r) {
  const at::Tensor* t = tensor(o);
  return t && t->sizes() == shape && rows_of(*t, device, type, r);
}
bool floats(PyObject* o, at::IntArrayRef shape, int device, const float** p) {
  const at::Tensor* t = tensor(o);
  if (!t || !placed(*t, device, at::kFloat) || t->sizes() != shape || !t->is_contiguous()) return false;
  *p = static_cast<const float*>(t->data_ptr());
  return true;
}
bool type_of(PyObject* o, at::ScalarType* type) {
  if (!THPDtype_Check(o)) return false;
  *type = reinterpret_cast<THPDtype*>(o)->scalar_type;
  return true;
}
int code(at::ScalarType t) { return t == at::kFloat ? WHTMIX_F32 : t == at::kBFloat16 ? WHTMIX_BF16 : WHTMIX_E4M3; }

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
}
bool current(int device) { return device >= 0 && c10::cuda::current_device() == device; }

// The entry point without the interpreter's lock: a launch waits while the stream's queue is full.
template <typename F>
bool run(const char* what, int device, F&& call) {
  void* stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = call(stream);
  Py_END_ALLOW_THREADS;
  if (rc == WHTMIX_OK) return true;
  Py_XDECREF(PyObject_CallFunction(g_check, "is", rc, what));
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, what);
  return false;
}

template <typename... T>
PyObject* tuple(T&&... t) {
  constexpr Py_ssize_t n = sizeof...(T);
  PyObject* out = PyTuple_New(n);
  if (!out) return nullptr;
  Py_ssize_t i = 0;
  bool ok = true;
  auto put = [&](const at::Tensor& v) {
    PyObject* o = v.defined() ? THPVariable_Wrap(v) : Py_NewRef(Py_None);
    if (!o) ok = false;
    PyTuple_SET_ITEM(out, i++, o);
  };
  (put(t), ...);
  if (ok) return out;
  Py_DECREF(out);
  return nullptr;
}

// x, w, residual or None, eps, out_dtype or None
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* x = n == 5 ? tensor(args[0]) : nullptr;
  if (!x || !PyFloat_CheckExact(args[3]) || !x->is_cuda()) Py_RETURN_NONE;
  const int device = x->get_device();
  const at::ScalarType type = x->scalar_type();
  if (!current(device) || (type != at::kBFloat16 && type != at::kFloat)) Py_RETURN_NONE;
  at::ScalarType to = type;
  if (args[4] != Py_None && (!type_of(args[4], &to) || (to != type && to != at::kFloat8_e4m3fn))) Py_RETURN_NONE;
  Rows rx, rr;
  const float* w;
  if (!rows_of(*x, device, type, &rx) || !floats(args[1], {rx.cols}, device, &w)) Py_RETURN_NONE;
  const bool sum = args[2] != Py_None, eight = to == at::kFloat8_e4m3fn;
  const at::IntArrayRef shape = x->sizes();
  if (sum && !rows_like(args[2], shape, device, type, &rr)) Py_RETURN_NONE;
  if (eight && rx.cols % 16) Py_RETURN_NONE;  // its rows lie at a wider pitch
  const at::Tensor y = empty(shape, to, *x), h = sum ? empty(shape, type, *x) : at::Tensor();
  const at::Tensor s = eight ? empty(shape.slice(0, shape.size() - 1), at::kFloat, *x) : at::Tensor();
  void *yp = y.data_ptr(), *hp = sum ? h.data_ptr() : nullptr;
  float* sp = eight ? static_cast<float*>(s.data_ptr()) : nullptr;
  const float eps = static_cast<float>(PyFloat_AS_DOUBLE(args[3]));
  if (!run("whtmix_rms_norm", device, [&](void* stream) {
        return whtmix_rms_norm(rx.p, rr.p, w, hp, yp, sp, rx.rows, rx.cols, rx.stride, rr.stride, sum ? rx.cols : 0, rx.cols, eps, code(type),
                               code(to), stream);
      }))
    return nullptr;
  if (eight) return sum ? tuple(y, s, h) : tuple(y, s);
  return sum ? tuple(y, h) : THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

// h, w, dy, dh or None, eps
PyObject* rms_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* h = n == 5 ? tensor(args[0]) : nullptr;
  if (!h || !PyFloat_CheckExact(args[4]) || !h->is_cuda()) Py_RETURN_NONE;
  const int device = h->get_device();
  const at::ScalarType type = h->scalar_type();
  if (!current(device) || (type != at::kBFloat16 && type != at::kFloat)) Py_RETURN_NONE;
  Rows rh, ry, rd;
  const float* w;
  if (!rows_of(*h, device, type, &rh) || !floats(args[1], {rh.cols}, device, &w) || !rows_like(args[2], h->sizes(), device, type, &ry) ||
      (args[3] != Py_None && !rows_like(args[3], h->sizes(), device, type, &rd)))
    Py_RETURN_NONE;
  const at::Tensor dx = empty(h->sizes(), type, *h), dw = empty({rh.cols}, at::kFloat, *h);
  void* dxp = dx.data_ptr();
  float* dwp = static_cast<float*>(dw.data_ptr());
  const float eps = static_cast<float>(PyFloat_AS_DOUBLE(args[4]));
  if (!run("whtmix_rms_norm_backward", device, [&](void* stream) {
        return whtmix_rms_norm_backward(rh.p, w, ry.p, rd.p, dxp, dwp, rh.rows, rh.cols, rh.stride, ry.stride, rd.stride, rh.cols, eps,
                                        code(type), stream);
      }))
    return nullptr;
  return tuple(dx, dw);
  END_HANDLE_TH_ERRORS
}

// x, w, bias or None, activation code, residual or None, x_scale or None, w_scale or None, preact (None, False or True), out_dtype
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *x = n == 9 ? tensor(args[0]) : nullptr, *w = x ? tensor(args[1]) : nullptr;
  if (!w || !x->is_cuda() || w->dim() != 2) Py_RETURN_NONE;
  const int device = x->get_device();
  const at::ScalarType type = x->scalar_type();
  const bool eight = type == at::kFloat8_e4m3fn, save = args[7] == Py_True;
  at::ScalarType to;
  if (!current(device) || (type != at::kBFloat16 && !eight) || !type_of(args[8], &to) || (to != at::kBFloat16 && to != at::kFloat) ||
      (save && to != at::kBFloat16))
    Py_RETURN_NONE;
  Rows rx, rw, rr;
  if (!rows_of(*x, device, type, &rx) || !rows_of(*w, device, type, &rw) || rw.cols != rx.cols) Py_RETURN_NONE;
  const at::IntArrayRef lead = x->sizes().slice(0, x->dim() - 1);
  at::DimVector shape(lead);
  shape.push_back(w->size(0));
  const float *bias = nullptr, *sx = nullptr, *sw = nullptr;
  if (eight ? !floats(args[5], lead, device, &sx) || !floats(args[6], {w->size(0)}, device, &sw) : args[5] != Py_None || args[6] != Py_None)
    Py_RETURN_NONE;
  if ((args[2] != Py_None && !floats(args[2], {w->size(0)}, device, &bias)) ||
      (args[4] != Py_None && !rows_like(args[4], shape, device, to, &rr)))
    Py_RETURN_NONE;
  const int act = static_cast<int>(PyLong_AsLong(args[3]));
  const at::Tensor y = empty(shape, to, *x), p = save ? empty(shape, at::kBFloat16, *x) : at::Tensor();
  void *yp = y.data_ptr(), *pp = save ? p.data_ptr() : nullptr;
  const int64_t N = w->size(0);
  if (!run("whtmix_linear", device, [&](void* stream) {
        return whtmix_linear(rx.p, rw.p, sx, sw, bias, rr.p, pp, yp, rx.rows, N, rx.cols, rx.stride, rw.stride, rr.stride, save ? N : 0, N, act,
                             code(type), code(to), stream);
      }))
    return nullptr;
  return save ? tuple(y, p) : THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

// x, w, dy, p or None, activation code, need_dx, need_dw, need_db, dw_dtype
PyObject* linear_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *x = n == 9 ? tensor(args[0]) : nullptr, *w = x ? tensor(args[1]) : nullptr;
  if (!w || !x->is_cuda() || w->dim() != 2) Py_RETURN_NONE;
  const int device = x->get_device();
  at::ScalarType to;
  if (!current(device) || !type_of(args[8], &to) || (to != at::kBFloat16 && to != at::kFloat)) Py_RETURN_NONE;
  Rows rx, rw, ry, rp;
  const at::ScalarType bf16 = at::kBFloat16;
  if (!rows_of(*x, device, bf16, &rx) || !rows_of(*w, device, bf16, &rw) || rw.cols != rx.cols) Py_RETURN_NONE;
  const int64_t N = w->size(0), K = rx.cols;
  at::DimVector shape(x->sizes().slice(0, x->dim() - 1));
  shape.push_back(N);
  const int act = static_cast<int>(PyLong_AsLong(args[4]));
  if (!rows_like(args[2], shape, device, bf16, &ry) || (act != WHTMIX_ACT_NONE && !rows_like(args[3], shape, device, bf16, &rp)))
    Py_RETURN_NONE;
  int need[3];
  for (int i = 0; i < 3; ++i)
    if ((need[i] = PyObject_IsTrue(args[5 + i])) < 0) return nullptr;
  const at::Tensor dx = need[0] ? empty(x->sizes(), bf16, *x) : at::Tensor();
  const at::Tensor dw = need[1] ? empty({N, K}, to, *x) : at::Tensor();
  const at::Tensor db = need[2] ? empty({N}, at::kFloat, *x) : at::Tensor();
  void *dxp = dx.defined() ? dx.data_ptr() : nullptr, *dwp = dw.defined() ? dw.data_ptr() : nullptr;
  float* dbp = db.defined() ? static_cast<float*>(db.data_ptr()) : nullptr;
  if (!run("whtmix_linear_backward", device, [&](void* stream) {
        return whtmix_linear_backward(rx.p, rw.p, ry.p, rp.p, dxp, dwp, dbp, rx.rows, N, K, rx.stride, rw.stride, ry.stride, rp.stride,
                                      dxp ? K : 0, act, code(to), stream);
      }))
    return nullptr;
  return tuple(dx, dw, db);
  END_HANDLE_TH_ERRORS
}

PyObject* bind(PyObject*, PyObject* check) {
  Py_INCREF(check);
  Py_XSETREF(g_check, check);
  Py_RETURN_NONE;
}

#define WHTMIX_QUICK(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {WHTMIX_QUICK(rms_norm), WHTMIX_QUICK(rms_norm_backward), WHTMIX_QUICK(linear), WHTMIX_QUICK(linear_backward),
                         {"bind", bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "whtmix_torch", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit_whtmix_torch() { return PyModule_Create(&module); }
