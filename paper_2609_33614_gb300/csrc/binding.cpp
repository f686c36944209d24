// Python binding of the operators around the layer (norm, balance loss, vocabulary head) on torch
// tensors: checks, output allocation and the call into libeat.so, nothing else.  A small call is
// bound by the host, and ctypes with Python-level allocations took most of it (RMS norm of one row:
// 13 us a call, here 4.4; its gradient 20 and 7.4; balance loss 15 and 6.5).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <sstream>
#include <string>

#include "eat.h"

namespace {

PyObject* g_error = nullptr;  // paper_2609_33614_gb300.eat.EatError

struct PyFailure {};  // a Python exception is set

[[noreturn]] void value_error(const std::string& msg) {
  PyErr_SetString(PyExc_ValueError, msg.c_str());
  throw PyFailure();
}

const at::Tensor& tensor(const char* name, PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s: need a tensor, got %s", name, Py_TYPE(o)->tp_name);
    throw PyFailure();
  }
  return THPVariable_Unpack(o);
}

// Fails unless t has this type and shape, contiguous on the GPU, and lies where `like` (the call's first
// tensor, or null for it) does.
const at::Tensor& check(const char* name, const at::Tensor& t, at::ScalarType type,
                        at::IntArrayRef shape, const at::Tensor* like) {
  if (t.scalar_type() != type || t.sizes() != shape) {
    std::ostringstream s;
    s << name << ": need " << shape << " " << type << ", got " << t.sizes() << " "
      << t.scalar_type();
    value_error(s.str());
  }
  if (!t.is_cuda() || !t.is_contiguous())
    value_error(std::string(name) + ": need a contiguous CUDA tensor");
  if (like && t.device() != like->device()) {
    std::ostringstream s;
    s << name << ": need a tensor on " << like->device() << ", got one on " << t.device();
    value_error(s.str());
  }
  return t;
}
const at::Tensor& take(const char* name, PyObject* o, at::ScalarType type,
                       std::initializer_list<int64_t> shape, const at::Tensor& like) {
  return check(name, tensor(name, o), type, at::IntArrayRef(shape.begin(), shape.size()), &like);
}
const void* take_or_null(const char* name, PyObject* o, at::ScalarType type,
                         std::initializer_list<int64_t> shape, const at::Tensor& like) {
  return o == Py_None ? nullptr : take(name, o, type, shape, like).const_data_ptr();
}

// fp32 or bf16 rows [T, d]
const at::Tensor& rows(const char* name, PyObject* o) {
  const at::Tensor& t = tensor(name, o);
  if (t.dim() != 2 || (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16))
    value_error(std::string(name) + ": need [T, d] fp32 or bf16 rows");
  return check(name, t, t.scalar_type(), t.sizes(), nullptr);
}
const at::Tensor& matrix(const char* name, PyObject* o, at::ScalarType type,
                         const at::Tensor* like = nullptr) {
  const at::Tensor& t = tensor(name, o);
  if (t.dim() != 2) value_error(std::string(name) + ": need a matrix");
  return check(name, t, type, t.sizes(), like);
}
const uint8_t* take_mask(PyObject* o, int64_t T, const at::Tensor& like) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor("mask", o);
  const at::ScalarType type = t.scalar_type() == at::kByte ? at::kByte : at::kBool;
  return (const uint8_t*)take("mask", o, type, {T}, like).const_data_ptr();
}

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
  return at::empty(shape, like.options().dtype(type));
}
int code(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 ? EAT_BF16 : EAT_F32; }
int32_t to_i32(const char* name, int64_t v) {
  if (v > INT32_MAX) value_error(std::string(name) + ": too large");
  return (int32_t)v;
}

void ok(eat_status s) {
  if (s == EAT_OK) return;
  PyObject* e = PyObject_CallFunction(g_error, "is", (int)s, eat_last_error(nullptr));
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw PyFailure();
}

void* stream_of(const at::Tensor& t) {
  return c10::cuda::getCurrentCUDAStream(t.device().index()).stream();
}

template <typename... T>
PyObject* results(T&&... t) {
  PyObject* r = PyTuple_New(sizeof...(t));
  if (!r) throw PyFailure();
  Py_ssize_t i = 0;
  auto put = [&](const at::Tensor& v) {
    PyObject* o = v.defined() ? THPVariable_Wrap(v) : Py_NewRef(Py_None);
    if (!o) {
      Py_DECREF(r);
      throw PyFailure();
    }
    PyTuple_SET_ITEM(r, i++, o);
  };
  (put(t), ...);
  return r;
}

// Runs f with n arguments; exceptions become Python's.
template <typename F>
PyObject* entry(const char* name, Py_ssize_t got, Py_ssize_t n, F&& f) {
  if (got != n) {
    PyErr_Format(PyExc_TypeError, "%s: need %zd arguments, got %zd", name, n, got);
    return nullptr;
  }
  try {
    return f();
  } catch (const PyFailure&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyFailure();
  return v;
}
eat_head* handle(PyObject* o) {
  void* p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw PyFailure();
  return (eat_head*)p;
}

// (x, gamma, eps, residual or None, fp8) -> (y, y's scales or None, h)
PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("norm", n, 5, [&] {
    const at::Tensor& x = rows("x", a[0]);
    const int64_t T = x.size(0), d = x.size(1);
    const at::Tensor& gamma = take("gamma", a[1], at::kFloat, {d}, x);
    const void* residual = take_or_null("residual", a[3], x.scalar_type(), {T, d}, x);
    const bool fp8 = a[4] == Py_True;
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor h = residual ? empty(x.sizes(), x.scalar_type(), x) : x;
    at::Tensor y = empty(x.sizes(), fp8 ? at::kFloat8_e4m3fn : x.scalar_type(), x), scale;
    if (fp8) scale = empty({T}, at::kFloat, x);
    ok(eat_rms_norm(x.const_data_ptr(), residual, to_i32("T", T), to_i32("d", d), code(x),
                    (const float*)gamma.const_data_ptr(), number(a[2]),
                    residual ? h.data_ptr() : nullptr, y.data_ptr(),
                    fp8 ? EAT_FP8_E4M3 : code(x), fp8 ? (float*)scale.data_ptr() : nullptr,
                    stream_of(x)));
    return results(y, scale, h);
  });
}

// (h, gamma, eps, dy, dres or None) -> (dx, dgamma)
PyObject* norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("norm_grad", n, 5, [&] {
    const at::Tensor& h = rows("h", a[0]);
    const int64_t T = h.size(0), d = h.size(1);
    const at::Tensor& gamma = take("gamma", a[1], at::kFloat, {d}, h);
    const at::Tensor& dy = take("dy", a[3], h.scalar_type(), {T, d}, h);
    const void* dres = take_or_null("dres", a[4], h.scalar_type(), {T, d}, h);
    const c10::cuda::CUDAGuard guard(h.device());
    at::Tensor dx = empty(h.sizes(), h.scalar_type(), h), dgamma = empty({d}, at::kFloat, h);
    const int32_t T32 = to_i32("T", T), d32 = to_i32("d", d);
    at::Tensor work = empty({eat_rms_norm_grad_workspace(T32, d32)}, at::kByte, h);
    ok(eat_rms_norm_grad(h.const_data_ptr(), T32, d32, code(h),
                         (const float*)gamma.const_data_ptr(), number(a[2]), dy.const_data_ptr(),
                         dres, dx.data_ptr(), (float*)dgamma.data_ptr(), work.data_ptr(),
                         stream_of(h)));
    return results(dx, dgamma);
  });
}

// (logits, idx, mask or None) -> (loss, counts, n_tokens)
PyObject* balance_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("balance_loss", n, 3, [&] {
    const at::Tensor& logits = matrix("logits", a[0], at::kFloat);
    const at::Tensor& idx = matrix("idx", a[1], at::kInt, &logits);
    const int64_t T = logits.size(0), E = logits.size(1), K = idx.size(1);
    check("idx", idx, at::kInt, {T, K}, &logits);
    const uint8_t* mask = take_mask(a[2], T, logits);
    const c10::cuda::CUDAGuard guard(logits.device());
    at::Tensor loss = empty({1}, at::kFloat, logits), counts = empty({E}, at::kInt, logits);
    at::Tensor count = empty({1}, at::kInt, logits);
    const int32_t T32 = to_i32("T", T), E32 = to_i32("E", E);
    at::Tensor work = empty({eat_balance_workspace(T32, E32)}, at::kByte, logits);
    ok(eat_balance_loss((const float*)logits.const_data_ptr(), T32, E32, to_i32("K", K),
                        (const int32_t*)idx.const_data_ptr(), mask, (float*)loss.data_ptr(),
                        (int32_t*)counts.data_ptr(), (int32_t*)count.data_ptr(), work.data_ptr(),
                        stream_of(logits)));
    return results(loss, counts, count);
  });
}

// (logits, counts, n_tokens, g, mask or None) -> dlogits
PyObject* balance_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("balance_grad", n, 5, [&] {
    const at::Tensor& logits = matrix("logits", a[0], at::kFloat);
    const int64_t T = logits.size(0), E = logits.size(1);
    const at::Tensor& counts = take("counts", a[1], at::kInt, {E}, logits);
    const at::Tensor& count = take("n_tokens", a[2], at::kInt, {1}, logits);
    const at::Tensor& g = take("g", a[3], at::kFloat, {1}, logits);
    const uint8_t* mask = take_mask(a[4], T, logits);
    const c10::cuda::CUDAGuard guard(logits.device());
    at::Tensor d = empty(logits.sizes(), at::kFloat, logits);
    ok(eat_balance_grad((const float*)logits.const_data_ptr(), to_i32("T", T), to_i32("E", E),
                        mask, (const int32_t*)counts.const_data_ptr(),
                        (const int32_t*)count.const_data_ptr(), (const float*)g.const_data_ptr(),
                        (float*)d.data_ptr(), stream_of(logits)));
    return THPVariable_Wrap(d);
  });
}

// (handle, w, x, target, x_scale or None) -> (nll, lse)
PyObject* head_nll(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("head_nll", n, 5, [&] {
    const at::Tensor &w = tensor("w", a[1]), &target = tensor("target", a[3]);
    const int64_t T = target.numel();
    const at::Tensor& x = take("x", a[2], w.scalar_type(), {T, w.size(1)}, w);
    check("target", target, at::kInt, {T}, &w);
    const void* xs = nullptr;
    if (w.scalar_type() == at::kFloat8_e4m3fn)
      xs = take("x_scale", a[4], at::kFloat, {T}, w).const_data_ptr();
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor nll = empty({T}, at::kFloat, x), lse = empty({T}, at::kFloat, x);
    ok(eat_head_nll(handle(a[0]), x.const_data_ptr(), (const float*)xs, to_i32("T", T),
                    (const int32_t*)target.const_data_ptr(), (float*)nll.data_ptr(),
                    (float*)lse.data_ptr(), stream_of(x)));
    return results(nll, lse);
  });
}

// (handle, w, x, target, g) -> (nll, lse, dx, dw)
PyObject* head_nll_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("head_nll_grad", n, 5, [&] {
    const at::Tensor &w = tensor("w", a[1]), &target = tensor("target", a[3]);
    const int64_t T = target.numel();
    const at::Tensor& x = take("x", a[2], w.scalar_type(), {T, w.size(1)}, w);
    check("target", target, at::kInt, {T}, &w);
    const at::Tensor& g = take("g", a[4], at::kFloat, {T}, w);
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor nll = empty({T}, at::kFloat, x), lse = empty({T}, at::kFloat, x);
    at::Tensor dx = empty(x.sizes(), x.scalar_type(), x), dw = empty(w.sizes(), w.scalar_type(), x);
    ok(eat_head_nll_grad(handle(a[0]), x.const_data_ptr(), to_i32("T", T),
                         (const int32_t*)target.const_data_ptr(), (const float*)g.const_data_ptr(),
                         (float*)nll.data_ptr(), (float*)lse.data_ptr(), dx.data_ptr(),
                         dw.data_ptr(), stream_of(x)));
    return results(nll, lse, dx, dw);
  });
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_XSETREF(g_error, Py_NewRef(type));
  Py_RETURN_NONE;
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {FAST(norm),         FAST(norm_grad), FAST(balance_loss),
                           FAST(balance_grad), FAST(head_nll),  FAST(head_nll_grad),
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_eatops", nullptr, -1, g_methods};

}  // namespace

PyMODINIT_FUNC PyInit__eatops() { return PyModule_Create(&g_module); }
