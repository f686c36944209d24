// Python binding of the operators around the layer (norm, balance loss, vocabulary head, rows sorted by
// expert and their e4m3 products) on torch tensors: checks, output allocation and the call into libeat.so, nothing else.  A small call is
// bound by the host, and ctypes with Python-level allocations took most of it (RMS norm of one row:
// 13 us a call, here 4.4; its gradient 20 and 7.4; balance loss 15 and 6.5).
#include <Python.h>

#include <ATen/Context.h>
#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
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

// Whether something watches or fills what torch allocates: a dispatch mode, a tracer or inference mode (they
// show in the thread's dispatch keys), an observer of torch's calls, or deterministic algorithms, which fill it.
bool watched() {
  if (c10::impl::tls_local_dispatch_key_set().included_ != c10::default_included_set) return true;
  const at::Context& c = at::globalContext();
  return (c.deterministicAlgorithms() && c.deterministicFillUninitializedMemory()) || at::hasCallbacks();
}
// For the thread's running call (a dispatch mode may make others before it is done).
thread_local bool t_watched = true;
struct Watch {
  const bool before = t_watched;
  Watch() { t_watched = watched(); }
  ~Watch() { t_watched = before; }
};
// As at::empty, past the dispatcher where nobody is there to see the difference (0.25 to 0.35 us an output; rows
// and columns, which have four, 7.1 -> 5.7 us a call).
at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
  if (t_watched) return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
  return at::Tensor(at::detail::empty_cuda(shape, type, like.device(), std::nullopt));
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
    const Watch watch;
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
int32_t integer(const char* name, PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PyFailure();
  if (v < INT32_MIN) value_error(std::string(name) + ": too small");
  return to_i32(name, v);
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

// ---- experts: rows sorted by expert
// (idx, number of experts, mask or None) -> (offsets, slot)
PyObject* expert_sort(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("expert_sort", n, 3, [&] {
    const at::Tensor& idx = matrix("idx", a[0], at::kInt);
    const int64_t T = idx.size(0), K = idx.size(1);
    const int32_t E = integer("n_experts", a[1]);
    const uint8_t* mask = take_mask(a[2], T, idx);
    const c10::cuda::CUDAGuard guard(idx.device());
    const int32_t T32 = to_i32("T", T), K32 = to_i32("K", K);
    at::Tensor offsets = empty({std::min(std::max(E, 0), 256) + 1}, at::kInt, idx);
    at::Tensor slot = empty(idx.sizes(), at::kInt, idx);
    const int64_t bytes = eat_expert_sort_workspace(T32, K32, E);
    at::Tensor work;
    if (bytes > 0) work = empty({bytes}, at::kByte, idx);
    ok(eat_expert_sort((const int32_t*)idx.const_data_ptr(), T32, K32, E, mask,
                       (int32_t*)offsets.data_ptr(), (int32_t*)slot.data_ptr(),
                       bytes > 0 ? work.data_ptr() : nullptr, stream_of(idx)));
    return results(offsets, slot);
  });
}

// offsets [E + 1] or None; E
const int32_t* take_offsets(PyObject* o, const at::Tensor& like, int64_t& E) {
  E = 1;
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor("offsets", o);
  if (t.dim() != 1 || t.numel() < 2) value_error("offsets: need [E + 1] int32");
  E = t.numel() - 1;
  return (const int32_t*)check("offsets", t, at::kInt, t.sizes(), &like).const_data_ptr();
}
int64_t blocks_of(int64_t n) { return (n + 127) / 128; }

// (x, slot, offsets, fp8) -> (rows, scale or None)
PyObject* expert_gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("expert_gather", n, 4, [&] {
    const at::Tensor& x = rows("x", a[0]);
    const at::Tensor& slot = matrix("slot", a[1], at::kInt, &x);
    const int64_t T = x.size(0), d = x.size(1), K = slot.size(1);
    check("slot", slot, at::kInt, {T, K}, &x);
    int64_t E;
    const int32_t* offsets = take_offsets(a[2], x, E);
    const bool fp8 = a[3] == Py_True;
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor out = empty({T * K, d}, fp8 ? at::kFloat8_e4m3fn : x.scalar_type(), x), scale;
    if (fp8) scale = empty({blocks_of(d), T * K}, at::kFloat, x);
    ok(eat_expert_gather(x.const_data_ptr(), to_i32("T", T), to_i32("K", K), to_i32("E", E),
                         to_i32("d", d), code(x), (const int32_t*)slot.const_data_ptr(), offsets,
                         out.data_ptr(), fp8 ? EAT_FP8_E4M3 : code(x),
                         fp8 ? (float*)scale.data_ptr() : nullptr, stream_of(x)));
    return results(out, scale);
  });
}

// (rows, slot, w or None) -> y
PyObject* expert_combine(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("expert_combine", n, 3, [&] {
    const at::Tensor& r = rows("rows", a[0]);
    const at::Tensor& slot = matrix("slot", a[1], at::kInt, &r);
    const int64_t T = slot.size(0), K = slot.size(1), d = r.size(1);
    check("rows", r, r.scalar_type(), {T * K, d}, nullptr);
    const void* w = take_or_null("w", a[2], at::kFloat, {T, K}, r);
    const c10::cuda::CUDAGuard guard(r.device());
    at::Tensor y = empty({T, d}, r.scalar_type(), r);
    ok(eat_expert_combine(r.const_data_ptr(), to_i32("T", T), to_i32("K", K), to_i32("d", d),
                          code(r), (const int32_t*)slot.const_data_ptr(), (const float*)w,
                          y.data_ptr(), stream_of(r)));
    return THPVariable_Wrap(y);
  });
}

// (dy, rows, slot, offsets, w) -> (drows, dw)
PyObject* expert_combine_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("expert_combine_grad", n, 5, [&] {
    const at::Tensor& dy = rows("dy", a[0]);
    const at::Tensor& slot = matrix("slot", a[2], at::kInt, &dy);
    const int64_t T = dy.size(0), d = dy.size(1), K = slot.size(1);
    check("slot", slot, at::kInt, {T, K}, &dy);
    const at::Tensor& r = take("rows", a[1], dy.scalar_type(), {T * K, d}, dy);
    int64_t E;
    const int32_t* offsets = take_offsets(a[3], dy, E);
    const at::Tensor& w = take("w", a[4], at::kFloat, {T, K}, dy);
    const c10::cuda::CUDAGuard guard(dy.device());
    at::Tensor drows = empty({T * K, d}, dy.scalar_type(), dy), dw = empty({T, K}, at::kFloat, dy);
    ok(eat_expert_combine_grad(dy.const_data_ptr(), r.const_data_ptr(), to_i32("T", T),
                               to_i32("K", K), to_i32("E", E), to_i32("d", d), code(dy),
                               (const int32_t*)slot.const_data_ptr(), offsets,
                               (const float*)w.const_data_ptr(), drows.data_ptr(),
                               (float*)dw.data_ptr(), stream_of(dy)));
    return results(drows, dw);
  });
}

// ---- e4m3 with a scale for each block of 128
// x -> (q, scale)
PyObject* quant_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("quant_rows", n, 1, [&] {
    const at::Tensor& x = rows("x", a[0]);
    const int64_t M = x.size(0), K = x.size(1);
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor q = empty(x.sizes(), at::kFloat8_e4m3fn, x);
    at::Tensor scale = empty({blocks_of(K), M}, at::kFloat, x);
    ok(eat_quant_rows(x.const_data_ptr(), to_i32("M", M), to_i32("K", K), code(x), q.data_ptr(),
                      (float*)scale.data_ptr(), stream_of(x)));
    return results(q, scale);
  });
}

// (x, offsets or None, whether the rows too) -> (q or None, scale or None, cq, cscale)
PyObject* quant_columns(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("quant_columns", n, 3, [&] {
    const at::Tensor& x = rows("x", a[0]);
    const int64_t M = x.size(0), K = x.size(1);
    int64_t E;
    const int32_t* offsets = take_offsets(a[1], x, E);
    const c10::cuda::CUDAGuard guard(x.device());
    const int32_t M32 = to_i32("M", M), E32 = to_i32("E", E);
    at::Tensor q, scale;
    if (a[2] == Py_True) {
      q = empty(x.sizes(), at::kFloat8_e4m3fn, x);
      scale = empty({blocks_of(K), M}, at::kFloat, x);
    }
    at::Tensor cq = empty({eat_quant_columns_rows(M32, E32), K}, at::kFloat8_e4m3fn, x);
    at::Tensor cscale = empty({eat_quant_columns_blocks(M32, E32), K}, at::kFloat, x);
    ok(eat_quant_columns(x.const_data_ptr(), M32, to_i32("K", K), code(x), offsets, E32,
                         q.defined() ? q.data_ptr() : nullptr,
                         q.defined() ? (float*)scale.data_ptr() : nullptr, cq.data_ptr(),
                         (float*)cscale.data_ptr(), stream_of(x)));
    return results(q, scale, cq, cscale);
  });
}

// w -> (q, scale)
PyObject* quant_tiles(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("quant_tiles", n, 1, [&] {
    const at::Tensor& w = tensor("w", a[0]);
    if ((w.dim() != 2 && w.dim() != 3) ||
        (w.scalar_type() != at::kFloat && w.scalar_type() != at::kBFloat16))
      value_error("w: need [N, K] or [E, N, K], fp32 or bf16");
    check("w", w, w.scalar_type(), w.sizes(), nullptr);
    const bool many = w.dim() == 3;
    const int64_t E = many ? w.size(0) : 1, N = w.size(-2), K = w.size(-1);
    const c10::cuda::CUDAGuard guard(w.device());
    at::Tensor q = empty(w.sizes(), at::kFloat8_e4m3fn, w);
    at::Tensor scale = many ? empty({E, blocks_of(N), blocks_of(K)}, at::kFloat, w)
                            : empty({blocks_of(N), blocks_of(K)}, at::kFloat, w);
    ok(eat_quant_tiles(w.const_data_ptr(), to_i32("E", E), to_i32("N", N), to_i32("K", K), code(w),
                       q.data_ptr(), (float*)scale.data_ptr(), stream_of(w)));
    return results(q, scale);
  });
}

// None (bf16), torch.bfloat16 or torch.float32
at::ScalarType out_type(PyObject* o) {
  if (o == Py_None) return at::kBFloat16;
  if (THPDtype_Check(o)) {
    const at::ScalarType t = ((THPDtype*)o)->scalar_type;
    if (t == at::kBFloat16 || t == at::kFloat) return t;
  }
  value_error("dtype: need torch.bfloat16 or torch.float32");
}

// (xq, xs, wq, ws, offsets or None, transposed, dtype or None) -> y
PyObject* block_mm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("block_mm", n, 7, [&] {
    const at::Tensor &xq = matrix("xq", a[0], at::kFloat8_e4m3fn), &wq = tensor("wq", a[2]);
    int64_t E;
    const int32_t* offsets = take_offsets(a[4], xq, E);
    const bool many = a[4] != Py_None;
    if (wq.dim() != (many ? 3 : 2))
      value_error(many ? "wq: need [E, N, K] with offsets" : "wq: need [N, K] without offsets");
    const int64_t N = wq.size(-2), K = wq.size(-1), M = xq.size(0);
    if (many) check("wq", wq, at::kFloat8_e4m3fn, {E, N, K}, &xq);
    else check("wq", wq, at::kFloat8_e4m3fn, {N, K}, &xq);
    const int back = PyObject_IsTrue(a[5]);
    if (back < 0) throw PyFailure();
    const int64_t inner = back ? N : K, cols = back ? K : N;
    check("xq", xq, at::kFloat8_e4m3fn, {M, inner}, nullptr);
    const at::Tensor& xs = take("xs", a[1], at::kFloat, {blocks_of(inner), M}, xq);
    const at::Tensor& ws = many
        ? take("ws", a[3], at::kFloat, {E, blocks_of(N), blocks_of(K)}, xq)
        : take("ws", a[3], at::kFloat, {blocks_of(N), blocks_of(K)}, xq);
    const at::ScalarType type = out_type(a[6]);
    const c10::cuda::CUDAGuard guard(xq.device());
    at::Tensor y = empty({M, cols}, type, xq);
    ok(eat_block_mm(xq.const_data_ptr(), (const float*)xs.const_data_ptr(), wq.const_data_ptr(),
                    (const float*)ws.const_data_ptr(), offsets, to_i32("E", E), to_i32("M", M),
                    to_i32("N", N), to_i32("K", K), back, y.data_ptr(), code(y), stream_of(xq)));
    return THPVariable_Wrap(y);
  });
}

// (gq, gs, xq, xs, offsets or None, dtype or None) -> dw
PyObject* block_mm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("block_mm_grad", n, 6, [&] {
    const at::Tensor& gq = matrix("gq", a[0], at::kFloat8_e4m3fn);
    const at::Tensor& xq = matrix("xq", a[2], at::kFloat8_e4m3fn, &gq);
    const at::Tensor& gs = matrix("gs", a[1], at::kFloat, &gq);
    const int64_t P = gq.size(0), N = gq.size(1), K = xq.size(1), B = gs.size(0);
    check("xq", xq, at::kFloat8_e4m3fn, {P, K}, &gq);
    int64_t E;
    const int32_t* offsets = take_offsets(a[4], gq, E);
    // (every operand that eat_quant_columns makes has these)
    if (P % 32 != 0 || B < blocks_of(P)) value_error("gq, gs: not quant_columns' rows and blocks");
    check("gs", gs, at::kFloat, {B, N}, &gq);
    const at::Tensor& xs = take("xs", a[3], at::kFloat, {B, K}, gq);
    const at::ScalarType type = out_type(a[5]);
    const c10::cuda::CUDAGuard guard(gq.device());
    at::Tensor dw = a[4] != Py_None ? empty({E, N, K}, type, gq) : empty({N, K}, type, gq);
    ok(eat_block_mm_grad(gq.const_data_ptr(), (const float*)gs.const_data_ptr(),
                         xq.const_data_ptr(), (const float*)xs.const_data_ptr(), offsets,
                         to_i32("E", E), to_i32("rows", P), to_i32("blocks", B), to_i32("N", N),
                         to_i32("K", K), dw.data_ptr(), code(dw), stream_of(gq)));
    return THPVariable_Wrap(dw);
  });
}

int64_t gated_width(const at::Tensor& gu) {
  if (gu.size(1) % 2) value_error("gu: need [R, 2 F] rows");
  return gu.size(1) / 2;
}

// (gu, fp8) -> (h, scale or None)
PyObject* swiglu(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("swiglu", n, 2, [&] {
    const at::Tensor& gu = rows("gu", a[0]);
    const int64_t R = gu.size(0), F = gated_width(gu);
    const bool fp8 = a[1] == Py_True;
    const c10::cuda::CUDAGuard guard(gu.device());
    at::Tensor h = empty({R, F}, fp8 ? at::kFloat8_e4m3fn : gu.scalar_type(), gu), scale;
    if (fp8) scale = empty({blocks_of(F), R}, at::kFloat, gu);
    ok(eat_swiglu(gu.const_data_ptr(), to_i32("R", R), to_i32("F", F), code(gu), h.data_ptr(),
                  fp8 ? EAT_FP8_E4M3 : code(gu), fp8 ? (float*)scale.data_ptr() : nullptr,
                  stream_of(gu)));
    return results(h, scale);
  });
}

// (gu, dh) -> dgu
PyObject* swiglu_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry("swiglu_grad", n, 2, [&] {
    const at::Tensor& gu = rows("gu", a[0]);
    const int64_t R = gu.size(0), F = gated_width(gu);
    const at::Tensor& dh = take("dh", a[1], gu.scalar_type(), {R, F}, gu);
    const c10::cuda::CUDAGuard guard(gu.device());
    at::Tensor dgu = empty(gu.sizes(), gu.scalar_type(), gu);
    ok(eat_swiglu_grad(gu.const_data_ptr(), dh.const_data_ptr(), to_i32("R", R), to_i32("F", F),
                       code(gu), dgu.data_ptr(), stream_of(gu)));
    return THPVariable_Wrap(dgu);
  });
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_XSETREF(g_error, Py_NewRef(type));
  Py_RETURN_NONE;
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {FAST(norm),         FAST(norm_grad), FAST(balance_loss),
                           FAST(balance_grad), FAST(head_nll),  FAST(head_nll_grad),
                           FAST(expert_sort), FAST(expert_gather), FAST(expert_combine),
                           FAST(expert_combine_grad), FAST(quant_rows), FAST(quant_columns),
                           FAST(quant_tiles), FAST(block_mm), FAST(block_mm_grad), FAST(swiglu),
                           FAST(swiglu_grad),
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_eatops", nullptr, -1, g_methods};

}  // namespace

PyMODINIT_FUNC PyInit__eatops() { return PyModule_Create(&g_module); }
