// Argument marshalling of the ordinary call, without Python objects per argument:
// plain contiguous device tensors of the expected types and shapes, preallocated
// outputs, a workspace and the current stream.  Each function checks exactly that
// and calls the C entry point it is given (include/vtrace.h, vtrace_tokens.h,
// vtrace_parameters.h); on
// anything else it returns None, having done nothing, and the Python path (binding.py,
// tokens.py), which allocates and reports errors, takes the call.
//
// In Python the checks and conversions of a loss call take about 9 us, more than
// the kernel of a 32-lane batch.  The token-policy functions also allocate the outputs
// that are not given.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>

#include <initializer_list>
#include <vector>

#include "vtrace.h"
#include "vtrace_parameters.h"
#include "vtrace_tokens.h"

namespace {

using at::ScalarType;

// An ordinary dense device tensor: no subclass, no functional transform, nothing
// that gives its storage another meaning.
const at::Tensor* plain_tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  static const c10::DispatchKeySet special(
      {c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::Functionalize,
       c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::BatchedNestedTensor,
       c10::DispatchKey::Conjugate, c10::DispatchKey::Negative, c10::DispatchKey::ZeroTensor});
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.is_quantized() ||
      t.key_set().has_any(special) || !t.is_contiguous())
    return nullptr;
  return &t;
}

// Collects pointers while everything is as expected.
struct Args {
  bool ok = true;
  c10::Device device{c10::DeviceType::CUDA, -1};

  const at::Tensor* first(PyObject* o, size_t dims) {
    const at::Tensor* t = plain_tensor(o);
    if (t == nullptr || static_cast<size_t>(t->dim()) != dims) {
      ok = false;
      return nullptr;
    }
    device = t->device();
    return t;
  }
  void* tensor(PyObject* o, std::initializer_list<int64_t> shape, ScalarType type) {
    const at::Tensor* t = ok ? plain_tensor(o) : nullptr;
    if (t == nullptr || t->scalar_type() != type || t->device() != device ||
        t->sizes() != c10::IntArrayRef(shape.begin(), shape.size())) {
      ok = false;
      return nullptr;
    }
    return t->data_ptr();
  }
  void* optional(PyObject* o, std::initializer_list<int64_t> shape, ScalarType type) {
    return o == Py_None ? nullptr : tensor(o, shape, type);
  }
  // The workspace's bytes (as many as `bytes` says, which the library checks).
  void* workspace(PyObject* o) {
    const at::Tensor* t = ok ? plain_tensor(o) : nullptr;
    if (t == nullptr) {
      ok = false;
      return nullptr;
    }
    return t->data_ptr();
  }
  float number(PyObject* o) {
    if (!PyFloat_CheckExact(o)) {
      ok = false;
      return 0.0f;
    }
    return static_cast<float>(PyFloat_AS_DOUBLE(o));
  }
  size_t integer(PyObject* o) {
    if (!PyLong_CheckExact(o)) {
      ok = false;
      return 0;
    }
    const size_t v = PyLong_AsSize_t(o);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return v;
  }
  template <typename T>
  T address(PyObject* o) {
    return reinterpret_cast<T>(integer(o));
  }
};

// Modes that watch tensor operations see the call through binding.py's path.
bool watched() {
  return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set();
}

constexpr ScalarType F32 = ScalarType::Float, BF16 = ScalarType::BFloat16, I32 = ScalarType::Int;

bool logits_type(const at::Tensor& t, vtrace_dtype* code) {
  *code = t.scalar_type() == BF16 ? VTRACE_BF16 : VTRACE_F32;
  return t.scalar_type() == BF16 || t.scalar_type() == F32;
}

// targets(fn, target, behaviour, actions, rewards, discounts, values, bootstrap,
//         rho_bar, c_bar, lambda, variant, log_probs, vs, pg, workspace, bytes, stream)
PyObject* targets(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 18 || watched()) Py_RETURN_NONE;
  Args a;
  const at::Tensor* z = a.first(v[1], 3);
  vtrace_dtype dt;
  if (!a.ok || !logits_type(*z, &dt)) Py_RETURN_NONE;
  const int64_t T = z->size(0), B = z->size(1), A = z->size(2);
  const auto fn = a.address<decltype(&vtrace_targets_ex)>(v[0]);
  void* const y = v[12] == Py_True ? a.tensor(v[2], {T, B}, F32) : a.tensor(v[2], {T, B, A}, z->scalar_type());
  void* const act = a.tensor(v[3], {T, B}, I32);
  void* const r = a.tensor(v[4], {T, B}, F32);
  void* const g = a.tensor(v[5], {T, B}, F32);
  void* const val = a.tensor(v[6], {T, B}, F32);
  void* const boot = a.tensor(v[7], {B}, F32);
  const float rho = a.number(v[8]), c = a.number(v[9]), lam = a.number(v[10]);
  const auto variant = a.address<const vtrace_variant*>(v[11]);
  void* const vs = a.tensor(v[13], {T, B}, F32);
  void* const pg = a.tensor(v[14], {T, B}, F32);
  void* const ws = v[15] == Py_None ? nullptr : a.workspace(v[15]);
  const size_t bytes = a.integer(v[16]);
  const auto stream = a.address<vtrace_stream_t>(v[17]);
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(T, B, A, dt, z->data_ptr(), y, static_cast<const int32_t*>(act), static_cast<const float*>(r),
          static_cast<const float*>(g), static_cast<const float*>(val), static_cast<const float*>(boot), rho, c, lam,
          variant, static_cast<float*>(vs), static_cast<float*>(pg), ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

// loss(fn, target, behaviour, actions, rewards, discounts, values, bootstrap, rho_bar,
//      c_bar, lambda, baseline_cost, entropy_cost, variant, log_probs, bf16_grad, losses,
//      d_logits, d_values, vs, pg, lane_losses, workspace, bytes, stream)
PyObject* loss(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 25 || watched()) Py_RETURN_NONE;
  Args a;
  const at::Tensor* z = a.first(v[1], 3);
  vtrace_dtype dt;
  if (!a.ok || !logits_type(*z, &dt)) Py_RETURN_NONE;
  const int64_t T = z->size(0), B = z->size(1), A = z->size(2);
  const auto fn = a.address<decltype(&vtrace_loss_grad_ex)>(v[0]);
  void* const y = v[14] == Py_True ? a.tensor(v[2], {T, B}, F32) : a.tensor(v[2], {T, B, A}, z->scalar_type());
  void* const act = a.tensor(v[3], {T, B}, I32);
  void* const r = a.tensor(v[4], {T, B}, F32);
  void* const g = a.tensor(v[5], {T, B}, F32);
  void* const val = a.tensor(v[6], {T, B}, F32);
  void* const boot = a.tensor(v[7], {B}, F32);
  const float rho = a.number(v[8]), c = a.number(v[9]), lam = a.number(v[10]);
  const float bc = a.number(v[11]), ec = a.number(v[12]);
  const auto variant = a.address<const vtrace_variant*>(v[13]);
  void* const losses = a.tensor(v[16], {4}, F32);
  void* const dl = a.tensor(v[17], {T, B, A}, v[15] == Py_True ? BF16 : F32);
  void* const dv = a.tensor(v[18], {T, B}, F32);
  void* const vs = a.optional(v[19], {T, B}, F32);
  void* const pg = a.optional(v[20], {T, B}, F32);
  void* const lane = a.optional(v[21], {B, 3}, F32);
  void* const ws = a.workspace(v[22]);
  const size_t bytes = a.integer(v[23]);
  const auto stream = a.address<vtrace_stream_t>(v[24]);
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(T, B, A, dt, z->data_ptr(), y, static_cast<const int32_t*>(act), static_cast<const float*>(r),
          static_cast<const float*>(g), static_cast<const float*>(val), static_cast<const float*>(boot), rho, c, lam,
          bc, ec, variant, static_cast<float*>(losses), dl, static_cast<float*>(dv), static_cast<float*>(vs),
          static_cast<float*>(pg), static_cast<float*>(lane), ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

// head(fn, hidden, weight, bias, behaviour, actions, rewards, discounts, bootstrap, rho_bar,
//      c_bar, lambda, baseline_cost, entropy_cost, variant, log_probs, bf16_grad, losses,
//      d_hidden, d_weight, d_bias, vs, pg, lane_losses, outputs, workspace, bytes, stream)
PyObject* head(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 28 || watched()) Py_RETURN_NONE;
  Args a;
  const at::Tensor* h = a.first(v[1], 3);
  const at::Tensor* w = a.ok ? plain_tensor(v[2]) : nullptr;
  if (h == nullptr || w == nullptr || h->scalar_type() != BF16 || w->dim() != 2) Py_RETURN_NONE;
  const int64_t T = h->size(0), B = h->size(1), H = h->size(2), A = w->size(1) - 1;
  const auto fn = a.address<decltype(&vtrace_head_loss_grad)>(v[0]);
  void* const weight = a.tensor(v[2], {H, A + 1}, BF16);
  void* const bias = a.tensor(v[3], {A + 1}, F32);
  vtrace_dtype dt = VTRACE_F32;
  void* y = nullptr;
  if (v[15] == Py_True) {
    y = a.tensor(v[4], {T, B}, F32);
  } else {
    const at::Tensor* b = plain_tensor(v[4]);
    if (b == nullptr || !logits_type(*b, &dt)) Py_RETURN_NONE;
    y = a.tensor(v[4], {T, B, A}, b->scalar_type());
  }
  void* const act = a.tensor(v[5], {T, B}, I32);
  void* const r = a.tensor(v[6], {T, B}, F32);
  void* const g = a.tensor(v[7], {T, B}, F32);
  void* const boot = a.tensor(v[8], {B}, F32);
  const float rho = a.number(v[9]), c = a.number(v[10]), lam = a.number(v[11]);
  const float bc = a.number(v[12]), ec = a.number(v[13]);
  const auto variant = a.address<const vtrace_variant*>(v[14]);
  void* const losses = a.tensor(v[17], {4}, F32);
  void* const dh = a.tensor(v[18], {T, B, H}, v[16] == Py_True ? BF16 : F32);
  void* const dw = a.tensor(v[19], {H, A + 1}, F32);
  void* const db = a.tensor(v[20], {A + 1}, F32);
  void* const vs = a.optional(v[21], {T, B}, F32);
  void* const pg = a.optional(v[22], {T, B}, F32);
  void* const lane = a.optional(v[23], {B, 3}, F32);
  void* const outs = a.optional(v[24], {T, B, A + 1}, F32);
  void* const ws = a.workspace(v[25]);
  const size_t bytes = a.integer(v[26]);
  const auto stream = a.address<vtrace_stream_t>(v[27]);
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(T, B, A, H, dt, h->data_ptr(), weight, static_cast<const float*>(bias), y, static_cast<const int32_t*>(act),
          static_cast<const float*>(r), static_cast<const float*>(g), static_cast<const float*>(boot), rho, c, lam, bc,
          ec, variant, static_cast<float*>(losses), dh, static_cast<float*>(dw), static_cast<float*>(db),
          static_cast<float*>(vs), static_cast<float*>(pg), static_cast<float*>(lane), static_cast<float*>(outs), ws,
          bytes, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

// The token-policy calls: outputs that are None are allocated where they are wanted.
struct Outputs {
  PyObject* tuple;
  Py_ssize_t at = 0;
  explicit Outputs(Py_ssize_t n) : tuple(PyTuple_New(n)) {}
  ~Outputs() { Py_XDECREF(tuple); }
  Outputs(const Outputs&) = delete;
  Outputs& operator=(const Outputs&) = delete;

  void* add(Args* a, PyObject* given, bool wanted, std::initializer_list<int64_t> shape, ScalarType type) {
    void* p = nullptr;
    PyObject* o = given;
    if (given != Py_None) {
      p = a->tensor(given, shape, type);
      Py_INCREF(o);
    } else if (wanted && a->ok && tuple != nullptr) {
      at::Tensor t = at::empty(c10::IntArrayRef(shape.begin(), shape.size()), at::TensorOptions(a->device).dtype(type));
      p = t.data_ptr();
      o = THPVariable_Wrap(std::move(t));
    } else {
      Py_INCREF(o);
    }
    if (tuple == nullptr || o == nullptr) {
      a->ok = false;
      PyErr_Clear();
      Py_XDECREF(o);
    } else {
      PyTuple_SET_ITEM(tuple, at++, o);
    }
    return p;
  }
  // The outputs, or a failed call's status.
  PyObject* result(vtrace_status st) {
    if (st != VTRACE_OK) return PyLong_FromLong(st);
    PyObject* const t = tuple;
    tuple = nullptr;
    return t;
  }
};

bool on_device(Args* a, PyObject* current) {
  if (!PyLong_CheckExact(current) || a->device.index() != PyLong_AsLong(current)) a->ok = false;
  return a->ok;
}

// The workspace's bytes, on the call's device.
void* workspace_here(Args* a, PyObject* o) {
  void* const p = a->workspace(o);
  if (a->ok && THPVariable_Unpack(o).device() != a->device) a->ok = false;
  return p;
}

const float* floats(Args* a, PyObject* o, std::initializer_list<int64_t> shape) {
  return static_cast<const float*>(a->optional(o, shape, F32));
}

// vocab_log_probs(fn, hidden, weight, bias, tokens, with_entropy, log_probs, log_sums, entropy,
//                 workspace, bytes, device, stream)
PyObject* vocab_log_probs(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 13 || watched()) Py_RETURN_NONE;
  Args a;
  const at::Tensor* h = a.first(v[1], 3);
  const at::Tensor* w = a.ok ? plain_tensor(v[2]) : nullptr;
  if (h == nullptr || w == nullptr || h->scalar_type() != BF16 || w->dim() != 2 || !on_device(&a, v[11])) Py_RETURN_NONE;
  const int64_t T = h->size(0), B = h->size(1), H = h->size(2), V = w->size(0);
  const auto fn = a.address<decltype(&vtrace_vocab_log_probs)>(v[0]);
  void* const weight = a.tensor(v[2], {V, H}, BF16);
  const float* const bias = floats(&a, v[3], {V});
  void* const tokens = a.tensor(v[4], {T, B}, I32);
  void* const ws = workspace_here(&a, v[9]);
  const size_t bytes = a.integer(v[10]);
  const auto stream = a.address<vtrace_stream_t>(v[12]);
  if (v[5] != Py_True && v[5] != Py_False) Py_RETURN_NONE;
  Outputs out(3);
  void* const lp = out.add(&a, v[6], true, {T, B}, F32);
  void* const ls = out.add(&a, v[7], true, {T, B}, F32);
  void* const ent = out.add(&a, v[8], v[5] == Py_True, {T, B}, F32);
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(T, B, V, H, h->data_ptr(), weight, bias, static_cast<const int32_t*>(tokens), static_cast<float*>(lp),
          static_cast<float*>(ls), static_cast<float*>(ent), ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return out.result(st);
}

// vocab_grad(fn, hidden, weight, bias, tokens, log_sums, entropy, d_log_probs, d_entropy, bf16_grad,
//            d_hidden, d_weight, d_bias, with_bias, workspace, bytes, device, stream)
PyObject* vocab_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 18 || watched()) Py_RETURN_NONE;
  Args a;
  const at::Tensor* h = a.first(v[1], 3);
  const at::Tensor* w = a.ok ? plain_tensor(v[2]) : nullptr;
  if (h == nullptr || w == nullptr || h->scalar_type() != BF16 || w->dim() != 2 || !on_device(&a, v[16])) Py_RETURN_NONE;
  const int64_t T = h->size(0), B = h->size(1), H = h->size(2), V = w->size(0);
  const auto fn = a.address<decltype(&vtrace_vocab_grad)>(v[0]);
  void* const weight = a.tensor(v[2], {V, H}, BF16);
  const float* const bias = floats(&a, v[3], {V});
  void* const tokens = a.tensor(v[4], {T, B}, I32);
  const float* const ls = static_cast<const float*>(a.tensor(v[5], {T, B}, F32));
  const float* const ent = floats(&a, v[6], {T, B});
  const float* const d_lp = static_cast<const float*>(a.tensor(v[7], {T, B}, F32));
  const float* const d_ent = floats(&a, v[8], {T, B});
  void* const ws = workspace_here(&a, v[14]);
  const size_t bytes = a.integer(v[15]);
  const auto stream = a.address<vtrace_stream_t>(v[17]);
  if (d_ent != nullptr && ent == nullptr) Py_RETURN_NONE;
  const bool bf16 = v[9] == Py_True;
  Outputs out(3);
  void* const dh = out.add(&a, v[10], true, {T, B, H}, bf16 ? BF16 : F32);
  void* const dw = out.add(&a, v[11], true, {V, H}, bf16 ? BF16 : F32);
  void* const db = out.add(&a, v[12], v[13] == Py_True, {V}, F32);
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(T, B, V, H, bf16 ? VTRACE_BF16 : VTRACE_F32, h->data_ptr(), weight, bias, static_cast<const int32_t*>(tokens),
          ls, ent, d_lp, d_ent, dh, dw, static_cast<float*>(db), ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return out.result(st);
}

// log_prob_loss(fn, target, behaviour, entropy, rewards, discounts, values, bootstrap, lengths, rho_bar,
//               c_bar, lambda, baseline_cost, entropy_cost, variant, losses, d_log_probs, d_values,
//               d_entropy, vs, pg, with_entropy, with_vs, with_pg, workspace, bytes, device, stream)
PyObject* log_prob_loss(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 28 || watched()) Py_RETURN_NONE;
  Args a;
  const at::Tensor* lp = a.first(v[1], 2);
  if (lp == nullptr || lp->scalar_type() != F32 || !on_device(&a, v[26])) Py_RETURN_NONE;
  const int64_t T = lp->size(0), B = lp->size(1);
  const auto fn = a.address<decltype(&vtrace_log_prob_loss_grad)>(v[0]);
  auto need = [&](PyObject* o, std::initializer_list<int64_t> shape) {
    return static_cast<const float*>(a.tensor(o, shape, F32));
  };
  const float* const lm = need(v[2], {T, B});
  const float* const ent = floats(&a, v[3], {T, B});
  const float* const r = need(v[4], {T, B});
  const float* const g = need(v[5], {T, B});
  const float* const val = need(v[6], {T, B});
  const float* const boot = need(v[7], {B});
  const auto lengths = static_cast<const int32_t*>(a.optional(v[8], {B}, I32));
  const float rho = a.number(v[9]), c = a.number(v[10]), lam = a.number(v[11]), bc = a.number(v[12]), ec = a.number(v[13]);
  const auto variant = a.address<const vtrace_variant*>(v[14]);
  void* const ws = workspace_here(&a, v[24]);
  const size_t bytes = a.integer(v[25]);
  const auto stream = a.address<vtrace_stream_t>(v[27]);
  Outputs out(6);
  auto output = [&](int i, bool wanted, std::initializer_list<int64_t> shape) {
    return static_cast<float*>(out.add(&a, v[i], wanted, shape, F32));
  };
  float* const losses = output(15, true, {4});
  float* const d_lp = output(16, true, {T, B});
  float* const d_v = output(17, true, {T, B});
  float* const d_ent = output(18, v[21] == Py_True, {T, B});
  float* const vs = output(19, v[22] == Py_True, {T, B});
  float* const pg = output(20, v[23] == Py_True, {T, B});
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(T, B, static_cast<const float*>(lp->data_ptr()), lm, ent, r, g, val, boot, lengths, rho, c, lam, bc, ec, variant,
          losses, d_lp, d_ent, d_v, vs, pg, ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return out.result(st);
}

// clip(fn, gradients, outputs, scales, max_norm, norm, workspace, bytes, device, stream): gradients a
// list, outputs a list (the gradients' own, to clip in place).
PyObject* clip(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 10 || watched() || !PyList_CheckExact(v[1]) || !PyList_CheckExact(v[2])) Py_RETURN_NONE;
  const Py_ssize_t count = PyList_GET_SIZE(v[1]);
  if (count == 0 || PyList_GET_SIZE(v[2]) != count) Py_RETURN_NONE;
  std::vector<const void*> in(count);
  std::vector<void*> to(count);
  std::vector<int64_t> sizes(count);
  std::vector<int32_t> types(count);
  Args a;
  for (Py_ssize_t i = 0; i < count; ++i) {
    PyObject* const gi = PyList_GET_ITEM(v[1], i);
    PyObject* const oi = PyList_GET_ITEM(v[2], i);
    const at::Tensor* g = plain_tensor(gi);
    const at::Tensor* o = oi == gi ? g : plain_tensor(oi);
    if (g == nullptr || o == nullptr) Py_RETURN_NONE;
    if (i == 0) a.device = g->device();
    vtrace_dtype dt;
    if (!logits_type(*g, &dt) || g->device() != a.device) Py_RETURN_NONE;
    if (o != g && (o->scalar_type() != g->scalar_type() || o->device() != a.device || o->sizes() != g->sizes()))
      Py_RETURN_NONE;
    in[i] = g->data_ptr();
    to[i] = o->data_ptr();
    sizes[i] = g->numel();
    types[i] = dt;
  }
  if (!on_device(&a, v[8])) Py_RETURN_NONE;
  const auto fn = a.address<decltype(&vtrace_clip_grad_norm)>(v[0]);
  const bool scales = v[3] == Py_True;
  const float max_norm = scales ? a.number(v[4]) : 0.0f;
  void* const ws = workspace_here(&a, v[6]);
  const size_t bytes = a.integer(v[7]);
  const auto stream = a.address<vtrace_stream_t>(v[9]);
  Outputs out(1);
  float* const norm = static_cast<float*>(out.add(&a, v[5], true, {}, F32));
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(count, in.data(), scales ? to.data() : nullptr, sizes.data(), types.data(), max_norm, norm, ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return out.result(st);
}

// vocab_embed(fn, weight, tokens, scale, bf16_out, out, workspace, bytes, device, stream)
PyObject* vocab_embed(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 10 || watched()) Py_RETURN_NONE;
  Args a;
  const at::Tensor* w = a.first(v[1], 2);
  const at::Tensor* t = a.ok ? plain_tensor(v[2]) : nullptr;
  vtrace_dtype dt;
  if (w == nullptr || t == nullptr || t->dim() != 2 || !logits_type(*w, &dt) || !on_device(&a, v[8])) Py_RETURN_NONE;
  const int64_t V = w->size(0), H = w->size(1), T = t->size(0), B = t->size(1);
  const auto fn = a.address<decltype(&vtrace_vocab_embed)>(v[0]);
  void* const tokens = a.tensor(v[2], {T, B}, I32);
  const float scale = a.number(v[3]);
  const bool bf16 = v[4] == Py_True;
  void* const ws = v[6] == Py_None ? nullptr : workspace_here(&a, v[6]);
  const size_t bytes = a.integer(v[7]);
  const auto stream = a.address<vtrace_stream_t>(v[9]);
  Outputs out(1);
  void* const rows = out.add(&a, v[5], true, {T, B, H}, bf16 ? BF16 : F32);
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(T, B, V, H, dt, bf16 ? VTRACE_BF16 : VTRACE_F32, w->data_ptr(), static_cast<const int32_t*>(tokens), scale, rows, ws,
          bytes, stream);
  Py_END_ALLOW_THREADS;
  return out.result(st);
}

// vocab_embed_grad(fn, d_embedded, tokens, V, scale, bf16_grad, accumulates, d_weight, workspace, bytes, device,
//                  stream)
PyObject* vocab_embed_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 12 || watched()) Py_RETURN_NONE;
  Args a;
  const at::Tensor* d = a.first(v[1], 3);
  vtrace_dtype dt;
  if (d == nullptr || !logits_type(*d, &dt) || !on_device(&a, v[10])) Py_RETURN_NONE;
  const int64_t T = d->size(0), B = d->size(1), H = d->size(2), V = static_cast<int64_t>(a.integer(v[3]));
  const auto fn = a.address<decltype(&vtrace_vocab_embed_grad)>(v[0]);
  void* const tokens = a.tensor(v[2], {T, B}, I32);
  const float scale = a.number(v[4]);
  const bool bf16 = v[5] == Py_True, accumulates = v[6] == Py_True;
  void* const ws = workspace_here(&a, v[8]);
  const size_t bytes = a.integer(v[9]);
  const auto stream = a.address<vtrace_stream_t>(v[11]);
  if (V < 1 || V > (int64_t(1) << 24) || (accumulates && v[7] == Py_None)) Py_RETURN_NONE;
  Outputs out(1);
  void* const d_weight = out.add(&a, v[7], true, {V, H}, bf16 ? BF16 : F32);
  if (!a.ok) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(T, B, V, H, dt, bf16 ? VTRACE_BF16 : VTRACE_F32, d->data_ptr(), static_cast<const int32_t*>(tokens), scale,
          accumulates ? 1 : 0, d_weight, ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return out.result(st);
}

// orthogonalize(fn, matrices, outputs, scale, steps, coefficients, epsilon, workspace, bytes, device, stream):
// matrices a list, outputs a list or None, coefficients an address.
PyObject* orthogonalize(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 11 || watched() || !PyList_CheckExact(v[1]) || (v[2] != Py_None && !PyList_CheckExact(v[2]))) Py_RETURN_NONE;
  const Py_ssize_t count = PyList_GET_SIZE(v[1]);
  if (count == 0 || (v[2] != Py_None && PyList_GET_SIZE(v[2]) != count)) Py_RETURN_NONE;
  std::vector<const void*> in(count);
  std::vector<void*> to(count);
  std::vector<int64_t> rows(count), columns(count);
  std::vector<int32_t> types(count);
  Args a;
  Outputs out(count);
  for (Py_ssize_t i = 0; i < count; ++i) {
    PyObject* const mi = PyList_GET_ITEM(v[1], i);
    const at::Tensor* m = plain_tensor(mi);
    vtrace_dtype dt;
    if (m == nullptr || m->dim() != 2 || !logits_type(*m, &dt)) Py_RETURN_NONE;
    if (i == 0) {
      a.device = m->device();
      if (!on_device(&a, v[9])) Py_RETURN_NONE;
    }
    if (m->device() != a.device) Py_RETURN_NONE;
    in[i] = m->data_ptr();
    rows[i] = m->size(0);
    columns[i] = m->size(1);
    types[i] = dt;
    to[i] = out.add(&a, v[2] == Py_None ? Py_None : PyList_GET_ITEM(v[2], i), true, {rows[i], columns[i]}, m->scalar_type());
    if (!a.ok) Py_RETURN_NONE;
  }
  const auto fn = a.address<decltype(&vtrace_orthogonalize)>(v[0]);
  const std::vector<float> scales(count, a.number(v[3]));
  const size_t steps = a.integer(v[4]);
  const auto coefficients = a.address<const float*>(v[5]);
  const float epsilon = a.number(v[6]);
  void* const ws = workspace_here(&a, v[7]);
  const size_t bytes = a.integer(v[8]);
  const auto stream = a.address<vtrace_stream_t>(v[10]);
  if (!a.ok || steps > 64) Py_RETURN_NONE;
  vtrace_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(count, in.data(), to.data(), rows.data(), columns.data(), types.data(), scales.data(), static_cast<int32_t>(steps),
          coefficients, epsilon, ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return out.result(st);
}

// A C++ exception (none is expected: every access is checked first) leaves the
// call to the Python path.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* v, Py_ssize_t n) {
  try {
    return F(self, v, n);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

#define METHOD(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(targets),    METHOD(loss),          METHOD(head), METHOD(vocab_log_probs),
                         METHOD(vocab_grad), METHOD(log_prob_loss), METHOD(clip), METHOD(vocab_embed), METHOD(vocab_embed_grad),
                         METHOD(orthogonalize), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast_call(void) { return PyModule_Create(&module); }
