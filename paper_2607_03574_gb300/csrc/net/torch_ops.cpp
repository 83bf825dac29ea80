// The network operators as differentiable PyTorch ops: argument marshalling and autograd nodes around the C
// ABI, in C++ because a node's Python costs more than a small launch (forward and backward on small inputs: dropout 138 us
// from Python, 83 from here, layer norm 178 and 116, gated projection 240 and 140; torch's own product takes 96 to 102).
//
// A function returns None where an argument is not what the operator takes; the Python layer's raw call
// then says what is wrong with it.
#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>

#include "../../../include/ndvm.h"

namespace py = pybind11;
using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

namespace {

using Maybe = std::optional<Tensor>;
Tensor some(const Maybe& t) { return t ? *t : Tensor(); }
Maybe maybe(const Tensor& t) { return t.defined() ? Maybe(t) : Maybe(); }

// sets the package's NdvmError as the pending Python error (with the interpreter's lock)
void set_error(int status, const char* message) {
  py::object type = py::module_::import("paper_2607_03574_gb300").attr("NdvmError");
  py::object e = type(status, message);
  PyErr_SetObject(type.ptr(), e.ptr());
}
[[noreturn]] void raise_forward(int status, const char* message) {  // (in a call from Python)
  py::gil_scoped_acquire lock;
  set_error(status, message);
  throw py::error_already_set();
}
void check_forward(int status) {
  if (status != NDVM_OK) raise_forward(status, ndvm_last_error());
}
[[noreturn]] void raise_backward(int status, const char* message) {  // (in a thread of the autograd engine)
  py::gil_scoped_acquire lock;
  set_error(status, message);
  python_error e;
  e.persist();
  throw std::move(e);
}
void check_backward(int status) {
  if (status != NDVM_OK) raise_backward(status, ndvm_last_error());
}
// Whether one of the tensors has a forward-mode tangent: a launch does not carry it on, and an output without one
// would say that the derivative is 0.
bool tangents(std::initializer_list<const Tensor*> ts) {
  if (!c10::AutogradState::get_tls_state().get_fw_grad_mode()) return false;
  for (const Tensor* t : ts)
    if (t->defined() && t->_fw_grad(0).defined()) return true;
  return false;
}
constexpr const char* kNoTangents = "the network operators have no forward-mode derivatives";
// Whether torch records a program here (torch.jit.trace, or torch.fx's proxies): it would record the allocation of an
// output and not the launch that fills it.
bool traced() {
  if (torch::jit::tracer::isTracing()) return true;
  const c10::DispatchKeySet on = c10::impl::tls_local_dispatch_key_set().included_;
  if (on.has(c10::DispatchKey::PreDispatch)) return true;
  return on.has(c10::DispatchKey::Python) &&  // (a mode of some kind is on)
         c10::impl::TorchDispatchModeTLS::get_mode(c10::impl::TorchDispatchModeKey::PROXY).has_value();
}
constexpr const char* kNoTraces = "the network operators cannot be traced: the trace would not hold their launches";
// what an op refuses of its inputs before it reads them
void check_inputs(std::initializer_list<const Tensor*> ts) {
  if (tangents(ts)) raise_forward(NDVM_E_UNSUPPORTED, kNoTangents);
  if (traced()) raise_forward(NDVM_E_UNSUPPORTED, kNoTraces);
}
// A backward pass records nothing (gradient mode is on in one only to differentiate it again).
void first_order(const Tensor& grad) {
  if (at::GradMode::is_enabled()) raise_backward(NDVM_E_UNSUPPORTED, "the network operators have no second derivatives");
  if (tangents({&grad})) raise_backward(NDVM_E_UNSUPPORTED, kNoTangents);
  if (traced()) raise_backward(NDVM_E_UNSUPPORTED, kNoTraces);
}

int type_code(const Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return NDVM_F32;
    case at::kHalf: return NDVM_F16;
    case at::kBFloat16: return NDVM_BF16;
    default: return -1;
  }
}
bool here(const Tensor& t, int device) { return t.is_cuda() && t.get_device() == device; }

// a tensor as rows of contiguous elements with one stride
struct Rows {
  int64_t rows = 1, cols = 0, stride = 0;
  bool ok = false;
  explicit Rows(const Tensor& t) {
    const int64_t dim = t.dim();
    if (dim == 0) return;
    cols = stride = t.size(dim - 1);
    if (t.is_contiguous()) {
      for (int64_t d = 0; d + 1 < dim; d++) rows *= t.size(d);
      ok = true;
      return;
    }
    bool first = true;
    ok = t.stride(dim - 1) == 1 || cols == 1;
    for (int64_t d = dim - 2; d >= 0; d--) {
      if (t.size(d) == 1) continue;
      if (first) stride = t.stride(d);
      else if (t.stride(d) != stride * rows) ok = false;
      first = false;
      rows *= t.size(d);
    }
    ok &= rows <= 1 || stride == 0 || stride >= cols;  // (rows that overlap, as those of sliding windows, are copied too)
  }
};
// (resolve_neg: the imaginary part of a conjugate is a view whose memory holds the opposite sign)
Tensor resolved(const Tensor& t) { return t.is_neg() ? t.resolve_neg() : t; }
Tensor rowed(const Tensor& t) {
  if (Rows(t).ok && !t.is_neg()) return t;
  return resolved(t.contiguous());
}

void* stream_of(int device) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
const void* in(const Tensor& t) { return t.defined() ? t.const_data_ptr() : nullptr; }
void* out(const Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
Tensor bytes(size_t n, const Tensor& like) {
  return n ? at::empty({(int64_t)n}, like.options().dtype(at::kByte)) : Tensor();
}
bool recorded(std::initializer_list<const Tensor*> ts) {
  if (!at::GradMode::is_enabled()) return false;
  for (const Tensor* t : ts)
    if (t->defined() && t->requires_grad()) return true;
  return false;
}

// ------------------------------------------------------------------------------------ layer norm
Tensor norm_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, double eps, Tensor* stats) {
  const Rows r(x);
  Tensor y = at::empty(x.sizes(), x.options());
  if (stats) *stats = at::empty({2, r.rows}, x.options().dtype(at::kFloat));
  const int wtype = weight.defined() ? type_code(weight) : bias.defined() ? type_code(bias) : type_code(x);
  check_forward(ndvm_layer_norm_forward((ndvm_dtype)type_code(x), (ndvm_dtype)wtype, r.rows, r.cols, in(x), r.stride, in(weight), in(bias), eps,
                                        out(y), r.cols, stats ? static_cast<float*>(out(*stats)) : nullptr, stream_of(x.get_device())));
  return y;
}
struct Norm : torch::autograd::Function<Norm> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Maybe& w, const Maybe& b, double eps) {
    const Tensor weight = some(w), bias = some(b);
    Tensor stats;
    Tensor y = norm_forward(x, weight, bias, eps, &stats);
    ctx->save_for_backward({x, weight, stats});
    if (bias.defined()) ctx->saved_data["bias"] = (int64_t)bias.scalar_type();
    return y;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    first_order(grads[0]);
    const variable_list saved = ctx->get_saved_variables();
    const Tensor &x = saved[0], &weight = saved[1], &stats = saved[2], dy = rowed(grads[0]);
    const Rows r(x);
    const auto bias = ctx->saved_data.find("bias");
    const bool biased = bias != ctx->saved_data.end();
    const auto wtype = weight.defined() ? weight.scalar_type() : biased ? (at::ScalarType)bias->second.toInt() : x.scalar_type();
    Tensor dx, dw, db;  // (the node's inputs are x and those of weight and bias that there are)
    if (ctx->needs_input_grad(0)) dx = at::empty(x.sizes(), x.options());
    if (weight.defined() && ctx->needs_input_grad(1)) dw = at::empty({r.cols}, x.options().dtype(wtype));
    if (biased && ctx->needs_input_grad(weight.defined() ? 2 : 1)) db = at::empty({r.cols}, x.options().dtype(wtype));
    const size_t need = dw.defined() || db.defined() ? ndvm_layer_norm_workspace_bytes(r.rows, r.cols) : 0;
    Tensor ws = bytes(need, x);
    check_backward(ndvm_layer_norm_backward((ndvm_dtype)type_code(x), wtype == at::kFloat ? NDVM_F32 : (ndvm_dtype)type_code(x), r.rows, r.cols,
                                            in(dy), Rows(dy).stride, in(x), r.stride, in(weight), static_cast<const float*>(in(stats)), out(dx),
                                            r.cols, out(dw), out(db), out(ws), need, stream_of(x.get_device())));
    return {dx, dw, db, Tensor()};
  }
};
Maybe layer_norm(const Tensor& given, const Maybe& w, const Maybe& b, double eps) {
  if (!given.is_cuda()) return std::nullopt;
  const int device = c10::cuda::current_device();
  if (!here(given, device) || given.dim() == 0 || type_code(given) < 0) return std::nullopt;
  const Tensor x = rowed(given);
  Tensor weight = some(w), bias = some(b);
  for (Tensor* t : {&weight, &bias}) {
    if (!t->defined()) continue;
    if (!here(*t, device) || t->dim() != 1 || t->size(0) != x.size(-1) || type_code(*t) < 0) return std::nullopt;
    if (!t->is_contiguous() || t->is_neg()) *t = resolved(t->contiguous());
  }
  if (weight.defined() && bias.defined() && weight.scalar_type() != bias.scalar_type()) return std::nullopt;
  check_inputs({&x, &weight, &bias});
  return recorded({&x, &weight, &bias}) ? Norm::apply(x, maybe(weight), maybe(bias), eps) : norm_forward(x, weight, bias, eps, nullptr);
}

// --------------------------------------------------------------------------------------- dropout
Tensor drop(const Tensor& x, double p, uint64_t seed, uint64_t offset, const Tensor& residual, int* status) {
  const Rows r(x);
  Tensor y = at::empty(x.sizes(), x.options());
  *status = ndvm_dropout((ndvm_dtype)type_code(x), r.rows, r.cols, in(x), r.stride, in(residual), residual.defined() ? Rows(residual).stride : 0, p,
                         seed, offset, out(y), r.cols, stream_of(x.get_device()));
  return y;
}
struct Drop : torch::autograd::Function<Drop> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Maybe& residual, double p, uint64_t seed, uint64_t offset) {
    int status;
    Tensor y = drop(x, p, seed, offset, some(residual), &status);
    ctx->saved_data["residual"] = residual.has_value();
    check_forward(status);
    ctx->saved_data["p"] = p;
    ctx->saved_data["seed"] = (int64_t)seed;
    ctx->saved_data["offset"] = (int64_t)offset;
    return y;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    first_order(grads[0]);
    Tensor dx, none;
    if (ctx->needs_input_grad(0)) {
      int status;
      dx = drop(rowed(grads[0]), ctx->saved_data["p"].toDouble(), (uint64_t)ctx->saved_data["seed"].toInt(),
                (uint64_t)ctx->saved_data["offset"].toInt(), none, &status);
      check_backward(status);
    }
    return {dx, ctx->saved_data["residual"].toBool() && ctx->needs_input_grad(1) ? grads[0] : none, none, none, none};
  }
};
Maybe dropout(const Tensor& given, double p, uint64_t seed, uint64_t offset, const Maybe& r) {
  if (!given.is_cuda()) return std::nullopt;
  const int device = c10::cuda::current_device();
  if (!here(given, device) || given.dim() == 0 || type_code(given) < 0) return std::nullopt;
  const Tensor x = rowed(given), residual = r && r->defined() ? rowed(*r) : Tensor();
  if (residual.defined() && (!here(residual, device) || residual.sizes() != x.sizes() || residual.scalar_type() != x.scalar_type())) return std::nullopt;
  check_inputs({&x, &residual});
  if (recorded({&x, &residual})) return Drop::apply(x, maybe(residual), p, seed, offset);
  int status;
  Tensor y = drop(x, p, seed, offset, residual, &status);
  check_forward(status);
  return y;
}

// ------------------------------------------------------------------------------ gated projection
// x and both weights as the C ABI takes them
struct Operands {
  Rows x, g, u;
  const void *px, *pg, *pu;
  bool ready;  // the products can read every one of them where it lies
  Operands(const Tensor& tx, const Tensor& tg, const Tensor& tu) : x(tx), g(tg), u(tu), px(in(tx)), pg(in(tg)), pu(in(tu)) {
    ready = ((uintptr_t)px | (uintptr_t)pg | (uintptr_t)pu) % 16 == 0 && (x.stride | g.stride | u.stride) % 8 == 0 && x.stride && g.stride && u.stride;
  }
};
Tensor gated_forward(const Tensor& x, const Tensor& w_gate, const Tensor& w_up, int64_t act, const Tensor& kept) {
  const Operands o(x, w_gate, w_up);
  const int64_t n = w_gate.size(0);
  auto shape = x.sizes().vec();
  shape.back() = n;
  Tensor h = at::empty(shape, x.options());
  const size_t need = o.ready ? 0 : ndvm_gated_workspace_bytes(o.x.rows, o.x.cols, n, 0, 0);
  Tensor ws = bytes(need, x);
  check_forward(ndvm_gated_forward_keep((ndvm_dtype)type_code(x), (ndvm_activation)act, o.x.rows, o.x.cols, n, o.px, o.x.stride, o.pg, o.g.stride, o.pu,
                                        o.u.stride, out(h), n, static_cast<float*>(out(kept)), out(ws), need, stream_of(x.get_device())));
  return h;
}
struct Gated : torch::autograd::Function<Gated> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& w_gate, const Tensor& w_up, int64_t act, int64_t keep) {
    // The two products are kept (8 bytes an element of h) if the caller says so (keep 1; 0: not), or by default (-1) where
    // that is the faster: a long contraction, or few elements.  Forward and backward, computed again / kept:
    // 16384 x 2048 -> 8192 2660 / 2357 us, 4096 x 2048 -> 8192 648 / 596, 16 x 2048 -> 8192 67 / 57, 1501 x 333 -> 777 49 / 44;
    // but 4096 x 1024 -> 4096 194 / 198, 4096 x 256 -> 1024 47 / 50, 16384 x 1024 -> 4096 687 / 725, 100000 x 256 -> 512
    // 238 / 310.
    const Rows r(x);
    const int64_t n = w_gate.size(0);
    Tensor kept;
    if (keep < 0 ? r.cols >= 1536 || r.rows * n <= (int64_t)1 << 21 : keep > 0)
      kept = at::empty({2, r.rows, ndvm_gated_kept_stride(n)}, x.options().dtype(at::kFloat));
    Tensor h = gated_forward(x, w_gate, w_up, act, kept);
    ctx->save_for_backward({x, w_gate, w_up, kept});
    ctx->saved_data["act"] = act;
    return h;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    first_order(grads[0]);
    const variable_list saved = ctx->get_saved_variables();
    const Tensor &x = saved[0], &w_gate = saved[1], &w_up = saved[2], &kept = saved[3], dh = rowed(grads[0]);
    const Operands o(x, w_gate, w_up);
    const Rows rh(dh);
    const int64_t n = w_gate.size(0);
    Tensor dx, dg, du;
    if (ctx->needs_input_grad(0)) dx = at::empty(x.sizes(), x.options());
    if (ctx->needs_input_grad(1)) dg = at::empty({n, o.x.cols}, x.options());
    if (ctx->needs_input_grad(2)) du = at::empty({n, o.x.cols}, x.options());
    const bool ready = o.ready && (uintptr_t)in(dh) % 16 == 0 && rh.stride % 8 == 0 && rh.stride;
    const size_t need = ndvm_gated_workspace_bytes(o.x.rows, o.x.cols, n, 1, ready);
    Tensor ws = bytes(need, x);
    check_backward(ndvm_gated_backward_kept((ndvm_dtype)type_code(x), (ndvm_activation)ctx->saved_data["act"].toInt(), o.x.rows, o.x.cols, n, in(dh),
                                            rh.stride, o.px, o.x.stride, o.pg, o.g.stride, o.pu, o.u.stride, static_cast<const float*>(in(kept)),
                                            out(dx), o.x.cols, out(dg), out(du), out(ws), need, stream_of(x.get_device())));
    return {dx, dg, du, Tensor(), Tensor()};
  }
};
Maybe gated(const Tensor& gx, const Tensor& gg, const Tensor& gu, int64_t act, int64_t keep) {
  if (!gx.is_cuda()) return std::nullopt;
  const int device = c10::cuda::current_device();
  if (!here(gx, device) || !here(gg, device) || !here(gu, device) || gx.dim() == 0 || gg.dim() != 2 || gu.dim() != 2) return std::nullopt;
  if (gg.sizes() != gu.sizes() || gg.size(1) != gx.size(-1)) return std::nullopt;
  if (act < 0 || type_code(gx) < 0 || gg.scalar_type() != gx.scalar_type() || gu.scalar_type() != gx.scalar_type()) return std::nullopt;
  const Tensor x = rowed(gx), w_gate = rowed(gg), w_up = rowed(gu);
  check_inputs({&x, &w_gate, &w_up});
  return recorded({&x, &w_gate, &w_up}) ? Gated::apply(x, w_gate, w_up, act, keep) : gated_forward(x, w_gate, w_up, act, Tensor());
}

}  // namespace

// (torch's errors as torch raises them)
PYBIND11_MODULE(ndvm_torch, m) {
  m.def("layer_norm", [](const Tensor& x, const Maybe& weight, const Maybe& bias, double eps) {
    HANDLE_TH_ERRORS return layer_norm(x, weight, bias, eps);
    END_HANDLE_TH_ERRORS_PYBIND
  });
  m.def("dropout", [](const Tensor& x, double p, uint64_t seed, uint64_t offset, const Maybe& residual) {
    HANDLE_TH_ERRORS return dropout(x, p, seed, offset, residual);
    END_HANDLE_TH_ERRORS_PYBIND
  });
  m.def("gated", [](const Tensor& x, const Tensor& w_gate, const Tensor& w_up, int64_t act, int64_t keep) {
    HANDLE_TH_ERRORS return gated(x, w_gate, w_up, act, keep);
    END_HANDLE_TH_ERRORS_PYBIND
  });
}
