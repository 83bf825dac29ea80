// The network operators as differentiable PyTorch ops: argument marshalling and autograd nodes around the C
// ABI, in C++ because a node's Python costs more than a small launch (forward and backward on small inputs: dropout 138 us
// from Python, 83 from here, layer norm 178 and 116, gated projection 240 and 140; torch's own product takes 96 to 102).
//
// A function returns None where an argument is not what the operator takes; the Python layer's raw call
// then says what is wrong with it.
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <c10/core/InferenceMode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/utils.h>
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

int type_code(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return NDVM_F32;
    case at::kHalf: return NDVM_F16;
    case at::kBFloat16: return NDVM_BF16;
    default: return -1;
  }
}
int type_code(const Tensor& t) { return type_code(t.scalar_type()); }
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
// (in inference mode nothing is, whatever the gradient mode within it: what is made there cannot be held for a backward pass)
bool recorded(std::initializer_list<const Tensor*> ts) {
  if (!at::GradMode::is_enabled() || c10::InferenceMode::is_enabled()) return false;
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
    // 16384 x 2048 -> 8192 2612 / 2270 us, 4096 x 2048 -> 8192 631 / 582, 16 x 2048 -> 8192 69 / 60, 1501 x 333 -> 777 47 / 41;
    // but 4096 x 1024 -> 4096 183 / 192, 4096 x 256 -> 1024 47 / 50, 16384 x 1024 -> 4096 637 / 678, 100000 x 256 -> 512
    // 235 / 307.
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

// ------------------------------------------------------------------------------------- rms norm
// An uninitialised tensor beside `like`, straight from the allocator (dispatching it costs as much again).
Tensor fresh(at::IntArrayRef sizes, const Tensor& like, at::ScalarType type) { return at::detail::empty_cuda(sizes, type, like.device(), std::nullopt); }
Tensor fresh(at::IntArrayRef sizes, const Tensor& like) { return fresh(sizes, like, like.scalar_type()); }

// (x, weight or undefined, residual or undefined) as the operator takes them; false: not its arguments
bool norm_arguments(const Tensor& given, const Maybe& w, const Maybe& r, Tensor* x, Tensor* weight, Tensor* residual) {
  if (!given.is_cuda()) return false;
  const int device = c10::cuda::current_device();
  if (!here(given, device) || given.dim() == 0 || type_code(given) < 0) return false;
  *x = rowed(given);
  *weight = some(w);
  if (weight->defined()) {
    if (!here(*weight, device) || weight->dim() != 1 || weight->size(0) != x->size(-1) || type_code(*weight) < 0) return false;
    if (!weight->is_contiguous() || weight->is_neg()) *weight = resolved(weight->contiguous());
  }
  if (r && r->defined()) {
    if (!here(*r, device) || r->sizes() != x->sizes() || r->scalar_type() != x->scalar_type()) return false;
    *residual = rowed(*r);
  }
  check_inputs({x, weight, residual});
  return true;
}
int weight_code(const Tensor& weight, const Tensor& x) { return weight.defined() ? type_code(weight) : type_code(x); }

// {y} or {y, sum}
variable_list rms_forward(const Tensor& x, const Tensor& weight, const Tensor& residual, double eps, Tensor* rstd) {
  const Rows r(x);
  Tensor y = fresh(x.sizes(), x), sum;
  if (residual.defined()) sum = fresh(x.sizes(), x);
  if (rstd) *rstd = fresh({r.rows}, x, at::kFloat);
  check_forward(ndvm_rms_norm_forward((ndvm_dtype)type_code(x), (ndvm_dtype)weight_code(weight, x), r.rows, r.cols, in(x), r.stride, in(residual),
                                      residual.defined() ? Rows(residual).stride : 0, in(weight), eps, out(y), r.cols, out(sum), r.cols,
                                      rstd ? static_cast<float*>(out(*rstd)) : nullptr, stream_of(x.get_device())));
  return sum.defined() ? variable_list{y, sum} : variable_list{y};
}
// The nodes of the norm and of the dense layers are plain ones: a Function's context costs 10 us more a pass (forward and backward
// on small inputs: norm 131 and 121 us, dense layer 149 and 136; torch's elementwise product 107).  Each is made when its outputs are there;
// edges are those of its inputs in order, undefined ones among them.
using torch::autograd::SavedVariable;
template <typename N>
std::shared_ptr<N> new_node(std::initializer_list<const Tensor*> inputs) {
  std::shared_ptr<N> node(new N(), torch::autograd::deleteNode);
  torch::autograd::edge_list edges;
  edges.reserve(inputs.size());
  for (const Tensor* t : inputs) edges.push_back(t->defined() ? torch::autograd::impl::gradient_edge(*t) : torch::autograd::Edge());
  node->set_next_edges(std::move(edges));
  return node;
}

// What they hold is saved where torch's hooks see it (checkpoints free it and make it again, save_on_cpu moves it away).  A hook
// may give back other memory: here a tensor of the saved one's type and sizes, as the kernels read it (rows with one stride, or, `whole`,
// contiguous from 16 bytes on).
Tensor unpacked(const SavedVariable& v, at::IntArrayRef sizes, at::ScalarType type, at::Device device, bool whole,
                std::shared_ptr<torch::autograd::Node> from = nullptr) {
  const Tensor t = v.unpack(std::move(from));
  if (!t.defined() || t.sizes() != sizes || t.scalar_type() != type || t.device() != device || t.layout() != at::kStrided)
    raise_backward(NDVM_E_INVALID_ARG, "a saved-tensor hook gave back a tensor of another shape, dtype or device");
  if (!whole) return rowed(t);
  return t.is_contiguous() && !t.is_neg() && (uintptr_t)in(t) % 16 == 0 ? t : resolved(t).clone(at::MemoryFormat::Contiguous);
}

struct RmsNormBackward : torch::autograd::Node {
  SavedVariable s, weight, rstd;
  std::vector<int64_t> sizes;  // s's
  at::ScalarType type = at::kFloat, wtype = at::kFloat;
  at::Device device = at::kCUDA;
  bool residual = false, weighted = false;
  std::string name() const override { return "RmsNormBackward"; }
  void release_variables() override {
    std::lock_guard<std::mutex> lock(mutex_);
    for (SavedVariable* v : {&s, &weight, &rstd}) v->reset_data();
  }
  variable_list apply(variable_list&& grads) override {
    std::lock_guard<std::mutex> lock(mutex_);
    for (const Tensor& g : grads)
      if (g.defined()) first_order(g);
    const Tensor dsum = residual && grads[1].defined() ? rowed(grads[1]) : Tensor();
    const bool want_x = task_should_compute_output(0), want_w = weighted && task_should_compute_output(1), want_r = residual && task_should_compute_output(2);
    const Tensor saved = unpacked(s, sizes, type, device, false, residual ? getptr() : nullptr);
    Tensor dx, dw;
    if (want_w) dw = fresh({saved.size(-1)}, saved, wtype);
    if (!grads[0].defined()) {  // (the sum alone has a cotangent, or nothing has)
      if (want_w) dw.zero_();
      dx = residual ? grads[1] : Tensor();
    } else {
      const Rows r(saved);
      const Tensor dy = rowed(grads[0]), stats = unpacked(rstd, r.rows, at::kFloat, device, true);
      Tensor w;
      if (want_x || want_r) {
        dx = fresh(saved.sizes(), saved);
        if (weighted) w = unpacked(weight, sizes.back(), wtype, device, true);
      }
      const size_t need = want_w ? ndvm_rms_norm_workspace_bytes(r.rows, r.cols) : 0;
      Tensor ws = need ? fresh({(int64_t)need}, saved, at::kByte) : Tensor();
      check_backward(ndvm_rms_norm_backward((ndvm_dtype)type_code(saved), (ndvm_dtype)type_code(weighted ? wtype : type), r.rows, r.cols, in(dy), Rows(dy).stride,
                                            in(dsum), dsum.defined() ? Rows(dsum).stride : 0, in(saved), r.stride, in(w),
                                            static_cast<const float*>(in(stats)), out(dx), r.cols, out(dw), out(ws), need,
                                            stream_of(saved.get_device())));
    }
    return {want_x ? dx : Tensor(), dw, want_r ? dx : Tensor()};
  }
};
variable_list rms_recorded(const Tensor& x, const Tensor& weight, const Tensor& residual, double eps) {
  Tensor rstd;
  variable_list y;
  {
    at::AutoDispatchBelowADInplaceOrView below;
    y = rms_forward(x, weight, residual, eps, &rstd);
  }
  const auto node = new_node<RmsNormBackward>({&x, &weight, &residual});
  node->residual = residual.defined();
  node->weighted = weight.defined();
  for (Tensor& t : y) torch::autograd::set_history(t, node);
  node->s = residual.defined() ? SavedVariable(y[1], true) : SavedVariable(x, false);
  node->sizes = x.sizes().vec();
  node->type = x.scalar_type();
  node->device = x.device();
  if (weight.defined()) {  // (its own gradient does not need it)
    node->wtype = weight.scalar_type();
    if (x.requires_grad() || (residual.defined() && residual.requires_grad())) node->weight = SavedVariable(weight, false);
  }
  node->rstd = SavedVariable(rstd, false);
  return y;
}
std::optional<variable_list> rms_norm(const Tensor& given, const Maybe& w, double eps, const Maybe& r) {
  Tensor x, weight, residual;
  if (!norm_arguments(given, w, r, &x, &weight, &residual)) return std::nullopt;
  return recorded({&x, &weight, &residual}) ? rms_recorded(x, weight, residual, eps) : rms_forward(x, weight, residual, eps, nullptr);
}

// --------------------------------------------------------------------------------- 8-bit blocks
constexpr const char* kNoGradient = "the operators on 8-bit blocks have no gradients: call them under torch.no_grad()";
struct Blocks {
  Tensor values, scales;  // values: of the given shape, rows of `stride` bytes
  int64_t rows, cols, stride;
  Blocks(const Tensor& like, at::IntArrayRef sizes, int64_t rows) : rows(rows), cols(sizes.back()), stride((cols + 15) / 16 * 16) {
    if (stride == cols) {
      values = fresh(sizes, like, at::kFloat8_e4m3fn);
    } else {
      auto strides = sizes.vec();
      int64_t step = stride;
      strides.back() = 1;
      for (int64_t d = (int64_t)sizes.size() - 2; d >= 0; d--) strides[d] = step, step *= std::max<int64_t>(sizes[d], 1);
      values = fresh({rows, stride}, like, at::kFloat8_e4m3fn).as_strided(sizes, strides);
    }
    scales = fresh({(rows + 127) / 128, (cols + 127) / 128, 32, 4, 4}, like, at::kByte);
  }
  uint8_t* v() const { return static_cast<uint8_t*>(out(values)); }
  uint8_t* s() const { return static_cast<uint8_t*>(out(scales)); }
};
using Held = std::tuple<Tensor, Tensor, int64_t, int64_t, int64_t>;  // values, scales, rows, cols, stride

// (rows, cols, row stride) of what may be 8-bit blocks, or nothing
std::optional<std::tuple<int64_t, int64_t, int64_t>> blocks_of(const Tensor& values, const Tensor& scales) {
  if (!values.is_cuda() || values.scalar_type() != at::kFloat8_e4m3fn || scales.scalar_type() != at::kByte || scales.device() != values.device()) return std::nullopt;
  const Rows r(values);
  if (!r.ok || (r.rows > 1 && (r.stride % 16 || r.stride < r.cols)) || (uintptr_t)in(values) % 16) return std::nullopt;
  const int64_t shape[5] = {(r.rows + 127) / 128, (r.cols + 127) / 128, 32, 4, 4};
  if (scales.sizes() != at::IntArrayRef(shape) || !scales.is_contiguous() || (uintptr_t)in(scales) % 16) return std::nullopt;
  return std::make_tuple(r.rows, r.cols, r.stride);
}
Blocks to_blocks(const Tensor& x) {
  const Rows r(x);
  Blocks b(x, x.sizes(), r.rows);
  check_forward(ndvm_quantize((ndvm_dtype)type_code(x), r.rows, r.cols, in(x), r.stride, b.v(), b.stride, b.s(), stream_of(x.get_device())));
  return b;
}
std::optional<Held> quantize(const Tensor& given) {
  if (!given.is_cuda()) return std::nullopt;
  if (!here(given, c10::cuda::current_device()) || given.dim() == 0 || type_code(given) < 0) return std::nullopt;
  check_inputs({&given});
  if (recorded({&given})) raise_forward(NDVM_E_UNSUPPORTED, kNoGradient);
  const Tensor x = rowed(given);
  const Blocks b = to_blocks(x);
  return Held{b.values, b.scales, b.rows, b.cols, b.stride};
}
std::optional<std::tuple<Tensor, Tensor, int64_t, int64_t, int64_t, Tensor>> rms_norm_quantized(const Tensor& given, const Maybe& w, double eps,
                                                                                                const Maybe& r) {
  Tensor x, weight, residual, sum;
  if (!norm_arguments(given, w, r, &x, &weight, &residual)) return std::nullopt;
  if (recorded({&x, &weight, &residual})) raise_forward(NDVM_E_UNSUPPORTED, kNoGradient);
  const Rows rows(x);
  const Blocks b(x, x.sizes(), rows.rows);
  if (residual.defined()) sum = fresh(x.sizes(), x);
  check_forward(ndvm_rms_norm_quantized((ndvm_dtype)type_code(x), (ndvm_dtype)weight_code(weight, x), rows.rows, rows.cols, in(x), rows.stride, in(residual),
                                        residual.defined() ? Rows(residual).stride : 0, in(weight), eps, b.v(), b.stride, b.s(), out(sum), rows.cols,
                                        stream_of(x.get_device())));
  return std::make_tuple(b.values, b.scales, b.rows, b.cols, b.stride, sum);
}

// ---------------------------------------------------------------------------------- dense layers
bool ready(const Tensor& t, const Rows& r) { return (uintptr_t)in(t) % 16 == 0 && (r.rows <= 1 || (r.stride % 8 == 0 && r.stride >= r.cols)); }
// bias (n) and residual (sizes) of a dense layer whose y has that type
bool linear_extras(int device, const Maybe& b, const Maybe& r, int64_t n, at::IntArrayRef sizes, at::ScalarType type, Tensor* bias, Tensor* residual) {
  *bias = some(b);
  if (bias->defined()) {
    if (!here(*bias, device) || bias->dim() != 1 || bias->size(0) != n || (bias->scalar_type() != type && bias->scalar_type() != at::kFloat)) return false;
    if (!bias->is_contiguous() || bias->is_neg()) *bias = resolved(bias->contiguous());
  }
  if (r && r->defined()) {
    if (!here(*r, device) || r->sizes() != sizes || r->scalar_type() != type) return false;
    *residual = rowed(*r);
  }
  return true;
}
// z: where it is kept, as floats, or beside scales as the bytes of blocks
Tensor linear_forward(const Tensor& x, const Tensor& w, const Tensor& bias, int64_t act, const Tensor& residual, const Tensor& z,
                      const Tensor& z_scales) {
  const Rows rx(x), rw(w);
  const int64_t n = w.size(0);
  auto shape = x.sizes().vec();
  shape.back() = n;
  Tensor y = fresh(shape, x);
  // (one row without blocks takes no workspace, whatever its operands start on)
  const size_t need = rx.rows == 1 && !z_scales.defined() ? 0
                      : ndvm_linear_workspace_bytes((ndvm_activation)act, rx.rows, rx.cols, n, 0, ready(x, rx) && ready(w, rw), 0);
  Tensor ws = need ? fresh({(int64_t)need}, x, at::kByte) : Tensor();
  check_forward(ndvm_linear_forward((ndvm_dtype)type_code(x), (ndvm_dtype)weight_code(bias, x), (ndvm_activation)act, rx.rows, rx.cols, n, in(x), rx.stride,
                                    in(w), rw.stride, in(bias), in(residual), residual.defined() ? Rows(residual).stride : 0, out(y), n,
                                    z_scales.defined() ? nullptr : static_cast<float*>(out(z)), z_scales.defined() ? static_cast<uint8_t*>(out(z)) : nullptr,
                                    static_cast<uint8_t*>(out(z_scales)), out(ws), need, stream_of(x.get_device())));
  return y;
}
// 8-bit blocks as a node holds them: bytes, in rows of whole 16s
struct HeldBlocks {
  Tensor values, scales;
  static int64_t pitch(int64_t cols) { return (cols + 15) / 16 * 16; }
  static std::array<int64_t, 2> value_sizes(int64_t rows, int64_t cols) { return {rows, pitch(cols)}; }
  static std::array<int64_t, 5> scale_sizes(int64_t rows, int64_t cols) { return {(rows + 127) / 128, (cols + 127) / 128, 32, 4, 4}; }
  HeldBlocks(const Tensor& like, int64_t rows, int64_t cols)
      : values(fresh(value_sizes(rows, cols), like, at::kByte)), scales(fresh(scale_sizes(rows, cols), like, at::kByte)) {}
};
struct LinearBackward : torch::autograd::Node {
  SavedVariable x, w, z;        // (x and z: as they are, or the bytes of their blocks)
  SavedVariable x_scales, z_scales;
  std::vector<int64_t> sizes;  // x's
  int64_t act = 0;
  at::ScalarType btype = at::kFloat;
  bool eight = false, biased = false, wants_z = false;
  std::string name() const override { return "LinearBackward"; }
  void release_variables() override {
    std::lock_guard<std::mutex> lock(mutex_);
    for (SavedVariable* v : {&x, &w, &z, &x_scales, &z_scales}) v->reset_data();
  }
  variable_list apply(variable_list&& grads) override {
    std::lock_guard<std::mutex> lock(mutex_);
    if (!grads[0].defined()) return {Tensor(), Tensor(), Tensor(), Tensor()};
    first_order(grads[0]);
    const Tensor dy = rowed(grads[0]);
    const Rows rd(dy);
    const int64_t rows = rd.rows, n = dy.size(-1), k = sizes.back();
    const at::ScalarType type = dy.scalar_type();
    Tensor dx, dw, db;
    if (task_should_compute_output(0)) dx = fresh(sizes, dy);
    if (task_should_compute_output(1)) dw = fresh({n, k}, dy);
    if (biased && task_should_compute_output(2)) db = fresh({n}, dy, btype);
    if (dx.defined() || dw.defined() || db.defined()) {
      Tensor weight, given, values, scales, held_z, held_scales;  // w; x, or its blocks; z, or its blocks
      if (dx.defined()) weight = unpacked(w, {n, k}, type, dy.device(), false);
      if (dw.defined() && !eight) given = unpacked(x, sizes, type, dy.device(), false);
      if (dw.defined() && eight) {
        values = unpacked(x, HeldBlocks::value_sizes(rows, k), at::kByte, dy.device(), true);
        scales = unpacked(x_scales, HeldBlocks::scale_sizes(rows, k), at::kByte, dy.device(), true);
      }
      if (wants_z && eight) {
        held_z = unpacked(z, HeldBlocks::value_sizes(rows, n), at::kByte, dy.device(), true);
        held_scales = unpacked(z_scales, HeldBlocks::scale_sizes(rows, n), at::kByte, dy.device(), true);
      } else if (wants_z) {
        held_z = unpacked(z, {rows, ndvm_linear_kept_stride(n)}, at::kFloat, dy.device(), true);
      }
      std::optional<Rows> rx, rw;
      if (given.defined()) rx.emplace(given);
      if (weight.defined()) rw.emplace(weight);
      const size_t need = ndvm_linear_workspace_bytes((ndvm_activation)act, rows, k, n, 1,
                                                      (!rx || ready(given, *rx)) && (!rw || ready(weight, *rw)) && ready(dy, rd), values.defined());
      Tensor ws = need ? fresh({(int64_t)need}, dy, at::kByte) : Tensor();
      check_backward(ndvm_linear_backward(
          (ndvm_dtype)type_code(dy), db.defined() && btype == at::kFloat ? NDVM_F32 : (ndvm_dtype)type_code(dy), (ndvm_activation)act, rows, k, n,
          in(dy), rd.stride, in(given), rx ? rx->stride : 0, static_cast<const uint8_t*>(in(values)), HeldBlocks::pitch(k),
          static_cast<const uint8_t*>(in(scales)), in(weight), rw ? rw->stride : 0, eight ? nullptr : static_cast<const float*>(in(held_z)),
          eight ? static_cast<const uint8_t*>(in(held_z)) : nullptr, static_cast<const uint8_t*>(in(held_scales)), out(dx), k, out(dw), out(db), out(ws),
          need, stream_of(dy.get_device())));
    }
    return {dx, dw, db, task_should_compute_output(3) ? grads[0] : Tensor()};
  }
};
Tensor linear_recorded(const Tensor& x, const Tensor& w, const Tensor& bias, const Tensor& residual, int64_t act, bool eight) {
  const Rows rx(x);
  const int64_t n = w.size(0);
  // what the gradients need: z of an activation, x for w's, and w for x's
  const bool wants_w = w.requires_grad();
  const bool wants_z = act != NDVM_ACT_NONE && (wants_w || x.requires_grad() || (bias.defined() && bias.requires_grad()));
  Tensor y, z, z_scales;
  std::optional<HeldBlocks> held;
  {
    at::AutoDispatchBelowADInplaceOrView below;
    if (eight && wants_w) {
      held.emplace(x, rx.rows, rx.cols);
      check_forward(ndvm_quantize((ndvm_dtype)type_code(x), rx.rows, rx.cols, in(x), rx.stride, static_cast<uint8_t*>(out(held->values)),
                                  HeldBlocks::pitch(rx.cols), static_cast<uint8_t*>(out(held->scales)), stream_of(x.get_device())));
    }
    if (eight && wants_z) {
      HeldBlocks blocks(x, rx.rows, n);
      z = blocks.values, z_scales = blocks.scales;
    } else if (wants_z) {
      z = fresh({rx.rows, ndvm_linear_kept_stride(n)}, x, at::kFloat);
    }
    y = linear_forward(x, w, bias, act, residual, z, z_scales);
  }
  const auto node = new_node<LinearBackward>({&x, &w, &bias, &residual});
  torch::autograd::set_history(y, node);
  if (x.requires_grad()) node->w = SavedVariable(w, false);
  if (held) node->x = SavedVariable(held->values, false), node->x_scales = SavedVariable(held->scales, false);
  else if (wants_w) node->x = SavedVariable(x, false);
  if (wants_z) node->z = SavedVariable(z, false);
  if (z_scales.defined()) node->z_scales = SavedVariable(z_scales, false);
  node->sizes = x.sizes().vec();
  node->act = act;
  node->eight = eight;
  node->wants_z = wants_z;
  if ((node->biased = bias.defined())) node->btype = bias.scalar_type();
  return y;
}
Maybe linear(const Tensor& gx, const Tensor& gw, const Maybe& b, int64_t act, const Maybe& r, bool eight) {
  if (!gx.is_cuda()) return std::nullopt;
  const int device = c10::cuda::current_device();
  if (!here(gx, device) || !here(gw, device) || gx.dim() == 0 || gw.dim() != 2 || gw.size(1) != gx.size(-1)) return std::nullopt;
  if (type_code(gx) <= NDVM_F32 || gw.scalar_type() != gx.scalar_type()) return std::nullopt;
  auto shape = gx.sizes().vec();
  shape.back() = gw.size(0);
  Tensor bias, residual;
  if (!linear_extras(device, b, r, gw.size(0), shape, gx.scalar_type(), &bias, &residual)) return std::nullopt;
  const Tensor x = rowed(gx), w = rowed(gw);
  check_inputs({&x, &w, &bias, &residual});
  if (recorded({&x, &w, &bias, &residual})) return linear_recorded(x, w, bias, residual, act, eight);
  return linear_forward(x, w, bias, act, residual, Tensor(), Tensor());
}
Maybe linear_quantized(const Tensor& xv, const Tensor& xs, int64_t rows, int64_t k, int64_t x_stride, const Tensor& wv, const Tensor& ws, int64_t n,
                       int64_t wk, int64_t w_stride, const Maybe& b, int64_t act, const Maybe& r, int64_t code) {
  const int device = c10::cuda::current_device();
  if (!here(xv, device) || !here(wv, device) || wv.dim() != 2 || wk != k || (code != NDVM_F16 && code != NDVM_BF16)) return std::nullopt;
  const at::ScalarType type = code == NDVM_F16 ? at::kHalf : at::kBFloat16;
  auto shape = xv.sizes().vec();
  shape.back() = n;
  Tensor bias, residual;
  if (!linear_extras(device, b, r, n, shape, type, &bias, &residual)) return std::nullopt;
  check_inputs({&xv, &wv, &bias, &residual});
  if (recorded({&bias, &residual})) raise_forward(NDVM_E_UNSUPPORTED, kNoGradient);
  Tensor y = fresh(shape, xv, type);
  const size_t need = ndvm_linear_quantized_workspace_bytes(rows, k, n);
  Tensor room = need ? fresh({(int64_t)need}, xv, at::kByte) : Tensor();
  check_forward(ndvm_linear_quantized((ndvm_dtype)type_code(y), (ndvm_dtype)weight_code(bias, y), (ndvm_activation)act, rows, k, n,
                                      static_cast<const uint8_t*>(in(xv)), x_stride, static_cast<const uint8_t*>(in(xs)),
                                      static_cast<const uint8_t*>(in(wv)), w_stride, static_cast<const uint8_t*>(in(ws)), in(bias), in(residual),
                                      residual.defined() ? Rows(residual).stride : 0, out(y), n, out(room), need, stream_of(device)));
  return y;
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
  m.def("rms_norm", [](const Tensor& x, const Maybe& weight, double eps, const Maybe& residual) {
    HANDLE_TH_ERRORS return rms_norm(x, weight, eps, residual);
    END_HANDLE_TH_ERRORS_PYBIND
  });
  m.def("quantize", [](const Tensor& x) {
    HANDLE_TH_ERRORS return quantize(x);
    END_HANDLE_TH_ERRORS_PYBIND
  });
  m.def("blocks_of", [](const Tensor& values, const Tensor& scales) {
    HANDLE_TH_ERRORS return blocks_of(values, scales);
    END_HANDLE_TH_ERRORS_PYBIND
  });
  m.def("rms_norm_quantized", [](const Tensor& x, const Maybe& weight, double eps, const Maybe& residual) {
    HANDLE_TH_ERRORS return rms_norm_quantized(x, weight, eps, residual);
    END_HANDLE_TH_ERRORS_PYBIND
  });
  m.def("linear", [](const Tensor& x, const Tensor& w, const Maybe& bias, int64_t act, const Maybe& residual, bool eight) {
    HANDLE_TH_ERRORS return linear(x, w, bias, act, residual, eight);
    END_HANDLE_TH_ERRORS_PYBIND
  });
  m.def("linear_quantized", [](const Tensor& xv, const Tensor& xs, int64_t rows, int64_t k, int64_t x_stride, const Tensor& wv, const Tensor& ws, int64_t n,
                               int64_t wk, int64_t w_stride, const Maybe& bias, int64_t act, const Maybe& residual, int64_t type) {
    HANDLE_TH_ERRORS return linear_quantized(xv, xs, rows, k, x_stride, wv, ws, n, wk, w_stride, bias, act, residual, type);
    END_HANDLE_TH_ERRORS_PYBIND
  });
}
