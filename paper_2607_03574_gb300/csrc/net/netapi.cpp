// C ABI of the network operators: argument checks, then one launcher each.
#include <cmath>
#include <cstdio>

#include "net.h"

using namespace ndvm;

namespace {

ndvm_status bad(const char* m) { return set_error(NDVM_E_INVALID_ARG, m); }

ndvm_status done(cudaError_t e, const char* where) {
  if (e == cudaSuccess) return NDVM_OK;
  char m[256];
  std::snprintf(m, sizeof m, "%s: %s", where, cudaGetErrorString(e));
  return set_error(e == cudaErrorMemoryAllocation ? NDVM_E_OOM : NDVM_E_CUDA, m);
}

size_t size_of(ndvm_dtype t) { return t == NDVM_F32 ? 4 : 2; }
bool is_float(ndvm_dtype t) { return t == NDVM_F32 || t == NDVM_F16 || t == NDVM_BF16; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

constexpr int64_t kMost = (int64_t)1 << 48;  // elements a matrix spans at most
constexpr int64_t kNormRows = ((int64_t)1 << 31) - 1;  // a block or more of them a launch

bool spans(int64_t rows, int64_t cols, int64_t stride) {
  return stride >= 0 && (rows <= 1 || stride <= kMost / rows) && cols <= kMost;
}
// an input's rows may all be the same memory; an output's are apart
const char* matrix_in(const void* p, int64_t rows, int64_t cols, int64_t stride, ndvm_dtype t) {
  if (!p) return "null input";
  if (!aligned(p, size_of(t))) return "an input is not aligned to its element type";
  if (!spans(rows, cols, stride) || (rows > 1 && stride != 0 && stride < cols)) return "bad row stride of an input";
  return nullptr;
}
const char* matrix_out(const void* p, int64_t rows, int64_t cols, int64_t stride, ndvm_dtype t) {
  if (!p) return "null output";
  if (!aligned(p, size_of(t))) return "an output is not aligned to its element type";
  if (!spans(rows, cols, stride) || (rows > 1 && stride < cols)) return "bad row stride of an output";
  return nullptr;
}
const char* vector_in(const void* p, ndvm_dtype t) {
  return p && !aligned(p, size_of(t)) ? "a vector is not aligned to its element type" : nullptr;
}
bool sizes(int64_t rows, int64_t cols) {
  return rows >= 0 && cols >= 1 && rows <= kMost && cols <= kMost && (rows == 0 || cols <= kMost / rows);
}

#define REFUSE(expr) \
  if (const char* m_ = (expr)) return bad(m_)

}  // namespace

extern "C" {

ndvm_status ndvm_layer_norm_forward(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* x,
                                    int64_t x_stride, const void* weight, const void* bias, double eps, void* y,
                                    int64_t y_stride, float* stats, void* stream) {
  if (!is_float(dtype) || (wtype != dtype && wtype != NDVM_F32))
    return set_error(NDVM_E_UNSUPPORTED, "layer norm takes F32, F16 and BF16, with weights of the same type or F32");
  if (!sizes(rows, cols) || rows > kNormRows) return bad("bad rows or cols");
  if (!(eps >= 0) || !std::isfinite(eps)) return bad("eps must be finite and not negative");
  if (rows == 0) return NDVM_OK;
  REFUSE(matrix_in(x, rows, cols, x_stride, dtype));
  REFUSE(matrix_out(y, rows, cols, y_stride, dtype));
  REFUSE(vector_in(weight, wtype));
  REFUSE(vector_in(bias, wtype));
  REFUSE(vector_in(stats, NDVM_F32));
  NormArgs a{};
  a.rows = rows; a.cols = cols; a.x = x; a.x_stride = x_stride; a.weight = weight; a.bias = bias;
  a.eps = (float)eps; a.y = y; a.y_stride = y_stride; a.stats = stats;
  return done(launch_norm_forward(a, dtype, wtype, (cudaStream_t)stream), "layer norm launch");
}

size_t ndvm_layer_norm_workspace_bytes(int64_t rows, int64_t cols) { return sizes(rows, cols) ? norm_workspace(rows, cols) : 0; }

ndvm_status ndvm_layer_norm_backward(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* dy,
                                     int64_t dy_stride, const void* x, int64_t x_stride, const void* weight,
                                     const float* stats, void* dx, int64_t dx_stride, void* dweight, void* dbias,
                                     void* workspace, size_t ws_bytes, void* stream) {
  if (!is_float(dtype) || (wtype != dtype && wtype != NDVM_F32))
    return set_error(NDVM_E_UNSUPPORTED, "layer norm takes F32, F16 and BF16, with weights of the same type or F32");
  if (!sizes(rows, cols) || rows > kNormRows) return bad("bad rows or cols");
  if (rows > 0) {
    REFUSE(matrix_in(dy, rows, cols, dy_stride, dtype));
    REFUSE(matrix_in(x, rows, cols, x_stride, dtype));
    if (!stats || !aligned(stats, 4)) return bad("stats is null or not aligned");
    if (dx) REFUSE(matrix_out(dx, rows, cols, dx_stride, dtype));
  }
  REFUSE(vector_in(weight, wtype));
  REFUSE(vector_in(dweight, wtype));
  REFUSE(vector_in(dbias, wtype));
  if ((dweight || dbias) && (!workspace || !aligned(workspace, 16) || ws_bytes < norm_workspace(rows, cols)))
    return bad("the workspace is null, not 16-byte aligned or smaller than ndvm_layer_norm_workspace_bytes");
  NormArgs a{};
  a.rows = rows; a.cols = cols; a.x = x; a.x_stride = x_stride; a.weight = weight;
  a.stats = const_cast<float*>(stats); a.dy = dy; a.dy_stride = dy_stride; a.dx = dx; a.dx_stride = dx_stride;
  a.dweight = dweight; a.dbias = dbias; a.partial = static_cast<float*>(workspace);
  return done(launch_norm_backward(a, dtype, wtype, (cudaStream_t)stream), "layer norm launch");
}

ndvm_status ndvm_dropout(ndvm_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride,
                         const void* residual, int64_t r_stride, double p, uint64_t seed, uint64_t offset, void* y,
                         int64_t y_stride, void* stream) {
  if (!is_float(dtype)) return set_error(NDVM_E_UNSUPPORTED, "dropout takes F32, F16 and BF16");
  if (rows < 0 || cols < 0 || rows > kMost || cols > kMost || (rows > 0 && cols > kMost / rows)) return bad("bad rows or cols");
  if (!(p >= 0 && p <= 1 - 0x1p-32)) return bad("p must be in [0, 1 - 2^-32]");
  if (offset % 4) return bad("offset must be a multiple of 4");
  if (rows == 0 || cols == 0) return NDVM_OK;
  REFUSE(matrix_in(x, rows, cols, x_stride, dtype));
  if (residual) REFUSE(matrix_in(residual, rows, cols, r_stride, dtype));
  REFUSE(matrix_out(y, rows, cols, y_stride, dtype));
  DropArgs a{};
  a.rows = rows; a.cols = cols; a.x = x; a.x_stride = x_stride; a.residual = residual; a.r_stride = r_stride;
  a.y = y; a.y_stride = y_stride; a.seed = seed; a.offset = offset;
  a.threshold = (uint32_t)std::llrint(p * 0x1p32);
  a.scale = (float)(1.0 / (1.0 - p));
  return done(launch_dropout(a, dtype, (cudaStream_t)stream), "dropout launch");
}

static constexpr int64_t kGatedMost = (int64_t)1 << 28;  // rows, k and n (a tile's coordinates are 32-bit, its sum's time bounded)

static ndvm_status gated_check(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n, const void* x,
                               int64_t x_stride, const void* w_gate, int64_t g_stride, const void* w_up, int64_t u_stride) {
  if (dtype != NDVM_F16 && dtype != NDVM_BF16) return set_error(NDVM_E_UNSUPPORTED, "the gated projection takes F16 and BF16");
  if (act < NDVM_ACT_SILU || act > NDVM_ACT_SIGMOID) return bad("unknown activation");
  if (rows < 0 || k < 1 || n < 1 || rows > kGatedMost || k > kGatedMost || n > kGatedMost) return bad("bad rows, k or n");
  if (rows > 0) REFUSE(matrix_in(x, rows, k, x_stride, dtype));
  REFUSE(matrix_in(w_gate, n, k, g_stride, dtype));
  REFUSE(matrix_in(w_up, n, k, u_stride, dtype));
  return NDVM_OK;
}

static const char* gated_room(const GatedArgs& a, bool backward, const void* workspace, size_t ws_bytes) {
  const size_t need = gated_workspace(a, backward);
  return need && (!workspace || !aligned(workspace, 256) || ws_bytes < need)
             ? "the workspace is null, not 256-byte aligned or smaller than ndvm_gated_workspace_bytes" : nullptr;
}

size_t ndvm_gated_workspace_bytes(int64_t rows, int64_t k, int64_t n, int backward, int aligned) {
  if (rows < 0 || k < 1 || n < 1 || rows > kGatedMost || k > kGatedMost || n > kGatedMost) return 0;
  return gated_workspace(rows, k, n, backward != 0, !aligned);
}

int64_t ndvm_gated_kept_stride(int64_t n) { return n < 1 || n > kGatedMost ? 0 : (n + 3) / 4 * 4; }

ndvm_status ndvm_gated_forward(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n, const void* x,
                               int64_t x_stride, const void* w_gate, int64_t g_stride, const void* w_up,
                               int64_t u_stride, void* h, int64_t h_stride, void* workspace, size_t ws_bytes,
                               void* stream) {
  return ndvm_gated_forward_keep(dtype, act, rows, k, n, x, x_stride, w_gate, g_stride, w_up, u_stride, h, h_stride, nullptr,
                                 workspace, ws_bytes, stream);
}

ndvm_status ndvm_gated_forward_keep(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                    const void* x, int64_t x_stride, const void* w_gate, int64_t g_stride,
                                    const void* w_up, int64_t u_stride, void* h, int64_t h_stride, float* kept,
                                    void* workspace, size_t ws_bytes, void* stream) {
  if (ndvm_status s = gated_check(dtype, act, rows, k, n, x, x_stride, w_gate, g_stride, w_up, u_stride)) return s;
  if (!aligned(kept, 16)) return bad("kept must be 16-byte aligned");
  if (rows == 0) return NDVM_OK;
  REFUSE(matrix_out(h, rows, n, h_stride, dtype));
  GatedArgs a{};
  a.rows = rows; a.k = k; a.n = n; a.x = x; a.x_stride = x_stride; a.w_gate = w_gate; a.w_up = w_up;
  a.g_stride = g_stride; a.u_stride = u_stride; a.act = act; a.h = h; a.h_stride = h_stride; a.workspace = workspace;
  a.kept = kept; a.kept_stride = ndvm_gated_kept_stride(n);
  REFUSE(gated_room(a, false, workspace, ws_bytes));
  return done(launch_gated_forward(a, dtype, (cudaStream_t)stream), "gated projection launch");
}

ndvm_status ndvm_gated_backward(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                const void* dh, int64_t dh_stride, const void* x, int64_t x_stride, const void* w_gate,
                                int64_t g_stride, const void* w_up, int64_t u_stride, void* dx, int64_t dx_stride,
                                void* dw_gate, void* dw_up, void* workspace, size_t ws_bytes, void* stream) {
  return ndvm_gated_backward_kept(dtype, act, rows, k, n, dh, dh_stride, x, x_stride, w_gate, g_stride, w_up, u_stride, nullptr,
                                  dx, dx_stride, dw_gate, dw_up, workspace, ws_bytes, stream);
}

ndvm_status ndvm_gated_backward_kept(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                     const void* dh, int64_t dh_stride, const void* x, int64_t x_stride,
                                     const void* w_gate, int64_t g_stride, const void* w_up, int64_t u_stride,
                                     const float* kept, void* dx, int64_t dx_stride, void* dw_gate, void* dw_up,
                                     void* workspace, size_t ws_bytes, void* stream) {
  if (ndvm_status s = gated_check(dtype, act, rows, k, n, x, x_stride, w_gate, g_stride, w_up, u_stride)) return s;
  if (rows > 0) {
    REFUSE(matrix_in(dh, rows, n, dh_stride, dtype));
    if (dx) REFUSE(matrix_out(dx, rows, k, dx_stride, dtype));
  }
  REFUSE(vector_in(dw_gate, dtype));
  REFUSE(vector_in(dw_up, dtype));
  if (!aligned(kept, 16)) return bad("kept must be 16-byte aligned");
  GatedArgs a{};
  a.rows = rows; a.k = k; a.n = n; a.x = x; a.x_stride = x_stride; a.w_gate = w_gate; a.w_up = w_up;
  a.g_stride = g_stride; a.u_stride = u_stride; a.act = act; a.dh = dh; a.dh_stride = dh_stride; a.dx = dx;
  a.dx_stride = dx_stride; a.dw_gate = dw_gate; a.dw_up = dw_up; a.workspace = workspace;
  a.kept = const_cast<float*>(kept); a.kept_stride = ndvm_gated_kept_stride(n);
  REFUSE(gated_room(a, true, workspace, ws_bytes));
  return done(launch_gated_backward(a, dtype, (cudaStream_t)stream), "gated projection launch");
}

ndvm_status ndvm_check_operators(void) {
  int flag = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = gated_stopped(&flag);
  if (e != cudaSuccess) return done(e, "read flag");
  return flag ? set_error(NDVM_E_DEVICE_CHECK, "a kernel of the gated projection gave up waiting for its operands") : NDVM_OK;
}

}  // extern "C"
