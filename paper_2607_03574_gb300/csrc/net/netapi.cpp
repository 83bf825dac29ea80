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

// ------------------------------------------------------------------- root-mean-square norm, 8-bit blocks
static constexpr int64_t kBlockMost = (int64_t)1 << 40;  // elements of a row

static const char* blocks(const void* values, int64_t rows, int64_t cols, int64_t v_stride, const void* scales) {
  if (!values || !scales) return "null values or scales of 8-bit blocks";
  if (!aligned(values, 16) || !aligned(scales, 16)) return "values or scales of 8-bit blocks are not 16-byte aligned";
  if (cols > kBlockMost || !spans(rows, cols, v_stride) || (rows > 1 && (v_stride % 16 || v_stride < (cols + 15) / 16 * 16)))
    return "the row stride of 8-bit blocks must be a multiple of 16 that holds a row";
  return nullptr;
}
static const char* kRmsTypes = "rms norm takes F32, F16 and BF16, with weights of the same type or F32";

static ndvm_status rms_forward(RmsArgs& a, ndvm_dtype dtype, ndvm_dtype wtype, double eps, void* stream) {
  if (!is_float(dtype) || (wtype != dtype && wtype != NDVM_F32)) return set_error(NDVM_E_UNSUPPORTED, kRmsTypes);
  if (!sizes(a.rows, a.cols) || a.rows > kNormRows - 127) return bad("bad rows or cols");
  if (!(eps >= 0) || !std::isfinite(eps)) return bad("eps must be finite and not negative");
  if (a.rows == 0) return NDVM_OK;
  REFUSE(matrix_in(a.x, a.rows, a.cols, a.x_stride, dtype));
  if (a.residual) REFUSE(matrix_in(a.residual, a.rows, a.cols, a.r_stride, dtype));
  if (a.sum && !a.residual) return bad("a sum is written where there is a residual");
  if (a.sum) REFUSE(matrix_out(a.sum, a.rows, a.cols, a.sum_stride, dtype));
  REFUSE(vector_in(a.weight, wtype));
  REFUSE(vector_in(a.rstd, NDVM_F32));
  a.eps = (float)eps;
  return done(launch_rms_forward(a, dtype, wtype, (cudaStream_t)stream), "rms norm launch");
}

ndvm_status ndvm_rms_norm_forward(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* x,
                                  int64_t x_stride, const void* residual, int64_t r_stride, const void* weight, double eps,
                                  void* y, int64_t y_stride, void* sum, int64_t sum_stride, float* rstd, void* stream) {
  if (sizes(rows, cols) && rows > 0 && is_float(dtype)) REFUSE(matrix_out(y, rows, cols, y_stride, dtype));
  RmsArgs a{};
  a.rows = rows; a.cols = cols; a.x = x; a.x_stride = x_stride; a.residual = residual; a.r_stride = r_stride; a.weight = weight;
  a.y = y; a.y_stride = y_stride; a.sum = sum; a.sum_stride = sum_stride; a.rstd = rstd;
  return rms_forward(a, dtype, wtype, eps, stream);
}

ndvm_status ndvm_rms_norm_quantized(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* x,
                                    int64_t x_stride, const void* residual, int64_t r_stride, const void* weight, double eps,
                                    uint8_t* values, int64_t v_stride, uint8_t* scales, void* sum, int64_t sum_stride,
                                    void* stream) {
  if (sizes(rows, cols) && rows > 0) REFUSE(blocks(values, rows, cols, v_stride, scales));
  RmsArgs a{};
  a.rows = rows; a.cols = cols; a.x = x; a.x_stride = x_stride; a.residual = residual; a.r_stride = r_stride; a.weight = weight;
  a.values = values; a.v_stride = v_stride; a.v_cols = (cols + 15) / 16 * 16; a.scales = scales; a.sum = sum; a.sum_stride = sum_stride;
  return rms_forward(a, dtype, wtype, eps, stream);
}

size_t ndvm_rms_norm_workspace_bytes(int64_t rows, int64_t cols) { return sizes(rows, cols) ? rms_workspace(rows, cols) : 0; }

ndvm_status ndvm_rms_norm_backward(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* dy,
                                   int64_t dy_stride, const void* dsum, int64_t dsum_stride, const void* s, int64_t s_stride,
                                   const void* weight, const float* rstd, void* dx, int64_t dx_stride, void* dweight,
                                   void* workspace, size_t ws_bytes, void* stream) {
  if (!is_float(dtype) || (wtype != dtype && wtype != NDVM_F32)) return set_error(NDVM_E_UNSUPPORTED, kRmsTypes);
  if (!sizes(rows, cols) || rows > kNormRows) return bad("bad rows or cols");
  if (rows > 0) {
    REFUSE(matrix_in(dy, rows, cols, dy_stride, dtype));
    REFUSE(matrix_in(s, rows, cols, s_stride, dtype));
    if (dsum) REFUSE(matrix_in(dsum, rows, cols, dsum_stride, dtype));
    if (!rstd || !aligned(rstd, 4)) return bad("rstd is null or not aligned");
    if (dx) REFUSE(matrix_out(dx, rows, cols, dx_stride, dtype));
  }
  REFUSE(vector_in(weight, wtype));
  REFUSE(vector_in(dweight, wtype));
  if (dweight && (!workspace || !aligned(workspace, 16) || ws_bytes < rms_workspace(rows, cols)))
    return bad("the workspace is null, not 16-byte aligned or smaller than ndvm_rms_norm_workspace_bytes");
  RmsArgs a{};
  a.rows = rows; a.cols = cols; a.x = s; a.x_stride = s_stride; a.weight = weight; a.rstd = const_cast<float*>(rstd);
  a.dy = dy; a.dy_stride = dy_stride; a.dsum = dsum; a.dsum_stride = dsum_stride; a.dx = dx; a.dx_stride = dx_stride;
  a.dweight = dweight; a.partial = static_cast<float*>(workspace);
  return done(launch_rms_backward(a, dtype, wtype, (cudaStream_t)stream), "rms norm launch");
}

size_t ndvm_quantized_scale_bytes(int64_t rows, int64_t cols) {
  return sizes(rows, cols) && cols <= kBlockMost ? (size_t)((rows + 127) / 128) * (size_t)((cols + 127) / 128) * 512 : 0;
}

static ndvm_status convert(bool back, ndvm_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride,
                           const uint8_t* values, int64_t v_stride, const uint8_t* scales, void* stream) {
  if (!is_float(dtype)) return set_error(NDVM_E_UNSUPPORTED, "8-bit blocks are made of F32, F16 and BF16");
  if (!sizes(rows, cols) || rows > kNormRows - 127) return bad("bad rows or cols");
  if (rows == 0) return NDVM_OK;
  REFUSE(back ? matrix_out(x, rows, cols, x_stride, dtype) : matrix_in(x, rows, cols, x_stride, dtype));
  REFUSE(blocks(values, rows, cols, v_stride, scales));
  RmsArgs a{};
  a.rows = rows; a.cols = cols; a.values = const_cast<uint8_t*>(values); a.v_stride = v_stride; a.v_cols = (cols + 15) / 16 * 16;
  a.scales = const_cast<uint8_t*>(scales);
  if (back) a.y = const_cast<void*>(x), a.y_stride = x_stride;
  else a.x = x, a.x_stride = x_stride;
  return back ? done(launch_dequantize(a, dtype, (cudaStream_t)stream), "dequantize launch")
              : done(launch_quantize(a, dtype, (cudaStream_t)stream), "quantize launch");
}

ndvm_status ndvm_quantize(ndvm_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, uint8_t* values,
                          int64_t v_stride, uint8_t* scales, void* stream) {
  return convert(false, dtype, rows, cols, x, x_stride, values, v_stride, scales, stream);
}

ndvm_status ndvm_dequantize(ndvm_dtype dtype, int64_t rows, int64_t cols, const uint8_t* values, int64_t v_stride,
                            const uint8_t* scales, void* x, int64_t x_stride, void* stream) {
  return convert(true, dtype, rows, cols, x, x_stride, values, v_stride, scales, stream);
}

// ---------------------------------------------------------------------------------------- dense layers
static bool linear_sizes(int64_t rows, int64_t k, int64_t n) {
  return rows >= 0 && k >= 1 && n >= 1 && rows <= kGatedMost && k <= kGatedMost && n <= kGatedMost;
}
static ndvm_status linear_check(ndvm_dtype dtype, ndvm_dtype btype, ndvm_activation act, int64_t rows, int64_t k, int64_t n, const void* bias) {
  if ((dtype != NDVM_F16 && dtype != NDVM_BF16) || (btype != dtype && btype != NDVM_F32))
    return set_error(NDVM_E_UNSUPPORTED, "dense layers take F16 and BF16, with a bias of the same type or F32");
  if (act < NDVM_ACT_SILU || act > NDVM_ACT_NONE) return bad("unknown activation");
  if (!linear_sizes(rows, k, n)) return bad("bad rows, k or n");
  REFUSE(vector_in(bias, btype));
  return NDVM_OK;
}
static const char* linear_room(size_t need, const void* workspace, size_t ws_bytes) {
  return need && (!workspace || !aligned(workspace, 256) || ws_bytes < need)
             ? "the workspace is null, not 256-byte aligned or smaller than its ..._workspace_bytes" : nullptr;
}
// z as it is kept: in binary32 or as 8-bit blocks
static const char* kept_z(LinearArgs& a, float* z, uint8_t* z_values, uint8_t* z_scales) {
  if (z && z_values) return "z is kept in binary32 or as 8-bit blocks, not both";
  if (!aligned(z, 16)) return "z must be 16-byte aligned";
  a.z_pitch = (a.n + 15) / 16 * 16;
  if (z_values || z_scales)
    if (const char* m = blocks(z_values, a.rows, a.n, a.z_pitch, z_scales)) return m;
  a.z = z; a.z_stride = ndvm_linear_kept_stride(a.n);
  a.z_values = z_values; a.z_scales = z_scales;
  return nullptr;
}

int64_t ndvm_linear_kept_stride(int64_t n) { return n < 1 || n > kGatedMost ? 0 : (n + 3) / 4 * 4; }

size_t ndvm_linear_workspace_bytes(ndvm_activation act, int64_t rows, int64_t k, int64_t n, int backward, int aligned, int held) {
  if (!linear_sizes(rows, k, n) || act < NDVM_ACT_SILU || act > NDVM_ACT_NONE) return 0;
  return linear_workspace(rows, k, n, act, backward != 0, !aligned, held != 0);
}

ndvm_status ndvm_linear_forward(ndvm_dtype dtype, ndvm_dtype btype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                const void* x, int64_t x_stride, const void* w, int64_t w_stride, const void* bias,
                                const void* residual, int64_t r_stride, void* y, int64_t y_stride, float* z,
                                uint8_t* z_values, uint8_t* z_scales, void* workspace, size_t ws_bytes, void* stream) {
  if (ndvm_status s = linear_check(dtype, btype, act, rows, k, n, bias)) return s;
  if (rows == 0) return NDVM_OK;
  REFUSE(matrix_in(x, rows, k, x_stride, dtype));
  REFUSE(matrix_in(w, n, k, w_stride, dtype));
  if (residual) REFUSE(matrix_in(residual, rows, n, r_stride, dtype));
  REFUSE(matrix_out(y, rows, n, y_stride, dtype));
  LinearArgs a{};
  a.rows = rows; a.k = k; a.n = n; a.x = x; a.x_stride = x_stride; a.w = w; a.w_stride = w_stride; a.bias = bias;
  a.bias_f32 = btype == NDVM_F32; a.act = act; a.residual = residual; a.r_stride = r_stride; a.y = y; a.y_stride = y_stride;
  a.workspace = workspace;
  REFUSE(kept_z(a, z, z_values, z_scales));
  REFUSE(linear_room(linear_workspace(a, false), workspace, ws_bytes));
  return done(launch_linear_forward(a, dtype, (cudaStream_t)stream), "dense layer launch");
}

ndvm_status ndvm_linear_backward(ndvm_dtype dtype, ndvm_dtype btype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                 const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const uint8_t* x_values,
                                 int64_t xv_stride, const uint8_t* x_scales, const void* w, int64_t w_stride, const float* z,
                                 const uint8_t* z_values, const uint8_t* z_scales, void* dx, int64_t dx_stride, void* dw,
                                 void* dbias, void* workspace, size_t ws_bytes, void* stream) {
  if (ndvm_status s = linear_check(dtype, btype, act, rows, k, n, dbias)) return s;
  REFUSE(vector_in(dw, dtype));
  LinearArgs a{};
  a.rows = rows; a.k = k; a.n = n; a.dy = dy; a.dy_stride = dy_stride; a.x = x; a.x_stride = x_stride; a.x_values = x_values;
  a.xv_stride = xv_stride; a.x_scales = x_scales; a.w = w; a.w_stride = w_stride; a.act = act; a.bias_f32 = btype == NDVM_F32;
  a.dx = dx; a.dx_stride = dx_stride; a.dw = dw; a.dbias = dbias; a.workspace = workspace;
  if (rows > 0) {
    REFUSE(matrix_in(dy, rows, n, dy_stride, dtype));
    if (x && x_values) return bad("x is given as it is or as 8-bit blocks, not both");
    if (dw && x) REFUSE(matrix_in(x, rows, k, x_stride, dtype));
    if (dw && !x) REFUSE(blocks(x_values, rows, k, xv_stride, x_scales));
    if (dx) REFUSE(matrix_in(w, n, k, w_stride, dtype));
    if (dx) REFUSE(matrix_out(dx, rows, k, dx_stride, dtype));
    REFUSE(kept_z(a, const_cast<float*>(z), const_cast<uint8_t*>(z_values), const_cast<uint8_t*>(z_scales)));
    if (act != NDVM_ACT_NONE && !z && !z_values) return bad("the gradients need the z that the forward call kept");
  }
  REFUSE(linear_room(linear_workspace(a, true), workspace, ws_bytes));
  return done(launch_linear_backward(a, dtype, (cudaStream_t)stream), "dense layer launch");
}

size_t ndvm_linear_quantized_workspace_bytes(int64_t rows, int64_t k, int64_t n) {
  return linear_sizes(rows, k, n) ? linear_blocks_workspace(rows, k, n) : 0;
}

ndvm_status ndvm_linear_quantized(ndvm_dtype dtype, ndvm_dtype btype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                  const uint8_t* x_values, int64_t xv_stride, const uint8_t* x_scales,
                                  const uint8_t* w_values, int64_t wv_stride, const uint8_t* w_scales, const void* bias,
                                  const void* residual, int64_t r_stride, void* y, int64_t y_stride, void* workspace,
                                  size_t ws_bytes, void* stream) {
  if (ndvm_status s = linear_check(dtype, btype, act, rows, k, n, bias)) return s;
  if (rows == 0) return NDVM_OK;
  REFUSE(blocks(x_values, rows, k, xv_stride, x_scales));
  REFUSE(blocks(w_values, n, k, wv_stride, w_scales));
  if (residual) REFUSE(matrix_in(residual, rows, n, r_stride, dtype));
  REFUSE(matrix_out(y, rows, n, y_stride, dtype));
  LinearArgs a{};
  a.rows = rows; a.k = k; a.n = n; a.x_values = x_values; a.xv_stride = xv_stride; a.x_scales = x_scales; a.w_values = w_values;
  a.wv_stride = wv_stride; a.w_scales = w_scales; a.bias = bias; a.bias_f32 = btype == NDVM_F32; a.act = act;
  a.residual = residual; a.r_stride = r_stride; a.y = y; a.y_stride = y_stride; a.workspace = workspace;
  REFUSE(linear_room(linear_blocks_workspace(rows, k, n), workspace, ws_bytes));
  return done(launch_linear_blocks(a, dtype, (cudaStream_t)stream), "dense layer launch");
}

ndvm_status ndvm_check_operators(void) {
  int flag = 0, linear = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = product_stopped(&flag);
  if (e == cudaSuccess) e = linear_stopped(&linear);
  if (e != cudaSuccess) return done(e, "read flag");
  return flag || linear ? set_error(NDVM_E_DEVICE_CHECK, "a kernel of the network operators gave up waiting for its operands") : NDVM_OK;
}

}  // extern "C"
