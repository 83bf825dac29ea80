// Network operators: layer norm, dropout and the gated projection (launchers; the C ABI is netapi.cpp).
// Rows are strided (strides in elements), a row's elements are contiguous.
#pragma once
#include <cuda_runtime.h>

#include "../status.h"

namespace ndvm {

constexpr int kSms = 152;

struct NormArgs {
  int64_t rows, cols;
  const void* x; int64_t x_stride;
  const void* weight; const void* bias;  // null: 1 and 0
  float eps;
  float* stats;                          // [2][rows]: mean, 1 / sqrt(variance + eps)
  void* y; int64_t y_stride;
  // backward
  const void* dy; int64_t dy_stride;
  void* dx; int64_t dx_stride;           // null: not wanted
  void* dweight; void* dbias;            // null: not wanted
  float* partial;                        // workspace: column sums of each block
};
cudaError_t launch_norm_forward(const NormArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s);
cudaError_t launch_norm_backward(const NormArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s);
size_t norm_workspace(int64_t rows, int64_t cols);

// Root-mean-square norm, and 8-bit blocks.
struct RmsArgs {
  int64_t rows, cols;
  const void* x; int64_t x_stride;         // (backward: s)
  const void* residual; int64_t r_stride;  // null: none
  const void* weight;                      // null: 1
  float eps;
  float* rstd;                             // 1 / sqrt(mean(s^2) + eps), or null
  void* sum; int64_t sum_stride;           // s, or null
  void* y; int64_t y_stride;
  uint8_t* values; int64_t v_stride, v_cols;  // blocks instead of y: e4m3 values (v_cols: cols up to a multiple of 16)
  uint8_t* scales;
  // backward
  const void* dy; int64_t dy_stride;
  const void* dsum; int64_t dsum_stride;   // null: 0
  void* dx; int64_t dx_stride;             // null: not wanted
  void* dweight;                           // null: not wanted
  float* partial;                          // workspace: column sums of each block
};
cudaError_t launch_rms_forward(const RmsArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s);
cudaError_t launch_rms_backward(const RmsArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s);
size_t rms_workspace(int64_t rows, int64_t cols);
cudaError_t launch_quantize(const RmsArgs& a, ndvm_dtype t, cudaStream_t s);    // x to values and scales
cudaError_t launch_dequantize(const RmsArgs& a, ndvm_dtype t, cudaStream_t s);  // and back to y

struct DropArgs {
  int64_t rows, cols;
  const void* x; int64_t x_stride;
  const void* residual; int64_t r_stride;  // null: none
  void* y; int64_t y_stride;
  uint32_t threshold;                      // an element whose word is below is dropped
  float scale;
  uint64_t seed, offset;
};
cudaError_t launch_dropout(const DropArgs& a, ndvm_dtype t, cudaStream_t s);

// Dense layer y = act(x w^T + bias) + residual, of 16-bit operands or of 8-bit blocks.
struct LinearArgs {
  int64_t rows, k, n;
  const void* x; int64_t x_stride;         // (backward: null if it is held as blocks)
  const void* w; int64_t w_stride;
  const void* bias; bool bias_f32;         // null: 0
  ndvm_activation act;
  const void* residual; int64_t r_stride;  // null: none
  void* y; int64_t y_stride;
  float* z; int64_t z_stride;              // z = x w^T + bias in binary32, or null
  uint8_t* z_values; int64_t z_pitch; uint8_t* z_scales;  // or as 8-bit blocks, or null
  const uint8_t* x_values; int64_t xv_stride; const uint8_t* x_scales;  // x as 8-bit blocks
  const uint8_t* w_values; int64_t wv_stride; const uint8_t* w_scales;  // w as 8-bit blocks
  // backward
  const void* dy; int64_t dy_stride;
  void* dx; int64_t dx_stride;             // null: not wanted
  void* dw;                                // n x k, contiguous; null: not wanted
  void* dbias;                             // null: not wanted
  void* workspace;
};
cudaError_t launch_linear_forward(const LinearArgs& a, ndvm_dtype t, cudaStream_t s);
cudaError_t launch_linear_blocks(const LinearArgs& a, ndvm_dtype t, cudaStream_t s);
cudaError_t launch_linear_backward(const LinearArgs& a, ndvm_dtype t, cudaStream_t s);
size_t linear_workspace(const LinearArgs& a, bool backward);  // of this call
// of any call of these sizes; copies: with operands that TMA cannot read; blocks: x is held as 8-bit blocks
size_t linear_workspace(int64_t rows, int64_t k, int64_t n, ndvm_activation act, bool backward, bool copies, bool blocks);
size_t linear_blocks_workspace(int64_t rows, int64_t k, int64_t n);
cudaError_t linear_stopped(int* flag);  // reads and clears: a kernel gave up waiting

struct GatedArgs {
  int64_t rows, k, n;
  const void* x; int64_t x_stride;
  const void* w_gate; const void* w_up; int64_t g_stride, u_stride;
  ndvm_activation act;
  void* h; int64_t h_stride;
  const void* dh; int64_t dh_stride;
  void* dx; int64_t dx_stride;
  void* dw_gate; void* dw_up;  // n x k, contiguous
  float* kept; int64_t kept_stride;  // G and U in binary32 (2 x rows rows), or null
  void* workspace;
};
cudaError_t launch_gated_forward(const GatedArgs& a, ndvm_dtype t, cudaStream_t s);
cudaError_t launch_gated_backward(const GatedArgs& a, ndvm_dtype t, cudaStream_t s);
size_t gated_workspace(int64_t rows, int64_t k, int64_t n, bool backward, bool copies);
size_t gated_workspace(const GatedArgs& a, bool backward);  // of this call
cudaError_t product_stopped(int* flag);                     // reads and clears: a kernel gave up waiting

}  // namespace ndvm
