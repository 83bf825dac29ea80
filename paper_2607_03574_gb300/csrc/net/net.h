// Network operators: layer norm, dropout and the gated projection (launchers; the C ABI is netapi.cpp).
// Rows are strided (strides in elements), a row's elements are contiguous.
#pragma once
#include <cuda_runtime.h>

#include "../status.h"

namespace ndvm {

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
cudaError_t gated_stopped(int* flag);                       // reads and clears: a kernel gave up waiting

}  // namespace ndvm
