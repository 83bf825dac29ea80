// Dropout from a counter-based generator: y = residual + (kept ? x * scale : 0), the mask never stored.
//
// The generator is Philox4x32 with 10 rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011): block q of the sequence is four 32-bit words, a bijection of the
// counter (q mod 2^32, q / 2^32, 0, 0) under the key `seed`.  Element i (row-major index) takes word
// offset + i.  The backward pass draws the same words again.
#include "net.h"
#include "types.cuh"

namespace ndvm {
namespace {

__device__ __forceinline__ uint4 philox(uint64_t block, uint32_t k0, uint32_t k1) {
  uint32_t a = (uint32_t)block, b = (uint32_t)(block >> 32), c = 0, d = 0;
#pragma unroll
  for (int r = 0; r < 10; r++) {
    const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
    a = (uint32_t)(q >> 32) ^ b ^ k0;
    b = (uint32_t)q;
    c = (uint32_t)(p >> 32) ^ d ^ k1;
    d = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(a, b, c, d);
}

// One generator block (four elements, which may lie in several rows) a thread and step.
template <typename T>
__global__ void k_dropout(DropArgs a) {
  const int64_t n = a.rows * a.cols, groups = (n + 3) / 4, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t g = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; g < groups; g += step) {
    const uint4 v = philox(a.offset / 4 + g, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int64_t i = g * 4 + e;
      if (i >= n) break;
      const int64_t r = i / a.cols, c = i - r * a.cols;
      float y = w[e] >= a.threshold ? to_f32(static_cast<const T*>(a.x)[r * a.x_stride + c]) * a.scale : 0.0f;
      if (a.residual) y += to_f32(static_cast<const T*>(a.residual)[r * a.r_stride + c]);
      static_cast<T*>(a.y)[r * a.y_stride + c] = from_f32<T>(y);
    }
  }
}

}  // namespace

cudaError_t launch_dropout(const DropArgs& a, ndvm_dtype t, cudaStream_t s) {
  const int64_t groups = (a.rows * a.cols + 3) / 4, blocks = (groups + 255) / 256;
  const unsigned grid = (unsigned)(blocks < 152 * 16 ? blocks : 152 * 16);
  if (t == NDVM_F32) k_dropout<float><<<grid, 256, 0, s>>>(a);
  else if (t == NDVM_F16) k_dropout<__half><<<grid, 256, 0, s>>>(a);
  else k_dropout<__nv_bfloat16><<<grid, 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace ndvm
