// Layer norm over a row of C elements, and its backward pass:
//   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), xh = (x - m) r, y = xh w + b
//   g = dy w, dx = r (g - mean(g) - xh mean(g xh)), dw = sum over rows of dy xh, db = sum over rows of dy
#include "net.h"
#include "types.cuh"

namespace ndvm {
namespace {

constexpr int kThreads = 256;
constexpr int kColumnBlocks = 64;  // row ranges whose column sums are added up apart

__device__ __forceinline__ float2 block_sum2(float a, float b) {
  __shared__ float2 part[kThreads / 32];
  for (int o = 16; o; o >>= 1) {
    a += __shfl_xor_sync(~0u, a, o);
    b += __shfl_xor_sync(~0u, b, o);
  }
  __syncthreads();
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = make_float2(a, b);
  __syncthreads();
  float2 s = part[0];
  for (int w = 1; w < kThreads / 32; w++) s.x += part[w].x, s.y += part[w].y;
  return s;
}

// a block a row
template <typename T, typename W>
__global__ void k_forward(NormArgs a) {
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    float s = 0.0f;
    for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) s += to_f32(x[c]);
    const float mean = block_sum2(s, 0.0f).x / (float)a.cols;
    s = 0.0f;
    for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
      const float d = to_f32(x[c]) - mean;
      s += d * d;
    }
    const float rstd = 1.0f / sqrtf(block_sum2(s, 0.0f).x / (float)a.cols + a.eps);
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
      float v = (to_f32(x[c]) - mean) * rstd;
      if (a.weight) v *= to_f32(static_cast<const W*>(a.weight)[c]);
      if (a.bias) v += to_f32(static_cast<const W*>(a.bias)[c]);
      y[c] = from_f32<T>(v);
    }
    if (threadIdx.x == 0 && a.stats) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = rstd;
    }
  }
}

template <typename T, typename W>
__global__ void k_backward_x(NormArgs a) {
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
    const float mean = a.stats[row], rstd = a.stats[a.rows + row];
    float sg = 0.0f, sgx = 0.0f;
    for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
      const float g = to_f32(dy[c]) * (a.weight ? to_f32(static_cast<const W*>(a.weight)[c]) : 1.0f);
      sg += g;
      sgx += g * ((to_f32(x[c]) - mean) * rstd);
    }
    const float2 s = block_sum2(sg, sgx);
    const float mg = s.x / (float)a.cols, mgx = s.y / (float)a.cols;
    T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
    for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
      const float g = to_f32(dy[c]) * (a.weight ? to_f32(static_cast<const W*>(a.weight)[c]) : 1.0f);
      dx[c] = from_f32<T>(rstd * (g - mg - (to_f32(x[c]) - mean) * rstd * mgx));
    }
  }
}

// column sums over a range of rows: partial[0][range][c] = sum dy xh, partial[1][range][c] = sum dy
template <typename T>
__global__ void k_columns(NormArgs a) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= a.cols) return;
  float sw = 0.0f, sb = 0.0f;
  for (int64_t row = blockIdx.y; row < a.rows; row += kColumnBlocks) {
    const float dy = to_f32(static_cast<const T*>(a.dy)[row * a.dy_stride + c]);
    sw += dy * ((to_f32(static_cast<const T*>(a.x)[row * a.x_stride + c]) - a.stats[row]) * a.stats[a.rows + row]);
    sb += dy;
  }
  a.partial[(int64_t)blockIdx.y * a.cols + c] = sw;
  a.partial[((int64_t)kColumnBlocks + blockIdx.y) * a.cols + c] = sb;
}

template <typename W>
__global__ void k_columns_join(NormArgs a) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= a.cols) return;
  float sw = 0.0f, sb = 0.0f;
  for (int p = 0; p < kColumnBlocks; p++) {
    sw += a.partial[(int64_t)p * a.cols + c];
    sb += a.partial[((int64_t)kColumnBlocks + p) * a.cols + c];
  }
  if (a.dweight) static_cast<W*>(a.dweight)[c] = from_f32<W>(sw);
  if (a.dbias) static_cast<W*>(a.dbias)[c] = from_f32<W>(sb);
}

template <typename T, typename W>
cudaError_t forward(const NormArgs& a, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  k_forward<T, W><<<(unsigned)(a.rows < 65536 ? a.rows : 65536), kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T, typename W>
cudaError_t backward(const NormArgs& a, cudaStream_t s) {
  if (a.dx && a.rows > 0) k_backward_x<T, W><<<(unsigned)(a.rows < 65536 ? a.rows : 65536), kThreads, 0, s>>>(a);
  if (a.dweight || a.dbias) {
    const unsigned g = (unsigned)((a.cols + kThreads - 1) / kThreads);
    k_columns<T><<<dim3(g, kColumnBlocks), kThreads, 0, s>>>(a);
    k_columns_join<W><<<g, kThreads, 0, s>>>(a);
  }
  return cudaGetLastError();
}

template <typename F>
cudaError_t by_type(ndvm_dtype t, ndvm_dtype wt, F&& f) {
  if (t == NDVM_F32) return f(float(), float());
  if (t == NDVM_F16) return wt == NDVM_F32 ? f(__half(), float()) : f(__half(), __half());
  return wt == NDVM_F32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
}

}  // namespace

cudaError_t launch_norm_forward(const NormArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s) {
  return by_type(t, wt, [&](auto x, auto w) { return forward<decltype(x), decltype(w)>(a, s); });
}
cudaError_t launch_norm_backward(const NormArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s) {
  return by_type(t, wt, [&](auto x, auto w) { return backward<decltype(x), decltype(w)>(a, s); });
}
size_t norm_workspace(int64_t, int64_t cols) { return (size_t)cols * 2 * kColumnBlocks * sizeof(float); }

}  // namespace ndvm
