// Gated projection h = act(G) U with G = x Wg^T, U = x Wu^T, and its backward pass:
//   dU = dh act(G), dG = dh U act'(G), dx = dG Wg + dU Wu, dWg = dG^T x, dWu = dU^T x.
// G and U are computed again in the backward pass rather than kept: they stay in binary32 until dG and
// dU are rounded, once, to the operands' type.
#include "net.h"
#include "types.cuh"

namespace ndvm {
namespace {

constexpr int kTile = 64, kStep = 16;

__device__ __forceinline__ void activate(int act, float g, float* a, float* da) {
  if (act == NDVM_ACT_RELU) {
    *a = g > 0.0f ? g : (g != g ? g : 0.0f);
    *da = g > 0.0f ? 1.0f : 0.0f;
  } else if (act == NDVM_ACT_GELU) {
    const float cdf = 0.5f * (1.0f + erff(g * 0.70710678f));
    *a = g * cdf;
    *da = cdf + g * expf(-0.5f * g * g) * 0.39894228f;
  } else {
    const float s = 1.0f / (1.0f + expf(-g));
    *a = act == NDVM_ACT_SILU ? g * s : s;
    *da = act == NDVM_ACT_SILU ? s * (1.0f + g * (1.0f - s)) : s * (1.0f - s);
  }
}

// A view of a matrix operand: element (i, j) at p[i * si + j * sj].
template <typename T>
struct View {
  const T* p;
  int64_t si, sj;
};

// acc += A[m0.., 0..k) B[n0.., 0..k)^T for a 64 x 64 tile, 4 x 4 elements a thread
template <typename T>
__device__ void tile_product(View<T> A, View<T> B, int64_t m0, int64_t n0, int64_t m, int64_t n, int64_t k,
                             float (&sa)[kStep][kTile + 1], float (&sb)[kStep][kTile + 1], float (&acc)[4][4]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int64_t k0 = 0; k0 < k; k0 += kStep) {
    for (int e = threadIdx.x; e < kTile * kStep; e += 256) {
      const int i = e / kStep, j = e % kStep;
      const bool in = k0 + j < k;
      sa[j][i] = in && m0 + i < m ? to_f32(A.p[(m0 + i) * A.si + (k0 + j) * A.sj]) : 0.0f;
      sb[j][i] = in && n0 + i < n ? to_f32(B.p[(n0 + i) * B.si + (k0 + j) * B.sj]) : 0.0f;
    }
    __syncthreads();
    for (int j = 0; j < kStep; j++)
      for (int p = 0; p < 4; p++)
        for (int q = 0; q < 4; q++) acc[p][q] += sa[j][ty + 16 * p] * sb[j][tx + 16 * q];
    __syncthreads();
  }
}

// the two products and, forward: h; backward: dG and dU (rows x n each, in the workspace)
template <typename T, bool kBackward>
__global__ void __launch_bounds__(256) k_products(GatedArgs a) {
  __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
  float g[4][4] = {}, u[4][4] = {};
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
  const View<T> x{static_cast<const T*>(a.x), a.x_stride, 1};
  tile_product(x, View<T>{static_cast<const T*>(a.w_gate), a.g_stride, 1}, m0, n0, a.rows, a.n, a.k, sa, sb, g);
  tile_product(x, View<T>{static_cast<const T*>(a.w_up), a.u_stride, 1}, m0, n0, a.rows, a.n, a.k, sa, sb, u);
  for (int p = 0; p < 4; p++)
    for (int q = 0; q < 4; q++) {
      const int64_t i = m0 + threadIdx.x / 16 + 16 * p, j = n0 + threadIdx.x % 16 + 16 * q;
      if (i >= a.rows || j >= a.n) continue;
      float act, da;
      activate(a.act, g[p][q], &act, &da);
      if (kBackward) {
        const float dh = to_f32(static_cast<const T*>(a.dh)[i * a.dh_stride + j]);
        T* d = static_cast<T*>(a.workspace);
        d[i * a.n + j] = from_f32<T>(dh * u[p][q] * da);
        d[(a.rows + i) * a.n + j] = from_f32<T>(dh * act);
      } else {
        static_cast<T*>(a.h)[i * a.h_stride + j] = from_f32<T>(act * u[p][q]);
      }
    }
}

// out[m x n] = A1 B1^T + A2 B2^T (A2 null: the first alone)
template <typename T>
__global__ void __launch_bounds__(256) k_product(View<T> A1, View<T> B1, View<T> A2, View<T> B2, int64_t m, int64_t n,
                                                 int64_t k, T* out, int64_t stride) {
  __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
  float acc[4][4] = {};
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
  tile_product(A1, B1, m0, n0, m, n, k, sa, sb, acc);
  if (A2.p) tile_product(A2, B2, m0, n0, m, n, k, sa, sb, acc);
  for (int p = 0; p < 4; p++)
    for (int q = 0; q < 4; q++) {
      const int64_t i = m0 + threadIdx.x / 16 + 16 * p, j = n0 + threadIdx.x % 16 + 16 * q;
      if (i < m && j < n) out[i * stride + j] = from_f32<T>(acc[p][q]);
    }
}

dim3 tiles(int64_t m, int64_t n) { return dim3((unsigned)((n + kTile - 1) / kTile), (unsigned)((m + kTile - 1) / kTile)); }

template <typename T>
cudaError_t forward(const GatedArgs& a, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  k_products<T, false><<<tiles(a.rows, a.n), 256, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const GatedArgs& a, cudaStream_t s) {
  if (a.rows > 0) k_products<T, true><<<tiles(a.rows, a.n), 256, 0, s>>>(a);
  const T* dg = static_cast<const T*>(a.workspace);
  const T* du = dg + a.rows * a.n;
  const T *x = static_cast<const T*>(a.x), *wg = static_cast<const T*>(a.w_gate), *wu = static_cast<const T*>(a.w_up);
  const View<T> none{nullptr, 0, 0};
  if (a.dx && a.rows > 0)
    k_product<T><<<tiles(a.rows, a.k), 256, 0, s>>>(View<T>{dg, a.n, 1}, View<T>{wg, 1, a.g_stride}, View<T>{du, a.n, 1},
                                                    View<T>{wu, 1, a.u_stride}, a.rows, a.k, a.n, static_cast<T*>(a.dx), a.dx_stride);
  if (a.dw_gate)
    k_product<T><<<tiles(a.n, a.k), 256, 0, s>>>(View<T>{dg, 1, a.n}, View<T>{x, 1, a.x_stride}, none, none, a.n, a.k, a.rows,
                                                 static_cast<T*>(a.dw_gate), a.k);
  if (a.dw_up)
    k_product<T><<<tiles(a.n, a.k), 256, 0, s>>>(View<T>{du, 1, a.n}, View<T>{x, 1, a.x_stride}, none, none, a.n, a.k, a.rows,
                                                 static_cast<T*>(a.dw_up), a.k);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_gated_forward(const GatedArgs& a, ndvm_dtype t, cudaStream_t s) {
  return t == NDVM_F16 ? forward<__half>(a, s) : forward<__nv_bfloat16>(a, s);
}
cudaError_t launch_gated_backward(const GatedArgs& a, ndvm_dtype t, cudaStream_t s) {
  return t == NDVM_F16 ? backward<__half>(a, s) : backward<__nv_bfloat16>(a, s);
}
size_t gated_workspace(int64_t rows, int64_t, int64_t n) { return (size_t)rows * (size_t)n * 4; }

}  // namespace ndvm
