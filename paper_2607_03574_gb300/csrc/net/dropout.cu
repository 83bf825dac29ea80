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

constexpr int kThreads = 256;

struct Words { uint32_t w[4]; };

__device__ __forceinline__ Words philox(uint64_t block, uint32_t k0, uint32_t k1) {
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
  return {{a, b, c, d}};
}

template <typename T, bool kResidual>
__device__ __forceinline__ T drop(const DropArgs& a, uint32_t word, T x, T r) {
  float y = word >= a.threshold ? to_f32(x) * a.scale : 0.0f;
  if (kResidual) y += to_f32(r);
  return from_f32<T>(y);
}

// 16 bytes of x (and of the residual) a thread and step, kSteps of them in flight: for rows that start on
// 16 bytes everywhere and hold whole vectors, and for one long row (a contiguous tensor) of any length.
template <typename T, bool kResidual, int kSteps>
__global__ void __launch_bounds__(kThreads) k_dropout_vectors(DropArgs a) {
  constexpr int V = 16 / sizeof(T);
  using P = Pack<T, V>;
  const int64_t vectors = a.cols / V;
  const uint32_t k0 = (uint32_t)a.seed, k1 = (uint32_t)(a.seed >> 32);
  for (int64_t row = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; row < a.rows; row += (int64_t)gridDim.y * blockDim.y) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* r = kResidual ? static_cast<const T*>(a.residual) + row * a.r_stride : nullptr;
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    const uint64_t first = a.offset / 4 + (uint64_t)(row * vectors) * (V / 4);
    const int64_t v0 = (int64_t)blockIdx.x * blockDim.x * kSteps + threadIdx.x;
    P px[kSteps], pr[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; s++) {
      const int64_t v = v0 + s * (int)blockDim.x;
      if (v < vectors) {
        px[s] = load_pack<T, V>(x + v * V);
        if (kResidual) pr[s] = load_pack<T, V>(r + v * V);
      }
    }
#pragma unroll
    for (int s = 0; s < kSteps; s++) {
      const int64_t v = v0 + s * (int)blockDim.x;
      if (v >= vectors) break;
      P out;
#pragma unroll
      for (int q = 0; q < V / 4; q++) {
        const Words w = philox(first + (uint64_t)v * (V / 4) + q, k0, k1);
#pragma unroll
        for (int e = 0; e < 4; e++) out.v[q * 4 + e] = drop<T, kResidual>(a, w.w[e], px[s].v[q * 4 + e], (kResidual ? pr : px)[s].v[q * 4 + e]);
      }
      store_pack(y + v * V, out);
    }
    // what a single row has beyond its vectors
    const int64_t c = vectors * V + threadIdx.x;
    if (blockIdx.x == 0 && c < a.cols) {
      const Words w = philox(a.offset / 4 + (uint64_t)(c / 4), k0, k1);
      const uint32_t word = c % 4 == 0 ? w.w[0] : c % 4 == 1 ? w.w[1] : c % 4 == 2 ? w.w[2] : w.w[3];
      y[c] = drop<T, kResidual>(a, word, x[c], kResidual ? r[c] : x[c]);
    }
  }
}

// Any layout: a generator block a thread and step, of which the row's elements are taken (a block that
// two rows share is drawn for both).
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kThreads) k_dropout_elements(DropArgs a) {
  const uint32_t k0 = (uint32_t)a.seed, k1 = (uint32_t)(a.seed >> 32);
  for (int64_t row = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; row < a.rows; row += (int64_t)gridDim.y * blockDim.y) {
    const int64_t i0 = row * a.cols, g = i0 / 4 + (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t c0 = g * 4 - i0;  // the column of the block's first word
    if (c0 >= a.cols) continue;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* r = kResidual ? static_cast<const T*>(a.residual) + row * a.r_stride : x;
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    const Words w = philox(a.offset / 4 + (uint64_t)g, k0, k1);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int64_t c = c0 + e;
      if (c >= 0 && c < a.cols) y[c] = drop<T, kResidual>(a, w.w[e], x[c], r[c]);
    }
  }
}

template <typename T, bool kResidual>
cudaError_t launch(DropArgs a, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  auto dense = [&](int64_t stride) { return a.rows == 1 || stride == a.cols; };
  if (dense(a.x_stride) && dense(a.y_stride) && (!kResidual || dense(a.r_stride))) {
    a.cols *= a.rows;  // one row
    a.rows = 1;
  }
  auto on16 = [&](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (a.rows == 1 || (stride * (int64_t)sizeof(T)) % 16 == 0);
  };
  const bool vectors = on16(a.x, a.x_stride) && on16(a.y, a.y_stride) && (!kResidual || on16(a.residual, a.r_stride)) &&
                       (a.rows == 1 || a.cols % V == 0);
  // items of a row: its vectors, or the blocks it meets (one more where it starts inside a block)
  const int64_t items = vectors ? std::max<int64_t>(a.cols / V, 1) : a.cols / 4 + 2;
  // two steps a thread keep four 16-byte loads in flight; few items go one a thread over more blocks
  const int steps = vectors && items * a.rows >= (int64_t)152 * 2048 * 2 ? 2 : 1;
  int bx = kThreads;
  while (bx > 8 && bx / 2 * steps >= items) bx /= 2;
  const dim3 block(bx, kThreads / bx);
  const int64_t gx = (items + (int64_t)bx * steps - 1) / ((int64_t)bx * steps), gy = (a.rows + block.y - 1) / block.y;
  if (gx > 0x7fffffff) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)gx, (unsigned)std::min<int64_t>(gy, 65535));
  if (!vectors) k_dropout_elements<T, kResidual><<<grid, block, 0, s>>>(a);
  else if (steps == 2) k_dropout_vectors<T, kResidual, 2><<<grid, block, 0, s>>>(a);
  else k_dropout_vectors<T, kResidual, 1><<<grid, block, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch(const DropArgs& a, cudaStream_t s) {
  return a.residual ? launch<T, true>(a, s) : launch<T, false>(a, s);
}

}  // namespace

cudaError_t launch_dropout(const DropArgs& a, ndvm_dtype t, cudaStream_t s) {
  return t == NDVM_F32 ? launch<float>(a, s) : t == NDVM_F16 ? launch<__half>(a, s) : launch<__nv_bfloat16>(a, s);
}

}  // namespace ndvm
