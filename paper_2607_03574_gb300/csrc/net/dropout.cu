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

// A round's two products in full, as the widening multiply that the hardware has: through 64-bit integers the
// compiler spends more (134 M bfloat16 elements with a residual: 156 us against 129).
__device__ __forceinline__ void product(uint32_t a, uint32_t m, uint32_t* high, uint32_t* low) {
  asm("{\n .reg .u64 t;\n mul.wide.u32 t, %2, %3;\n mov.b64 {%1, %0}, t;\n}" : "=r"(*high), "=r"(*low) : "r"(a), "r"(m));
}
// The rounds' keys are the launch's: the host works them out once (constant operands here).
struct Keys { uint32_t k[10][2]; };
__device__ __forceinline__ Words philox(uint64_t block, const Keys& keys) {
  uint32_t a = (uint32_t)block, b = (uint32_t)(block >> 32), c = 0, d = 0;
#pragma unroll
  for (int r = 0; r < 10; r++) {
    uint32_t p1, p0, q1, q0;
    product(a, 0xD2511F53u, &p1, &p0);
    product(c, 0xCD9E8D57u, &q1, &q0);
    a = q1 ^ b ^ keys.k[r][0];
    b = q0;
    c = p1 ^ d ^ keys.k[r][1];
    d = p0;
  }
  return {{a, b, c, d}};
}

template <typename T, bool kResidual>
__device__ __forceinline__ T drop(const DropArgs& a, uint32_t word, T x, T r) {
  float y = word >= a.threshold ? to_f32(x) * a.scale : 0.0f;
  if (kResidual) y += to_f32(r);
  return from_f32<T>(y);
}
__device__ __forceinline__ float2 drop(const DropArgs& a, uint32_t w0, uint32_t w1, float2 x) {
  const float2 y = mul(x, make_float2(a.scale, a.scale));
  return make_float2(w0 >= a.threshold ? y.x : 0.0f, w1 >= a.threshold ? y.y : 0.0f);  // (chosen, not multiplied by 0)
}

// 16 bytes of x (and of the residual) from its v-th vector on
template <typename T, bool kResidual>
__device__ __forceinline__ void drop_vector(const DropArgs& a, const Keys& keys, const T* x, const T* r, T* y, uint64_t block) {
  constexpr int V = 16 / sizeof(T);
  Pack<T, V> p = load_pack<T, V>(x), pr;
  if (kResidual) pr = load_pack<T, V>(r);
#pragma unroll
  for (int q = 0; q < V / 4; q++) {
    const Words w = philox(block + q, keys);
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      float2 d = drop(a, w.w[e], w.w[e + 1], widen(p.v + q * 4 + e));
      if (kResidual) d = add(d, widen(pr.v + q * 4 + e));
      narrow(p.v + q * 4 + e, d);
    }
  }
  store_pack(y, p);
}

// Contiguous tensors (one row of any length).  With a residual bound by memory: 134 M bfloat16 elements in 114 us,
// 7.1 TB/s; without, by the generator's instructions: 107 us, 5.0 TB/s (the pipe of the widening multiplies is busy 69 % of
// the time, that of the xors 59 %; a warp waits 8.8 cycles an instruction for a pipe or its dispatch, 2.6 for memory).
// Binary32 has half as many a byte and waits for memory again, 6.4 TB/s.  One vector a thread and all the threads an SM holds: with 40 of its 64 warps 126 us, with several vectors a
// thread, the next one's loads in flight or not, 143 to 191 us.
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kThreads, 8) k_dropout_flat(const __grid_constant__ DropArgs a, const __grid_constant__ Keys keys) {
  constexpr int V = 16 / sizeof(T);
  const T *x = static_cast<const T*>(a.x), *r = static_cast<const T*>(a.residual);
  T* y = static_cast<T*>(a.y);
  const int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x, vectors = a.cols / V;
  if (v < vectors) {
    drop_vector<T, kResidual>(a, keys, x + v * V, kResidual ? r + v * V : r, y + v * V, a.offset / 4 + (uint64_t)v * (V / 4));
  } else if (v == vectors) {  // what is left beyond the vectors
#pragma unroll 1
    for (int64_t c = vectors * V; c < a.cols; c += 4) {
      const Words w = philox(a.offset / 4 + (uint64_t)(c / 4), keys);
#pragma unroll
      for (int e = 0; e < 4; e++)
        if (c + e < a.cols) y[c + e] = drop<T, kResidual>(a, w.w[e], x[c + e], kResidual ? r[c + e] : x[c + e]);
    }
  }
}

// rows of whole vectors that start on 16 bytes
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kThreads, 8) k_dropout_rows(const __grid_constant__ DropArgs a, const __grid_constant__ Keys keys) {
  constexpr int V = 16 / sizeof(T);
  const int64_t v = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, vectors = a.cols / V;
  if (v >= vectors) return;
  for (int64_t row = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; row < a.rows; row += (int64_t)gridDim.y * blockDim.y)
    drop_vector<T, kResidual>(a, keys, static_cast<const T*>(a.x) + row * a.x_stride + v * V,
                              kResidual ? static_cast<const T*>(a.residual) + row * a.r_stride + v * V : nullptr,
                              static_cast<T*>(a.y) + row * a.y_stride + v * V,
                              a.offset / 4 + (uint64_t)(row * vectors + v) * (V / 4));
}

// Any layout: a generator block a thread and step, of which the row's elements are taken (a block that
// two rows share is drawn for both).
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kThreads) k_dropout_elements(const __grid_constant__ DropArgs a, const __grid_constant__ Keys keys) {
  for (int64_t row = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; row < a.rows; row += (int64_t)gridDim.y * blockDim.y) {
    const int64_t i0 = row * a.cols, g = i0 / 4 + (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t c0 = g * 4 - i0;  // the column of the block's first word
    if (c0 >= a.cols) continue;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* r = kResidual ? static_cast<const T*>(a.residual) + row * a.r_stride : x;
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    const Words w = philox(a.offset / 4 + (uint64_t)g, keys);
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
  Keys keys;
  for (int r = 0; r < 10; r++) {
    keys.k[r][0] = (uint32_t)a.seed + (uint32_t)r * 0x9E3779B9u;
    keys.k[r][1] = (uint32_t)(a.seed >> 32) + (uint32_t)r * 0xBB67AE85u;
  }
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
  if (vectors && a.rows == 1) {
    const int64_t blocks = a.cols / V / kThreads + 1;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    k_dropout_flat<T, kResidual><<<(unsigned)blocks, kThreads, 0, s>>>(a, keys);
    return cudaGetLastError();
  }
  // items of a row: its vectors, or the blocks it meets (one more where it starts inside a block)
  const int64_t items = vectors ? a.cols / V : a.cols / 4 + 2;
  int bx = kThreads;
  while (bx > 8 && bx / 2 >= items) bx /= 2;
  const dim3 block(bx, kThreads / bx);
  const int64_t gx = (items + bx - 1) / bx, gy = (a.rows + block.y - 1) / block.y;
  if (gx > 0x7fffffff) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)gx, (unsigned)std::min<int64_t>(gy, 65535));
  if (vectors) k_dropout_rows<T, kResidual><<<grid, block, 0, s>>>(a, keys);
  else k_dropout_elements<T, kResidual><<<grid, block, 0, s>>>(a, keys);
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
