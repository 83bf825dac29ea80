// What the row norms share: rows in the registers of the threads that share them, sums over a row and over columns, and
// which variant takes which rows.
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <utility>

#include "net.h"
#include "types.cuh"

namespace ndvm {
namespace {

// weights are of the activations' type or binary32
template <typename T, int V>
__device__ __forceinline__ void load_weight(Pairs<V> (&w)[kPairs<V>], const void* p, int f32, int64_t c, float none) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < kPairs<V>; e++) w[e] = both(none, w[e]);
  } else if (f32) {
    if constexpr (V == 1) {
      w[0] = static_cast<const float*>(p)[c];
    } else if constexpr (V == 2) {
      w[0] = *reinterpret_cast<const float2*>(static_cast<const float*>(p) + c);
    } else {
#pragma unroll
      for (int q = 0; q < V; q += 4) {
        const Pack<float, 4> v = load_pack<float, 4>(static_cast<const float*>(p) + c + q);
        w[q / 2] = make_float2(v.v[0], v.v[1]);
        w[q / 2 + 1] = make_float2(v.v[2], v.v[3]);
      }
    }
  } else {
    widen<T, V>(load_pack<T, V>(static_cast<const T*>(p) + c), w);
  }
}

// the lanes of this thread's group of kRow, or of its warp
template <int kRow>
__device__ __forceinline__ uint32_t group_lanes() {
  return kRow >= 32 ? ~0u : ((1u << (kRow & 31)) - 1) << (threadIdx.x % 32 / kRow * kRow);
}

// Sums over the kRow threads that share a row: a warp's shuffles, then the warps' sums in shared memory
// (`part` is the caller's, another one for each sum of a row, so one barrier a sum is enough).
template <int kRow>
__device__ __forceinline__ float row_sum(float v, float* part) {
#pragma unroll
  for (int o = (kRow < 32 ? kRow : 32) / 2; o; o >>= 1) v += __shfl_xor_sync(group_lanes<kRow>(), v, o);
  if constexpr (kRow > 32) {
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kRow / 32; w++) v += part[w];
  }
  return v;
}

template <int kRow> constexpr int kBlock = kRow > 32 ? kRow : 128;  // threads a block
template <int kRow> constexpr int kBackBlock = kRow > 256 ? kRow : 256;
constexpr int kLong = 512;  // threads a row that no variant holds

// Two sums over the kRow threads of a group that shares a row, by the group's own barrier; `part` is another
// one on the next call (a group's warp may still read this one then, but not on the call after).
template <int kRow>
__device__ __forceinline__ float2 group_sum(float a, float b, float2* part, int group) {
#pragma unroll
  for (int o = (kRow < 32 ? kRow : 32) / 2; o; o >>= 1) {
    a += __shfl_xor_sync(group_lanes<kRow>(), a, o);
    b += __shfl_xor_sync(group_lanes<kRow>(), b, o);
  }
  float2 s = make_float2(a, b);
  if constexpr (kRow > 32) {
    if (threadIdx.x % 32 == 0) part[threadIdx.x % kRow / 32] = s;
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kRow) : "memory");
    s = part[0];
#pragma unroll
    for (int w = 1; w < kRow / 32; w++) s = add(s, part[w]);
  }
  return s;
}

// adds up the blocks' column sums ([block][set][column], one or two sets): 32 columns a block, 32 chains each, joined in shared memory
template <typename W>
__global__ void __launch_bounds__(1024) k_columns_join(const float* partial, int blocks, int sets, int64_t cols, W* first, W* second) {
  __shared__ float part[32][33];
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
  W* out = blockIdx.y ? second : first;
  if (!out) return;
  float s = 0.0f;
  if (c < cols) {
    const float* p = partial + (int64_t)blockIdx.y * cols + c;
#pragma unroll 8
    for (int b = threadIdx.y; b < blocks; b += 32) s += p[(int64_t)b * sets * cols];
  }
  part[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  s = part[threadIdx.x][threadIdx.y];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
  const int64_t d = (int64_t)blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && d < cols) out[d] = from_f32<W>(s);
}

constexpr int64_t kHeld = 8192;        // columns that k_backward holds at most (backward_variant); from there on
constexpr int kMostBlocks = kSms * 6;  // of k_backward: their column sums are what the workspace holds
constexpr int kLongBlocks = 64;        // row ranges of k_columns_long


bool starts_on(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
// Elements a load: 16 bytes, two elements or one, whatever every row (and the weights) start and end on.
template <typename T>
int load_width(int64_t rows, int64_t cols, int w_f32, std::initializer_list<const void*> vectors,
               std::initializer_list<std::pair<const void*, int64_t>> matrices) {
  for (const int v : {16 / (int)sizeof(T), 2}) {
    bool ok = cols % v == 0;
    for (const auto& m : matrices) ok &= starts_on(m.first, v * sizeof(T)) && (rows <= 1 || m.second % v == 0);
    const size_t w = v == 2 ? (w_f32 ? 8 : 2 * sizeof(T)) : 16;
    for (const void* p : vectors) ok &= starts_on(p, w);
    if (ok) return v;
  }
  return 1;
}

// The kernel variant for rows of `cols` elements: V elements a load, N loads a thread, kRow threads a row, blocks an
// SM.  `f` is called with them as integral constants; false: the row is longer than any variant holds.  (Two
// elements a load: 30000 x 2050 bfloat16 forward 94 us, with 2051 columns, one a load, 122.)
template <int K> using Int = std::integral_constant<int, K>;

template <typename T, typename F>
bool forward_variant(int width, int64_t cols, F&& f) {
  constexpr int V = 16 / sizeof(T);
  if (width == V) {
    const int64_t packs = cols / V;  // a quarter of a warp, then a warp a row up to 8 loads a thread (no barriers), then blocks
    if (packs <= 8) f(Int<V>(), Int<1>(), Int<8>(), Int<12>());
    else if (packs <= 16) f(Int<V>(), Int<2>(), Int<8>(), Int<12>());
    else if (packs <= 32) f(Int<V>(), Int<1>(), Int<32>(), Int<12>());
    else if (packs <= 64) f(Int<V>(), Int<2>(), Int<32>(), Int<12>());
    else if (packs <= 128) f(Int<V>(), Int<4>(), Int<32>(), Int<10>());
    else if (packs <= 256) f(Int<V>(), Int<8>(), Int<32>(), Int<7>());
    else if (packs <= 512) f(Int<V>(), Int<4>(), Int<128>(), Int<10>());
    else if (packs <= 1024) f(Int<V>(), Int<4>(), Int<256>(), Int<5>());
    else if (packs <= 2048) f(Int<V>(), Int<4>(), Int<512>(), Int<2>());
    else return false;
  } else if (width == 2) {
    if (cols <= 256) f(Int<2>(), Int<4>(), Int<32>(), Int<12>());
    else if (cols <= 1024) f(Int<2>(), Int<16>(), Int<32>(), Int<8>());
    else if (cols <= 2048) f(Int<2>(), Int<8>(), Int<128>(), Int<10>());
    else if (cols <= 4096) f(Int<2>(), Int<8>(), Int<256>(), Int<5>());
    else if (cols <= 8192) f(Int<2>(), Int<8>(), Int<512>(), Int<2>());
    else return false;
  } else {
    if (cols <= 64) f(Int<1>(), Int<8>(), Int<8>(), Int<12>());
    else if (cols <= 128) f(Int<1>(), Int<4>(), Int<32>(), Int<12>());
    else if (cols <= 512) f(Int<1>(), Int<16>(), Int<32>(), Int<10>());
    else if (cols <= 2048) f(Int<1>(), Int<16>(), Int<128>(), Int<10>());
    else if (cols <= 4096) f(Int<1>(), Int<16>(), Int<256>(), Int<5>());
    else if (cols <= 8192) f(Int<1>(), Int<16>(), Int<512>(), Int<2>());
    else return false;
  }
  return true;
}

template <typename T, typename F>
bool backward_variant(int width, int64_t rows, int64_t cols, F&& f) {
  constexpr int V = 16 / sizeof(T);
  if (cols > kHeld) return false;
  if (width == V) {
    const int64_t packs = cols / V;
    if (packs <= 8) f(Int<V>(), Int<1>(), Int<8>(), Int<3>());
    else if (packs <= 16) f(Int<V>(), Int<2>(), Int<8>(), Int<2>());
    else if (packs <= 32) f(Int<V>(), Int<1>(), Int<32>(), Int<3>());
    else if (packs <= 64) f(Int<V>(), Int<2>(), Int<32>(), Int<2>());
    else if (packs <= 128) f(Int<V>(), Int<2>(), Int<64>(), Int<2>());
    // one load and twice the threads: more warps for many rows, more column sums to join for few.  bf16, us, one load
    // against two: 2048 columns 18.2 / 15.4 at 4096 rows, 45.1 / 43.2 at 16384, 78.5 / 78.3 at 32768, 146 / 150 at 65536;
    // 1536 columns 16.6 / 15.1, 38.5 / 39.0, 67.7 / 70.6, 125 / 133
    else if (packs <= 256 && rows >= 32768) f(Int<V>(), Int<1>(), Int<256>(), Int<4>());
    else if (packs <= 256) f(Int<V>(), Int<2>(), Int<128>(), Int<2>());
    else if (packs <= 512) f(Int<V>(), Int<2>(), Int<256>(), Int<2>());
    else if (packs <= 1024) f(Int<V>(), Int<2>(), Int<512>(), Int<1>());
    else if (packs <= 2048 && sizeof(T) == 4) f(Int<4>(), Int<4>(), Int<512>(), Int<1>());  // (16-bit rows would not fit in 128 registers)
    else return false;
  } else if (width == 2) {
    if (cols <= 256) f(Int<2>(), Int<4>(), Int<32>(), Int<3>());
    else if (cols <= 512) f(Int<2>(), Int<4>(), Int<64>(), Int<3>());
    else if (cols <= 1024) f(Int<2>(), Int<4>(), Int<128>(), Int<3>());
    else if (cols <= 2048) f(Int<2>(), Int<4>(), Int<256>(), Int<3>());
    else if (cols <= 4096) f(Int<2>(), Int<4>(), Int<512>(), Int<1>());
    else if (cols <= 8192) f(Int<2>(), Int<8>(), Int<512>(), Int<1>());
    else return false;
  } else {
    if (cols <= 64) f(Int<1>(), Int<8>(), Int<8>(), Int<3>());
    else if (cols <= 256) f(Int<1>(), Int<8>(), Int<32>(), Int<3>());
    else if (cols <= 512) f(Int<1>(), Int<8>(), Int<64>(), Int<3>());
    else if (cols <= 1024) f(Int<1>(), Int<8>(), Int<128>(), Int<3>());
    else if (cols <= 2048) f(Int<1>(), Int<8>(), Int<256>(), Int<3>());
    else if (cols <= 4096) f(Int<1>(), Int<8>(), Int<512>(), Int<1>());
    else if (cols <= 8192) f(Int<1>(), Int<16>(), Int<512>(), Int<1>());
    else return false;
  }
  return true;
}

}  // namespace
}  // namespace ndvm
