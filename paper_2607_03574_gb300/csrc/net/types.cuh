// Element types of the network operators: everything is computed in binary32 and rounded once, to
// nearest, when it is stored.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

namespace ndvm {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// V elements that are loaded and stored together (16 bytes, or one element)
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
  T v[V];
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
  if constexpr (sizeof(T) * V == 16) {
    union { uint4 u; Pack<T, V> p; } b;
    b.u = *reinterpret_cast<const uint4*>(p);
    return b.p;
  } else {
    return *reinterpret_cast<const Pack<T, V>*>(p);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& v) {
  if constexpr (sizeof(T) * V == 16) {
    union { uint4 u; Pack<T, V> p; } b;
    b.p = v;
    *reinterpret_cast<uint4*>(p) = b.u;
  } else {
    *reinterpret_cast<Pack<T, V>*>(p) = v;
  }
}

}  // namespace ndvm
