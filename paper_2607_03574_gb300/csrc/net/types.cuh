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

// Pairs of binary32 values, which one instruction adds, multiplies or fuses (sm_100 and later); a lone value
// has the same operations, so a kernel is written once for packs of 8, 4 and 1 elements.
__device__ __forceinline__ uint64_t bits(float2 v) {
  uint64_t b;
  asm("mov.b64 %0, {%1, %2};" : "=l"(b) : "f"(v.x), "f"(v.y));
  return b;
}
__device__ __forceinline__ float2 pair(uint64_t b) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(b));
  return v;
}
__device__ __forceinline__ float2 add(float2 a, float2 b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)));
  return pair(d);
}
__device__ __forceinline__ float2 mul(float2 a, float2 b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)));
  return pair(d);
}
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
  return pair(d);
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float mul(float a, float b) { return a * b; }
__device__ __forceinline__ float fma(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float total(float2 a) { return a.x + a.y; }
__device__ __forceinline__ float total(float a) { return a; }

template <int V> struct PairsOf { using Type = float2; static constexpr int kCount = V / 2; };
template <> struct PairsOf<1> { using Type = float; static constexpr int kCount = 1; };
template <int V> using Pairs = typename PairsOf<V>::Type;
template <int V> constexpr int kPairs = PairsOf<V>::kCount;

__device__ __forceinline__ float2 both(float v, float2) { return make_float2(v, v); }
__device__ __forceinline__ float both(float v, float) { return v; }

__device__ __forceinline__ float2 widen(const float* p) { return make_float2(p[0], p[1]); }
__device__ __forceinline__ float2 widen(const __half* p) { return __half22float2(*reinterpret_cast<const __half2*>(p)); }
__device__ __forceinline__ float2 widen(const __nv_bfloat16* p) {  // (its bits are the upper half of a binary32)
  const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ void narrow(float* p, float2 v) { p[0] = v.x, p[1] = v.y; }
__device__ __forceinline__ void narrow(__half* p, float2 v) { *reinterpret_cast<__half2*>(p) = __float22half2_rn(v); }
__device__ __forceinline__ void narrow(__nv_bfloat16* p, float2 v) { *reinterpret_cast<__nv_bfloat162*>(p) = __float22bfloat162_rn(v); }

template <typename T, int V>
__device__ __forceinline__ void widen(const Pack<T, V>& p, Pairs<V> (&v)[kPairs<V>]) {
  if constexpr (V == 1) {
    v[0] = to_f32(p.v[0]);
  } else {
#pragma unroll
    for (int i = 0; i < V / 2; i++) v[i] = widen(p.v + 2 * i);
  }
}
template <typename T, int V>
__device__ __forceinline__ void narrow(Pack<T, V>& p, int i, Pairs<V> v) {
  if constexpr (V == 1) p.v[0] = from_f32<T>(v);
  else narrow(p.v + 2 * i, v);
}

}  // namespace ndvm
