// 8-bit blocks: 32 consecutive elements of a row share a scale 2^e, the least (from e = -127 on) with which none is over 448
// in size, e4m3's largest; an element is the nearest e4m3 value to v / 2^e (ties to even).  The scale is held as e + 127
// in a byte, 255 where the block has an element that is not finite: then the whole block is NaN.
//
// Scales lie as the tensor cores read them: 512 bytes hold those of 128 rows and 128 columns, in the order [row % 32][row / 32
// % 4][column / 32 % 4]; those 512 bytes follow one another along a row first.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "types.cuh"

namespace ndvm {

// where the scale of block `block` of row `row` is; chunks: 128s of columns
__host__ __device__ __forceinline__ int64_t scale_at(int64_t row, int64_t block, int64_t chunks) {
  return (row / 128 * chunks + block / 4) * 512 + row % 32 * 16 + row / 32 % 4 * 4 + block % 4;
}

// The bits of |v|: they order as the values do, infinities and NaNs above all.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ float larger(float a, float b) {  // of the sizes; a NaN wins
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(fabsf(a)), "f"(fabsf(b)));
  return m;
}
// The scale of a block whose largest magnitude is `most`: with |v| = (1 + f) 2^x, 448 2^e = 1.75 2^(8 + e) is not below it
// from e = x - 8 on, or x - 7 if 1 + f > 1.75.
__device__ __forceinline__ uint32_t block_code(uint32_t most) {
  if (most >= 0x7f800000u) return 255;
  const int code = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u);
  return (uint32_t)max(code, 0);
}
// (255 says it all: what the elements of such a block are does not count)
__device__ __forceinline__ float block_inverse(uint32_t code) { return __uint_as_float(code == 255 ? 0x3f800000u : (254 - code) << 23); }
__device__ __forceinline__ float block_scale(uint32_t code) {
  return __uint_as_float(code == 255 ? 0x7fc00000u : code == 0 ? 0x400000u : code << 23);
}
// two values as e4m3, a in the lower byte
__device__ __forceinline__ uint32_t to_e4m3(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ float2 from_e4m3(uint16_t v) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(v));
  return __half22float2(*reinterpret_cast<__half2*>(&h));
}
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) { return to_e4m3(a, b) | to_e4m3(c, d) << 16; }

// The largest finite value of a type: rounding to e4m3 can lift an element beyond its block's largest, and what is stored
// of it in T stays finite.
template <typename T> __device__ __forceinline__ float largest();
template <> __device__ __forceinline__ float largest<float>() { return 3.4028234664e38f; }
template <> __device__ __forceinline__ float largest<__half>() { return 65504.0f; }
template <> __device__ __forceinline__ float largest<__nv_bfloat16>() { return 3.3895313893e38f; }
template <typename T>
__device__ __forceinline__ float2 held(float2 v, float scale, uint32_t code) {
  float2 h = mul(v, make_float2(scale, scale));
  if (code > (std::is_same<T, __half>::value ? 134u : 245u)) {  // (448 2^e is finite below)
    h.x = fabsf(h.x) > largest<T>() ? copysignf(largest<T>(), h.x) : h.x;
    h.y = fabsf(h.y) > largest<T>() ? copysignf(largest<T>(), h.y) : h.y;
  }
  return h;
}

// V elements of a row (those beyond its end are 0) to blocks: 32 / V consecutive lanes, `lanes` among them, share one.
template <int V>
__device__ __forceinline__ void store_block(const Pairs<V> (&v)[kPairs<V>], uint32_t lanes, uint8_t* values, bool inside, uint8_t* scale) {
  float size;
  if constexpr (V == 1) {
    size = v[0];
  } else {
    size = larger(v[0].x, v[0].y);
#pragma unroll
    for (int e = 1; e < kPairs<V>; e++) size = larger(size, larger(v[e].x, v[e].y));
  }
  uint32_t most = magnitude(size);
#pragma unroll
  for (int o = 16 / V; o; o >>= 1) most = max(most, __shfl_xor_sync(lanes, most, o));
  const uint32_t code = block_code(most);
  const float inverse = block_inverse(code);
  if (inside) {
    if constexpr (V == 1) {
      *values = (uint8_t)to_e4m3(v[0] * inverse, 0.0f);
    } else if constexpr (V == 2) {
      *reinterpret_cast<uint16_t*>(values) = (uint16_t)to_e4m3(v[0].x * inverse, v[0].y * inverse);
    } else {
      uint32_t q[V / 4];
#pragma unroll
      for (int e = 0; e < V / 4; e++)
        q[e] = to_e4m3(v[2 * e].x * inverse, v[2 * e].y * inverse, v[2 * e + 1].x * inverse, v[2 * e + 1].y * inverse);
      if constexpr (V == 8) *reinterpret_cast<uint2*>(values) = make_uint2(q[0], q[1]);
      else *reinterpret_cast<uint32_t*>(values) = q[0];
    }
  }
  if (scale && threadIdx.x % (32 / V) == 0) *scale = (uint8_t)code;
}

}  // namespace ndvm
