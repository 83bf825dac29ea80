// Activations of the network operators and their derivatives, two values at a time.
#pragma once
#include <cuda_runtime.h>

#include <type_traits>

#include "../status.h"
#include "types.cuh"

namespace ndvm {

// act(g) and act'(g), two at a time: off by a few units of binary32's last place, and by a share of |g| (gelu: g^2) of
// them where the value itself vanishes.  Powers of two and reciprocals are the hardware's.
__device__ __forceinline__ float power2(float x) {  // (down to binary32's smallest)
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <int kAct>
__device__ __forceinline__ void activate(float2 g, float2* a, float2* da) {
  const float2 one = make_float2(1.0f, 1.0f);
  if constexpr (kAct == NDVM_ACT_NONE) {
    *a = g;
    *da = one;
  } else if constexpr (kAct == NDVM_ACT_RELU) {
    *a = make_float2(g.x > 0.0f ? g.x : (g.x != g.x ? g.x : 0.0f), g.y > 0.0f ? g.y : (g.y != g.y ? g.y : 0.0f));
    *da = make_float2(g.x > 0.0f ? 1.0f : 0.0f, g.y > 0.0f ? 1.0f : 0.0f);
  } else if constexpr (kAct == NDVM_ACT_GELU) {
    // The normal distribution function by its tail, cdf(-|g|) = e^(-g^2 / 2) t Q(t) with t = 1 / (1 + 0.35 |g|): relative
    // accuracy on both sides (1 + erf cancels below zero, to 4 % at -5 and to nothing from -5.5 on).  Q is the polynomial
    // of degree 8 with the least largest relative error on 0 <= |g| <= 15 (3.2e-8), by reweighted least squares.
    const float2 q = mul(mul(g, g), make_float2(-0.72134752f, -0.72134752f));  // -g^2 / 2 in powers of two
    const float2 e = make_float2(power2(q.x), power2(q.y));
    const float2 d = make_float2(fmaf(fabsf(g.x), 0.35f, 1.0f), fmaf(fabsf(g.y), 0.35f, 1.0f));
    const float2 t = make_float2(reciprocal(d.x), reciprocal(d.y));
    constexpr float kQ[9] = {0.139621258f, 0.139864326f,  0.119815566f, 0.105574533f,   -0.0232631564f,
                             0.15939188f,  -0.255900919f, 0.144060329f, -0.0291638281f};
    float2 tail = make_float2(kQ[8], kQ[8]);
#pragma unroll
    for (int i = 7; i >= 0; i--) tail = fma(tail, t, make_float2(kQ[i], kQ[i]));
    tail = mul(mul(e, t), tail);
    const float2 cdf = make_float2(g.x < 0.0f ? tail.x : 1.0f - tail.x, g.y < 0.0f ? tail.y : 1.0f - tail.y);
    *a = mul(g, cdf);
    *da = fma(mul(g, e), make_float2(0.39894228f, 0.39894228f), cdf);
  } else {
    // s = 1 / (1 + e^-g) and 1 - s are r and e r, with e = e^-|g| and r = 1 / (1 + e), the one or the other way round: nothing
    // cancels, overflows or is flushed in either tail
    const float2 e = make_float2(power2(fabsf(g.x) * -1.44269504f), power2(fabsf(g.y) * -1.44269504f));
    const float2 d = add(e, one), r = make_float2(reciprocal(d.x), reciprocal(d.y)), er = mul(e, r);
    const float2 s = make_float2(g.x < 0.0f ? er.x : r.x, g.y < 0.0f ? er.y : r.y);
    const float2 rest = make_float2(g.x < 0.0f ? r.x : er.x, g.y < 0.0f ? r.y : er.y);
    *a = kAct == NDVM_ACT_SILU ? mul(g, s) : s;
    *da = kAct == NDVM_ACT_SILU ? fma(*a, rest, s) : mul(s, rest);
  }
}
// act(g) alone, as it is stored in 16 bits: fewer instructions than activate(), which the epilogue of a product counts.  Tails
// keep their relative accuracy down to binary32's smallest here too (a power of two is the square of half the power's, which
// is never flushed before the result is 0), and nothing is chosen by the sign where a maximum can do it.
__device__ __forceinline__ float power2_normal(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <int kAct>
__device__ __forceinline__ float2 activation(float2 g) {
  if constexpr (kAct == NDVM_ACT_NONE) {
    return g;
  } else if constexpr (kAct == NDVM_ACT_RELU) {
    return make_float2(g.x < 0.0f ? 0.0f : g.x, g.y < 0.0f ? 0.0f : g.y);  // (a NaN stays one)
  } else if constexpr (kAct == NDVM_ACT_GELU) {
    // max(g, 0) - |g| cdf(-|g|), the tail as in activate(); from |g| = 40 on it is 0
    const float2 half = mul(mul(g, g), make_float2(-0.36067376f, -0.36067376f));
    const float2 h = make_float2(power2_normal(half.x), power2_normal(half.y)), e = mul(h, h);
    const float2 p = make_float2(fminf(fabsf(g.x), 40.0f), fminf(fabsf(g.y), 40.0f));
    const float2 t = make_float2(reciprocal(fmaf(p.x, 0.35f, 1.0f)), reciprocal(fmaf(p.y, 0.35f, 1.0f)));
    constexpr float kQ[9] = {0.139621258f, 0.139864326f,  0.119815566f, 0.105574533f,   -0.0232631564f,
                             0.15939188f,  -0.255900919f, 0.144060329f, -0.0291638281f};
    float2 tail = make_float2(kQ[8], kQ[8]);
#pragma unroll
    for (int i = 7; i >= 0; i--) tail = fma(tail, t, make_float2(kQ[i], kQ[i]));
    tail = mul(mul(e, t), tail);
    return make_float2(fmaf(-p.x, tail.x, fmaxf(g.x, 0.0f)), fmaf(-p.y, tail.y, fmaxf(g.y, 0.0f)));
  } else {
    const float2 h = make_float2(power2_normal(fabsf(g.x) * -0.72134752f), power2_normal(fabsf(g.y) * -0.72134752f)), e = mul(h, h);
    const float2 d = add(e, make_float2(1.0f, 1.0f)), r = make_float2(reciprocal(d.x), reciprocal(d.y));
    const float2 s = mul(r, make_float2(g.x < 0.0f ? e.x : 1.0f, g.y < 0.0f ? e.y : 1.0f));
    return kAct == NDVM_ACT_SILU ? mul(g, s) : s;
  }
}
// act'(g) alone, with fewer instructions than activate(): s (1 - s) is the same on both sides of 0.
template <int kAct>
__device__ __forceinline__ float2 derivative(float2 g) {
  const float2 one = make_float2(1.0f, 1.0f);
  if constexpr (kAct == NDVM_ACT_NONE) {
    return one;
  } else if constexpr (kAct == NDVM_ACT_RELU) {
    return make_float2(g.x > 0.0f ? 1.0f : 0.0f, g.y > 0.0f ? 1.0f : 0.0f);
  } else if constexpr (kAct == NDVM_ACT_GELU) {
    const float2 half = mul(mul(g, g), make_float2(-0.36067376f, -0.36067376f));
    const float2 h = make_float2(power2_normal(half.x), power2_normal(half.y)), e = mul(h, h);
    const float2 t = make_float2(reciprocal(fmaf(fabsf(g.x), 0.35f, 1.0f)), reciprocal(fmaf(fabsf(g.y), 0.35f, 1.0f)));
    constexpr float kQ[9] = {0.139621258f, 0.139864326f,  0.119815566f, 0.105574533f,   -0.0232631564f,
                             0.15939188f,  -0.255900919f, 0.144060329f, -0.0291638281f};
    float2 tail = make_float2(kQ[8], kQ[8]);
#pragma unroll
    for (int i = 7; i >= 0; i--) tail = fma(tail, t, make_float2(kQ[i], kQ[i]));
    tail = mul(mul(e, t), tail);
    const float2 cdf = make_float2(g.x < 0.0f ? tail.x : 1.0f - tail.x, g.y < 0.0f ? tail.y : 1.0f - tail.y);
    return fma(mul(g, e), make_float2(0.39894228f, 0.39894228f), cdf);
  } else {
    const float2 h = make_float2(power2_normal(fabsf(g.x) * -0.72134752f), power2_normal(fabsf(g.y) * -0.72134752f)), e = mul(h, h);
    const float2 d = add(e, one), r = make_float2(reciprocal(d.x), reciprocal(d.y)), er = mul(e, r);
    if constexpr (kAct == NDVM_ACT_SIGMOID) return mul(er, r);
    return fma(mul(g, er), r, make_float2(g.x < 0.0f ? er.x : r.x, g.y < 0.0f ? er.y : r.y));
  }
}
// f(activation as a constant): one branch around a loop over many elements, not one in each
template <typename F>
__device__ __forceinline__ void by_activation(int act, F&& f) {
  if (act == NDVM_ACT_SILU) f(std::integral_constant<int, NDVM_ACT_SILU>());
  else if (act == NDVM_ACT_GELU) f(std::integral_constant<int, NDVM_ACT_GELU>());
  else if (act == NDVM_ACT_RELU) f(std::integral_constant<int, NDVM_ACT_RELU>());
  else f(std::integral_constant<int, NDVM_ACT_SIGMOID>());
}
template <typename F>
__device__ __forceinline__ void by_activation_or_none(int act, F&& f) {
  if (act == NDVM_ACT_NONE) f(std::integral_constant<int, NDVM_ACT_NONE>());
  else by_activation(act, f);
}

}  // namespace ndvm
