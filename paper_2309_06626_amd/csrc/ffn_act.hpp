// Activations of the gated feed-forward block.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace sc {

// T: what the results are rounded to.  The hardware's exponential of 1.44 v is off by |v| units of a float, its reciprocal by one: nothing to a
// 16-bit result, up to 80 units of a float one.
template <typename T> __device__ __forceinline__ float ffn_exp(float v) {
  if constexpr (sizeof(T) == 4) return expf(v);
  else return __expf(v);
}
// sigma(v), and 1 - sigma(v) in `rest` (of a float it keeps its digits where sigma(v) is close to 1)
template <typename T> __device__ __forceinline__ float ffn_sigmoid(float v, float& rest) {
  const float t = ffn_exp<T>(-v);
  if constexpr (sizeof(T) == 4) {
    const float s = 1.0f / (1.0f + t);
    rest = v > 0.0f ? t * s : 1.0f - s;
    return s;
  } else {
    const float s = __builtin_amdgcn_rcpf(1.0f + t);
    rest = 1.0f - s;
    return s;
  }
}

// Phi(v) = erfc(-v / sqrt 2) / 2 and e = exp(-v^2 / 2).  For 16-bit results Phi(-a) = e t P(t), t = 1 / (1 + 0.3 a), a rational form that
// shares the exponential with the derivative; P of degree 5, fitted here to erfcx(a / sqrt 2) / 2 for a of 0 .. 14 so that its relative error
// is evened out: below 1.2e-6 up to a = 1.5, 6e-6 up to 3 and 2.5e-5 beyond, where a form within so much of Phi alone would lose the small
// results (half a unit is 5e-4 of an f16, 4e-3 of a bf16).  erfcf takes some eighty operations (gated
// 6 272 x 768 -> 2 048 in f16: 54 us, with erfcf 67)
template <typename T> __device__ __forceinline__ float ffn_phi(float v, float& e) {
  e = ffn_exp<T>(-0.5f * v * v);
  if constexpr (sizeof(T) == 4) {
    return 0.5f * erfcf(-0.70710678118654752f * v);
  } else {
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.3f * fabsf(v));
    const float q = e * t * (0.12010857f + t * (0.113153685f + t * (0.147376575f + t * (-0.024197675f + t * (0.22335236f + t * -0.079793915f)))));
    return v < 0.0f ? q : 1.0f - q;
  }
}
// a = act(v), da = its derivative; KIND: sc_activation; T: what the results are rounded to
template <int KIND, typename T> __device__ __forceinline__ void ffn_act_of(float v, float& a, float& da) {
  if constexpr (KIND == 0) {                             // v sigma(v)
    float rest;
    const float s = ffn_sigmoid<T>(v, rest);
    a = v * s;
    da = s * (1.0f + v * rest);
  } else if constexpr (KIND == 1) {                      // v Phi(v), Phi the normal distribution
    float e;
    const float p = ffn_phi<T>(v, e);
    a = v * p;
    da = p + v * 0.39894228040143268f * e;
  } else {                                               // v sigma(2 t), t = sqrt(2 / pi) (v + 0.044715 v^3)
    const float c = 0.79788456080286536f, v2 = fminf(v * v, 1e4f);      // (beyond 100 sigma is 0 or 1; v^2 may be infinite)
    float rest;
    const float s = ffn_sigmoid<T>(2.0f * c * v * (1.0f + 0.044715f * v2), rest);
    a = v * s;
    da = s + v * s * rest * 2.0f * c * (1.0f + 3.0f * 0.044715f * v2);
  }
}
// fn(kind) with the kind as a constant: one branch for as many values as fn takes
template <class Fn> __device__ __forceinline__ void ffn_act_kind(int kind, Fn&& fn) {
  if (kind == 0) fn(std::integral_constant<int, 0>{});
  else if (kind == 1) fn(std::integral_constant<int, 1>{});
  else fn(std::integral_constant<int, 2>{});
}
template <typename T> __device__ __forceinline__ void ffn_act(int kind, float v, float& a, float& da) {
  ffn_act_kind(kind, [&](auto k) { ffn_act_of<decltype(k)::value, T>(v, a, da); });
}

}  // namespace sc
