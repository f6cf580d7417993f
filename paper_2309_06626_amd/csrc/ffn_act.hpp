// Activations of the gated feed-forward block.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace sc {

__device__ __forceinline__ float ffn_sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }

// a = act(v), da = its derivative; KIND: sc_activation
template <int KIND> __device__ __forceinline__ void ffn_act_of(float v, float& a, float& da) {
  if constexpr (KIND == 0) {                             // v sigma(v)
    const float s = ffn_sigmoid(v);
    a = v * s;
    da = s * (1.0f + v * (1.0f - s));
  } else if constexpr (KIND == 1) {                      // v Phi(v), Phi the normal distribution
    const float p = 0.5f * erfcf(-0.70710678118654752f * v);
    a = v * p;
    da = p + v * 0.39894228040143268f * __expf(-0.5f * v * v);
  } else {                                               // v sigma(2 t), t = sqrt(2 / pi) (v + 0.044715 v^3)
    const float c = 0.79788456080286536f, v2 = v * v;
    const float s = ffn_sigmoid(2.0f * c * v * (1.0f + 0.044715f * v2));
    a = v * s;
    da = s + v * s * (1.0f - s) * 2.0f * c * (1.0f + 3.0f * 0.044715f * v2);
  }
}
// fn(kind) with the kind as a constant: one branch for as many values as fn takes
template <class Fn> __device__ __forceinline__ void ffn_act_kind(int kind, Fn&& fn) {
  if (kind == 0) fn(std::integral_constant<int, 0>{});
  else if (kind == 1) fn(std::integral_constant<int, 1>{});
  else fn(std::integral_constant<int, 2>{});
}
__device__ __forceinline__ void ffn_act(int kind, float v, float& a, float& da) {
  ffn_act_kind(kind, [&](auto k) { ffn_act_of<decltype(k)::value>(v, a, da); });
}

}  // namespace sc
