// What a training step's forward pass keeps of g and u for the backward pass: [3][rows][d_hidden] of the operands' type.
//
// Floats: g, u (the third matrix is not used).  16-bit types: 24 bits each of the floats g and u, the upper halves in the first two matrices
// and a byte of each in the third.  Rounded to the type instead they would be off by half a unit each, and so would be the gradients of x,
// Wg and Wu: 0.0031 from the 64-bit result in bf16 against 0.0023 (0.0017 is the rounding of the result itself, the rest that of dg and du).
// hidden, which has no room beside them, is formed again.  8 192 x 2 048 -> 5 632 in bf16, forward and backward: 1 640 us, 1 574 with g, u and
// hidden in 16 bits (gated product 361 and 345, hidden gradient 282 and 239: three more matrices of 92 MB pass).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sc {

template <typename T> struct FfnSaved;
template <> struct FfnSaved<float> {
  static constexpr int PLANES = 2;
  using U = float;
  static __device__ __forceinline__ void keep(float g, float u, U (&p)[PLANES]) { p[0] = g, p[1] = u; }
  static __device__ __forceinline__ void back(const U (&p)[PLANES], float& g, float& u) { g = p[0], u = p[1]; }
  // a word of each matrix, from and into as many entries as it holds
  static constexpr int PER = 1;
  static __device__ __forceinline__ void keep_word(const float (&g)[PER], const float (&u)[PER], unsigned (&p)[PLANES]) {
    p[0] = __builtin_bit_cast(unsigned, g[0]), p[1] = __builtin_bit_cast(unsigned, u[0]);
  }
  static __device__ __forceinline__ void back_word(const unsigned (&p)[PLANES], float (&g)[PER], float (&u)[PER]) {
    g[0] = __builtin_bit_cast(float, p[0]), u[0] = __builtin_bit_cast(float, p[1]);
  }
};
struct FfnSaved24 {
  static constexpr int PLANES = 3;
  using U = uint16_t;
  // rounded to the nearest of 24 bits, within 2^-16 of the number, by a carry out of the byte that is left out.  (A NaN stays one: those that
  // sums of 16-bit operands can hold have zeros there.)
  static __device__ __forceinline__ unsigned bits(float v) { return __builtin_bit_cast(unsigned, v) + 0x80u; }
  static __device__ __forceinline__ void keep(float g, float u, U (&p)[PLANES]) {
    const unsigned a = bits(g), b = bits(u);
    p[0] = (U)(a >> 16);
    p[1] = (U)(b >> 16);
    p[2] = (U)((a >> 8 & 0xffu) | (b & 0xff00u));
  }
  static __device__ __forceinline__ void back(const U (&p)[PLANES], float& g, float& u) {
    g = __builtin_bit_cast(float, (unsigned)p[0] << 16 | (p[2] & 0xffu) << 8);
    u = __builtin_bit_cast(float, (unsigned)p[1] << 16 | (p[2] & 0xff00u));
  }
  static constexpr int PER = 2;      // (in bytes: 4 to 7 are the first operand's, 0xc is zero)
  static __device__ __forceinline__ void keep_word(const float (&g)[PER], const float (&u)[PER], unsigned (&p)[PLANES]) {
    const unsigned a0 = bits(g[0]), a1 = bits(g[1]), b0 = bits(u[0]), b1 = bits(u[1]);
    p[0] = __builtin_amdgcn_perm(a1, a0, 0x07060302u);
    p[1] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
    p[2] = __builtin_amdgcn_perm(b0, a0, 0x0c0c0501u) | __builtin_amdgcn_perm(b1, a1, 0x05010c0cu);
  }
  static __device__ __forceinline__ void back_word(const unsigned (&p)[PLANES], float (&g)[PER], float (&u)[PER]) {
    g[0] = __builtin_bit_cast(float, __builtin_amdgcn_perm(p[0], p[2], 0x0504000cu));
    g[1] = __builtin_bit_cast(float, __builtin_amdgcn_perm(p[0], p[2], 0x0706020cu));
    u[0] = __builtin_bit_cast(float, __builtin_amdgcn_perm(p[1], p[2], 0x0504010cu));
    u[1] = __builtin_bit_cast(float, __builtin_amdgcn_perm(p[1], p[2], 0x0706030cu));
  }
};
template <> struct FfnSaved<_Float16> : FfnSaved24 {};
template <> struct FfnSaved<__bf16> : FfnSaved24 {};

}  // namespace sc
