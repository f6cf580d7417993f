// Products of the gated feed-forward block for a few rows: C[i][j] = sum_k P[i][k] Q[j][k], Q a weight matrix that is read once.
//
// Bound by reading the weights.  A workgroup has 16 outputs (of one matrix, or of gate and up) for up to 64 rows; its wavefronts share k
// and add their sums up in LDS, in order.  The weights go from memory straight into the left operand of 16 x 16 matrix instructions (16
// rows x 64 bytes an instruction: the four lanes of a row take 16 bytes each), the rows of P into the right one, so that 1 and 16 rows
// cost the same.
// Up to 4 (8) rows: the 16 rows of an operand are 4 (8) outputs or rows in 4 (2) neighbouring stretches of k.  The diagonal blocks of
// the products are the sums of a stretch each, the rest is not looked at.  4 (2) times as many workgroups, and 256 (128) bytes in a row.
#pragma once
#include "ffn_act.hpp"
#include "ffn_params.hpp"
#include "ffn_saved.hpp"
#include "mma_common.hpp"

namespace sc {

template <int DT> struct FewMma;
template <> struct FewMma<kBF16> {
  static __device__ __forceinline__ v4f mma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct FewMma<kF16> {
  static __device__ __forceinline__ v4f mma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <> struct FewMma<kF32> {      // entry e of the four groups of a row: any pairing of k between the operands is an order of the sum
  static __device__ __forceinline__ v4f mma(v4i a, v4i b, v4f c) {
    const v4f p = __builtin_bit_cast(v4f, a), q = __builtin_bit_cast(v4f, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(p[e], q[e], c, 0, 0, 0);
    return c;
  }
};

// MT tiles of 16 rows; S stretches of k a tile; GATED: q[0] gate, q[1] up; WHOLE: rows are whole 16-byte groups
template <int DT, int MT, int S, bool GATED, bool WHOLE, int WAVES> __global__ __launch_bounds__(64 * WAVES) void ffn_few_kernel(const FfnGemm p) {
  using T = typename Elem<DT>::T;
  constexpr int V = 16 / (int)sizeof(T), STEP = 4 * V * S, MATS = GATED ? 2 : 1, O = 16 / S;
  static_assert(S == 1 || MT == 1, "rows and stretches share the 16 columns");
  constexpr int AHEAD = S == 4 ? 2 : 4;       // k steps whose operands a wavefront asks for at once
  extern __shared__ float few_sum[];          // [WAVES][MATS][MT][64][4]
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int l16 = lane & 15, kg = lane >> 4;
  const int n0 = blockIdx.x * O, row0 = blockIdx.y * (16 * MT);
  const int own = (l16 / O) * (4 * V) + kg * V;      // first of the lane's entries of a step

  const T* w[MATS];
#pragma unroll
  for (int a = 0; a < MATS; ++a) w[a] = static_cast<const T*>(p.q[a]) + (int64_t)min(n0 + l16 % O, p.n - 1) * p.ldq + own;
  const T* x[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int r = min(row0 + 16 * i + l16 % O, p.m - 1);      // a row that is not there: the last one again, whose results are not stored
    x[i] = static_cast<const T*>(p.p[0]) + (p.p_rows ? (int64_t)p.p_rows[r] : r) * p.ldp + own;
  }
  auto group = [=](const T* s, int left) -> v4i {      // `left` entries of a row from here on
    v4i g = {0, 0, 0, 0};
    if (left >= V) {
      if constexpr (WHOLE) g = *reinterpret_cast<const v4i*>(s);
      else __builtin_memcpy(&g, s, 16);
    } else if (!WHOLE && left > 0) {
      T e[V];
#pragma unroll
      for (int u = 0; u < V; ++u) e[u] = u < left ? s[u] : T(0);
      __builtin_memcpy(&g, e, 16);
    }
    return g;
  };

  v4f acc[MATS][MT];
#pragma unroll
  for (int a = 0; a < MATS; ++a)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[a][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  // a wavefront takes AHEAD neighbouring steps, then the next wavefront's follow
  for (int k0 = wave * (AHEAD * STEP); k0 < p.k; k0 += WAVES * (AHEAD * STEP)) {
    v4i wf[MATS][AHEAD], xf[MT][AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int k = k0 + s * STEP, left = p.k - k - own;
#pragma unroll
      for (int a = 0; a < MATS; ++a) wf[a][s] = group(w[a] + k, left);
    }
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int k = k0 + s * STEP, left = p.k - k - own;
#pragma unroll
      for (int i = 0; i < MT; ++i) xf[i][s] = group(x[i] + k, left);
    }
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
#pragma unroll
      for (int a = 0; a < MATS; ++a)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[a][i] = FewMma<DT>::mma(wf[a][s], xf[i][s], acc[a][i]);
  }
  v4f* const mine = reinterpret_cast<v4f*>(few_sum) + (size_t)wave * (MATS * MT * 64) + lane;
#pragma unroll
  for (int a = 0; a < MATS; ++a)
#pragma unroll
    for (int i = 0; i < MT; ++i) mine[(a * MT + i) * 64] = acc[a][i];
  __syncthreads();
  // value (output q of 16, row c of 16) lies in entry q % 4 of lane 16 (q / 4) + c; stretch s: outputs and rows from s O on
  for (int at = t; at < MT * O * O; at += 64 * WAVES) {
    const int q = at % O, r = at / O, n = n0 + q, row = row0 + r;
    float v[MATS];
#pragma unroll
    for (int a = 0; a < MATS; ++a) {
      v[a] = 0.0f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int qs = q + s * O, word = ((r >> 4) * 64 + (qs >> 2) * 16 + (r & 15) + s * O) * 4 + (qs & 3);
#pragma unroll
        for (int u = 0; u < WAVES; ++u) v[a] += few_sum[(u * MATS + a) * (MT * 256) + word];
      }
    }
    if (n >= p.n || row >= p.m) continue;
    if constexpr (GATED) {
      float act, slope;
      ffn_act<T>(p.activation, v[0], act, slope);
      static_cast<T*>(p.c[0])[(int64_t)row * p.ldc + n] = (T)(act * v[1]);
      if (p.saved) {
        using Saved = FfnSaved<T>;
        typename Saved::U kept[Saved::PLANES];
        Saved::keep(v[0], v[1], kept);
#pragma unroll
        for (int s = 0; s < Saved::PLANES; ++s)
          static_cast<typename Saved::U*>(p.saved)[((int64_t)s * p.m + row) * p.n + n] = kept[s];
      }
    } else {
      static_cast<T*>(p.c[0])[(p.c_rows ? (int64_t)p.c_rows[row] : row) * p.ldc + n] = (T)v[0];
    }
  }
}

template <int DT, int MT, int S, bool GATED, bool WHOLE, int WAVES> hipError_t ffn_few_launch(const FfnGemm& g, hipStream_t s) {
  auto kernel = ffn_few_kernel<DT, MT, S, GATED, WHOLE, WAVES>;
  constexpr int lds = WAVES * (GATED ? 2 : 1) * MT * 1024;
  static std::atomic<uint64_t> told{0};
  const hipError_t e = ffn_allow_lds(reinterpret_cast<const void*>(kernel), lds, told);
  if (e != hipSuccess) return e;
  constexpr int outputs = 16 / S;
  kernel<<<dim3((unsigned)((g.n + outputs - 1) / outputs), (unsigned)((g.m + 16 * MT - 1) / (16 * MT))), dim3(64 * WAVES), lds, s>>>(g);
  return hipGetLastError();
}
// Stretches: up to 4 rows and up to 8.  1 row, weights from memory, bf16: gated 2048 -> 5632 9.0 us (5.1 TB/s), in 2 stretches 9.2, in one 11.5;
// 5632 -> 2048 5.6 (4.1 TB/s), 5.5 and 8.1; gated 4096 -> 8192 25 (5.4 TB/s), 27.6 and 27.  Without: sixteen wavefronts where there are
// fewer workgroups than compute units, each with half as many steps.
template <int DT, bool GATED, bool WHOLE> hipError_t ffn_few_rows(const FfnGemm& g, hipStream_t s) {
  if (g.m <= 4) return ffn_few_launch<DT, 1, 4, GATED, WHOLE, 8>(g, s);
  if (g.m <= 8) return ffn_few_launch<DT, 1, 2, GATED, WHOLE, 8>(g, s);
  const bool more = (g.n + 15) / 16 < 256;
  if (g.m <= 16) return more ? ffn_few_launch<DT, 1, 1, GATED, WHOLE, 16>(g, s) : ffn_few_launch<DT, 1, 1, GATED, WHOLE, 8>(g, s);
  if (g.m <= 32) return ffn_few_launch<DT, 2, 1, GATED, WHOLE, 8>(g, s);
  return ffn_few_launch<DT, 4, 1, GATED, WHOLE, 8>(g, s);
}
template <int DT> hipError_t ffn_few_type(bool gated, const FfnGemm& g, bool whole, hipStream_t s) {
  if (gated) return whole ? ffn_few_rows<DT, true, true>(g, s) : ffn_few_rows<DT, true, false>(g, s);
  return whole ? ffn_few_rows<DT, false, true>(g, s) : ffn_few_rows<DT, false, false>(g, s);
}

}  // namespace sc
