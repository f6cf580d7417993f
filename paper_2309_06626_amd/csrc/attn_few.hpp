// Attention over packed sequences where there are few rows: forward pass and gradients, the mathematics of attn_kernel.hpp.
//
// A workgroup takes 32 packed rows (or keys) in place of 128 or 256, and its four wavefronts every fourth block of 32 of what passes by, each on its
// own: a transfer, two or four products and the softmax between, without a meeting.  Their shares (of the forward pass with maxima and sums) are joined
// in LDS at the end, in a fixed order.  Keys and values are read four times as often, which does not matter as long as a compute unit has no more than
// a few workgroups.
//
// Bound by the latency of a wavefront's steps, of which it has a quarter as many.  Training, gradients and in floats the forward pass by these kernels:
// 2 048 rows, 16 heads of 128 on 4 in bf16, 235 us (367 with tiles of 128 and 256 rows); 512 rows, 8 heads of 64 floats, 71 (175); 8 x 196 rows of
// which 30 % are dropped, 10 heads of 41 floats, 84 (105), where transfers of 4 bytes a lane and their addresses are half of it (40 channels: 57).
#pragma once
#include "attn_kernel.hpp"

namespace sc {

constexpr int kFewWaves = 4;

// Shares of the wavefronts in LDS: [wave][row][DP], rows padded by a 16-byte group, and what belongs to a row behind.
template <int DT, int DP, int VEC> struct AttnFew {
  using A = AttnTile<DT, DP>;
  using T = typename A::T;
  static constexpr int TILE = 32 * A::RB, STATS = 256;           // of a wavefront: two tiles, and a row's two statistics
  static constexpr int WAVE = 2 * TILE + STATS, ROW = DP + 4, SHARES = kFewWaves * 32 * ROW;
  static constexpr int LDS = kFewWaves * WAVE > (SHARES + 2 * kFewWaves * 32) * 4 ? kFewWaves * WAVE : (SHARES + 2 * kFewWaves * 32) * 4;
  // When shares are joined: lanes of a row, and channels of a lane.  One where rows are not whole groups, so that lanes write side by side.
  static constexpr int CH = VEC == 2 ? DP / 8 : 1, LANES = DP / CH, ROWS = 64 * kFewWaves / LANES;

  static __device__ __forceinline__ void put(float* shares, int wave, int l32, int h, const floatx16 (&acc)[A::DB]) {
#pragma unroll
    for (int db = 0; db < A::DB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v4f part;
#pragma unroll
        for (int e = 0; e < 4; ++e) part[e] = acc[db][4 * q + e];
        *reinterpret_cast<v4f*>(shares + (wave * 32 + l32) * ROW + 32 * db + 16 * h + 4 * q) = part;
      }
  }
  static __device__ __forceinline__ void add(const float* shares, int wave, int row, int c0, float factor, float (&x)[CH]) {
    const float* const from = shares + (wave * 32 + row) * ROW + c0;
    if constexpr (CH == 1) {
      x[0] = __builtin_fmaf(*from, factor, x[0]);
    } else {
#pragma unroll
      for (int q = 0; q < CH / 4; ++q) {
        const v4f part = *reinterpret_cast<const v4f*>(from + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * q + e] = __builtin_fmaf(part[e], factor, x[4 * q + e]);
      }
    }
  }
  static __device__ __forceinline__ void write(T* row, int c0, int d, const float (&x)[CH], float factor) {
    if constexpr (CH == 1) {
      if (c0 < d) row[c0] = A::E::from_float(x[0] * factor);
    } else {
      T r[CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) r[i] = A::E::from_float(x[i] * factor);
      v4i g[CH / A::V];
      __builtin_memcpy(g, r, sizeof(r));
#pragma unroll
      for (int i = 0; i < CH / A::V; ++i)
        if (c0 + i * A::V < d) *reinterpret_cast<v4i*>(row + c0 + i * A::V) = g[i];
    }
  }
  // the sum of the shares
  static __device__ __forceinline__ void sum(const float* shares, int row, int c0, float (&x)[CH]) {
#pragma unroll
    for (int i = 0; i < CH; ++i) x[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) add(shares, w, row, c0, 1.0f, x);
  }
};

// all but the youngest N of this wavefront's transfers have landed
template <int N> __device__ __forceinline__ void few_wait() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N < 63 ? N : 63) : "memory"); }
__device__ __forceinline__ void few_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }      // what was asked of LDS is in registers

// d, so that comparisons with it are made anew: held from place to place, they take all scalar registers
__device__ __forceinline__ int few_width(const AttnParams& p) {
  int d = __builtin_amdgcn_readfirstlane(p.d);
  asm volatile("" : "+s"(d));
  return d;
}

// what lane r has; ALL: r is the same in all lanes, as it is where 4-byte transfers take a row at once
template <bool ALL> __device__ __forceinline__ int few_of(int x, int r) { return ALL ? __builtin_amdgcn_readlane(x, __builtin_amdgcn_readfirstlane(r)) : __shfl(x, r); }
template <bool ALL, class T> __device__ __forceinline__ const T* few_of(const T* x, int r) {
  const uint64_t at = reinterpret_cast<uint64_t>(x);
  return reinterpret_cast<const T*>((uint64_t)(unsigned)few_of<ALL>((int)(at >> 32), r) << 32 | (unsigned)few_of<ALL>((int)at, r));
}

// Rows of a transfer: row r of the tile is that of lane r.
template <class A, int VEC, class T> __device__ __forceinline__ auto few_place(const T* base, int64_t stride, int rows) {
  constexpr bool ALL = VEC == 1 && A::RB >= 256;
  if constexpr (ALL) {
    const T* const at = rows < 0 ? nullptr : base + rows * stride;
    return [=](int r) { return few_of<ALL>(at, r); };
  } else {
    return [=](int r) -> const T* {
      const int row = few_of<ALL>(rows, r);
      return row < 0 ? nullptr : base + row * stride;
    };
  }
}

// The workgroup's own rows of N tensors, `at` being that of a lane (null: none).  Where rows are not whole 16-byte groups, a lane that read a row by
// itself would ask for a cache line an entry (the 84 us above 91): they come as tiles, one a wavefront,
// into the places where what passes by will lie.
template <class F, int VEC, int N, class T>
__device__ __forceinline__ void few_own(const AttnParams& p, unsigned lds, const T* const (&at)[N], v4i (&f)[N][F::A::KS]) {
  using A = typename F::A;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if constexpr (VEC == 2) {
#pragma unroll
    for (int k = 0; k < N; ++k) A::template read_row<2>(at[k], p.d, lane >> 5, at[k] != nullptr, f[k]);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (wave == k) A::template request<32, 64, VEC>(lds + k * F::WAVE, p.d, [&](int r) { return few_of<VEC == 1 && A::RB >= 256>(at[k], r); }, lane);
    attn_meet<0>();
    const typename A::Along along = A::along(lane);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int ks = 0; ks < A::KS; ++ks) f[k][ks] = A::read_along(along, lds + k * F::WAVE, 0, ks);
    attn_meet<0>();
  }
}

// rows of the tensors that hold kept rows first + j0 .. + 31 of a sequence of n, a lane each
__device__ __forceinline__ int few_look_up(const AttnParams& p, int first, int j0, int n) {
  const int j = j0 + (threadIdx.x & 31);
  if (j >= n) return -1;
  return p.map ? p.map[first + j] : first + j;
}
template <int DT, int DP, int VEC> __global__ __launch_bounds__(64 * kFewWaves, DT == kF32 && DP > 64 ? 1 : 2) void attn_few_forward_kernel(const AttnParams p) {
  using F = AttnFew<DT, DP, VEC>;
  using A = typename F::A;
  using T = typename A::T;
  constexpr int J = VEC == 0 ? 0 : VEC == 1 ? F::TILE / 256 : F::TILE / 1024;      // transfers of a tile
  extern __shared__ __align__(16) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, l32 = lane & 31;

  if (attn_zeros_of_dropped<kFewWaves>(p)) return;
  const AttnWork w = attn_work(p);
  const int n = w.item.rows, first = w.item.first, packed = n * p.group;
  const int r0 = w.item.tile * 32, r = r0 + l32;
  const bool there = r < packed;
  const int i = there ? r / p.group : 0, head = w.head * p.group + (there ? r - i * p.group : 0);
  const int64_t row = p.map ? p.map[first + i] : first + i;
  const AttnSpan mine = attn_keys(p, i, n), from = attn_keys(p, r0 / p.group, n), to = attn_keys(p, (min(r0 + 32, packed) - 1) / p.group, n);
  const int k_begin = from.lo / 32 * 32, blocks = (to.hi - k_begin) / 32 + 1, own = (blocks - wave + kFewWaves - 1) / kFewWaves;
  const int lo = there ? mine.lo : 0x40000000;
  const unsigned span = there ? mine.hi - mine.lo : 0;

  const T* const k_base = static_cast<const T*>(p.k) + (int64_t)w.head * p.d;
  const T* const v_base = static_cast<const T*>(p.v) + (int64_t)w.head * p.d;
  const unsigned lds = attn_lds(smem) + wave * F::WAVE;
  auto key0 = [&](int b) { return k_begin + (wave + kFewWaves * b) * 32; };
  auto request = [&](const T* base, int64_t stride, int rows, unsigned at) {
    A::template request<32, 64, VEC>(lds + at, few_width(p), few_place<A, VEC>(base, stride, rows), lane);
  };
  int rows = own > 0 ? few_look_up(p, first, key0(0), n) : -1, rows_next = own > 1 ? few_look_up(p, first, key0(1), n) : -1;
  v4i own_f[1][A::KS], (&qf)[A::KS] = own_f[0];
  const T* const own_at[1] = {there ? static_cast<const T*>(p.q) + row * p.q_stride + (int64_t)head * p.d : nullptr};
  few_own<F, VEC>(p, attn_lds(smem), own_at, own_f);
  if (own > 0) {
    request(k_base, p.k_stride, rows, 0);
    request(v_base, p.v_stride, rows, F::TILE);
  }
  const float c = p.scale * kAttnLog2e;
  typename A::Along along = A::along(lane);
  typename A::Across across = A::across(lane);
  along.add(lds);
  across.add(lds);
  floatx16 acc[A::DB], s;
#pragma unroll
  for (int db = 0; db < A::DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.0f;
  float m = -INFINITY, sum = 0.0f;                     // m is a maximum times c, as it was rounded

  for (int b = 0; b < own; ++b) {
    const bool more = b + 1 < own;
    few_wait<J>();                                     // (the values, which came behind the keys, may be on their way)
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(s, A::read_along(along, 0, 0, ks), qf[ks]);
    few_read();
    rows = rows_next;
    if (more) request(k_base, p.k_stride, rows, 0);
    const int k0 = key0(b);
    if (k0 < to.lo || k0 + 31 > from.hi || r0 + 32 > packed) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = (unsigned)(k0 + 4 * h - lo + (8 * (v >> 2) + (v & 3))) <= span ? s[v] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) top = fmaxf(top, s[v]);
    top = fmaxf(attn_max_halves(top) * c, m);
    if (attn_any(top > m + 8.0f)) {                    // (a maximum that grew by less than 2^8 stays, as in the other kernel)
      const float less = attn_exp2(m - (top == -INFINITY ? 0.0f : top));
      m = top;
      sum *= less;
#pragma unroll
      for (int db = 0; db < A::DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[db][v] *= less;
    }
    static_assert(DT == kF32, "weights of f16 would be formed larger");
    const float shift = attn_shift<false>(m);
    float part[4];                                     // (one weight after the other is lost beside a large sum)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s[v] = attn_exp2(__builtin_fmaf(s[v], c, -shift));
      part[v & 3] = v < 4 ? s[v] : part[v & 3] + s[v];
    }
    sum += (part[0] + part[1]) + (part[2] + part[3]);
    v4i pf[A::SS];
    A::pack(s, pf);
    if (more) few_wait<J>();
    else few_wait<0>();
#pragma unroll
    for (int ss = 0; ss < A::SS; ++ss)
#pragma unroll
      for (int db = 0; db < A::DB; ++db) A::E::mma(acc[db], A::read_across(across, F::TILE, 0, ss, db), pf[ss]);
    few_read();
    if (more) {
      request(v_base, p.v_stride, rows, F::TILE);
      rows_next = b + 2 < own ? few_look_up(p, first, key0(b + 2), n) : -1;
    }
  }
  sum = attn_add_halves(sum);

  float *const shares = reinterpret_cast<float*>(smem), *const s_max = shares + F::SHARES, *const s_sum = s_max + kFewWaves * 32;
  __syncthreads();
  F::put(shares, wave, l32, h, acc);
  if (h == 0) {
    s_max[wave * 32 + l32] = m;
    s_sum[wave * 32 + l32] = sum;
  }
  __syncthreads();
  const int c0 = t % F::LANES * F::CH;
#pragma unroll 4
  for (int r_out = t / F::LANES; r_out < min(32, packed - r0); r_out += F::ROWS) {
    float top = s_max[r_out], all = 0.0f, x[F::CH];
#pragma unroll
    for (int v = 1; v < kFewWaves; ++v) top = fmaxf(top, s_max[v * 32 + r_out]);
#pragma unroll
    for (int e = 0; e < F::CH; ++e) x[e] = 0.0f;
#pragma unroll
    for (int v = 0; v < kFewWaves; ++v) {
      const float part = s_sum[v * 32 + r_out];
      if (part == 0.0f) continue;
      const float f = attn_exp2(s_max[v * 32 + r_out] - top);
      all += part * f;
      F::add(shares, v, r_out, c0, f, x);
    }
    all = attn_total(top, all);
    const int i_out = (r0 + r_out) / p.group, head_out = w.head * p.group + (r0 + r_out - i_out * p.group);
    const int64_t row_out = p.map ? p.map[first + i_out] : first + i_out;
    if (p.lse && c0 == 0) p.lse[(int64_t)(first + i_out) * p.heads + head_out] = all == 0.0f ? -INFINITY : attn_lse<DT>(top, all);
    const float per = all > 0.0f ? 1.0f / all : all == 0.0f ? 0.0f : all;      // (NaN stays)
    F::write(static_cast<T*>(p.out) + (row_out * p.heads + head_out) * p.d, c0, p.d, x, per);
  }
}

template <int DT, int DP, int VEC> __global__ __launch_bounds__(64 * kFewWaves, DP > 64 && (DT == kF32 || VEC < 2) ? 1 : 2) void attn_few_rows_kernel(const AttnParams p) {
  using F = AttnFew<DT, DP, VEC>;
  using A = typename F::A;
  using T = typename A::T;
  extern __shared__ __align__(16) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, l32 = lane & 31;

  if (attn_zeros_of_dropped<kFewWaves>(p)) return;
  const AttnWork w = attn_work(p);
  const int n = w.item.rows, first = w.item.first, packed = n * p.group;
  const int r0 = w.item.tile * 32, r = r0 + l32;
  const bool there = r < packed;
  const int i = there ? r / p.group : 0, head = w.head * p.group + (there ? r - i * p.group : 0);
  const int64_t row = p.map ? p.map[first + i] : first + i;
  const AttnSpan mine = attn_keys(p, i, n), from = attn_keys(p, r0 / p.group, n), to = attn_keys(p, (min(r0 + 32, packed) - 1) / p.group, n);
  const int k_begin = from.lo / 32 * 32, blocks = (to.hi - k_begin) / 32 + 1, own = (blocks - wave + kFewWaves - 1) / kFewWaves;
  const int lo = there ? mine.lo : 0x40000000;
  const unsigned span = there ? mine.hi - mine.lo : 0;

  const T* const k_base = static_cast<const T*>(p.k) + (int64_t)w.head * p.d;
  const T* const v_base = static_cast<const T*>(p.v) + (int64_t)w.head * p.d;
  const unsigned lds = attn_lds(smem) + wave * F::WAVE;
  auto key0 = [&](int b) { return k_begin + (wave + kFewWaves * b) * 32; };
  auto request = [&](const T* base, int64_t stride, int rows, unsigned at) {
    A::template request<32, 64, VEC>(lds + at, few_width(p), few_place<A, VEC>(base, stride, rows), lane);
  };
  int rows = own > 0 ? few_look_up(p, first, key0(0), n) : -1, rows_next = own > 1 ? few_look_up(p, first, key0(1), n) : -1;
  v4i own_f[3][A::KS], (&qf)[A::KS] = own_f[0], (&gf)[A::KS] = own_f[1], (&of)[A::KS] = own_f[2];
  const int64_t own_place = (row * p.heads + head) * p.d;
  const T* const own_at[3] = {there ? static_cast<const T*>(p.q) + row * p.q_stride + (int64_t)head * p.d : nullptr,
                              there ? static_cast<const T*>(p.d_o) + own_place : nullptr, there ? static_cast<const T*>(p.o) + own_place : nullptr};
  few_own<F, VEC>(p, attn_lds(smem), own_at, own_f);
  const float c = p.scale * kAttnLog2e;
  float lse2 = 0.0f, keys_lse2 = 0.0f, delta = 0.0f;
  const int64_t stat = (int64_t)(first + i) * p.heads + head;
  {
    lse2 = there ? p.lse[stat] : 0.0f;
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) {
      T a[A::V], b[A::V];
      __builtin_memcpy(a, &gf[ks], 16);
      __builtin_memcpy(b, &of[ks], 16);
#pragma unroll
      for (int e = 0; e < A::V; ++e) delta += (float)a[e] * (float)b[e];
    }
    delta = attn_add_halves(delta);
    keys_lse2 = attn_lse2(lse2, kAttnKeysUp<DT>);
    lse2 = attn_lse2(lse2);
  }
  __builtin_amdgcn_sched_barrier(0);
  if (own > 0) {
    request(v_base, p.v_stride, rows, F::TILE);
    request(k_base, p.k_stride, rows, 0);
  }
  typename A::Along along = A::along(lane);
  typename A::Across across = A::across(lane);
  along.add(lds);
  across.add(lds);
  floatx16 acc[A::DB], s, g;
#pragma unroll
  for (int db = 0; db < A::DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.0f;
  float part[2] = {0.0f, 0.0f};                        // delta from the probabilities themselves, for the keys

  for (int b = 0; b < own; ++b) {
    const bool more = b + 1 < own;
    few_wait<0>();
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = g[v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(g, A::read_along(along, F::TILE, 0, ks), gf[ks]);
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(s, A::read_along(along, 0, 0, ks), qf[ks]);
    few_read();
    rows = rows_next;
    if (more) request(v_base, p.v_stride, rows, F::TILE);
    const int k0 = key0(b);
    if (k0 < to.lo || k0 + 31 > from.hi || r0 + 32 > packed) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = (unsigned)(k0 + 4 * h - lo + (8 * (v >> 2) + (v & 3))) <= span ? s[v] : -INFINITY;
    }
    v4i pf[A::SS];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float e = attn_exp2(__builtin_fmaf(s[v], c, -lse2));
      part[v & 1] = __builtin_fmaf(e, g[v], part[v & 1]);
      g[v] = e * (g[v] - delta);
    }
    A::pack(g, pf);
#pragma unroll
    for (int ss = 0; ss < A::SS; ++ss)
#pragma unroll
      for (int db = 0; db < A::DB; ++db) A::E::mma(acc[db], A::read_across(across, 0, 0, ss, db), pf[ss]);
    few_read();
    if (more) {
      request(k_base, p.k_stride, rows, 0);
      rows_next = b + 2 < own ? few_look_up(p, first, key0(b + 2), n) : -1;
    }
  }
  delta = attn_add_halves(part[0] + part[1]);

  float *const shares = reinterpret_cast<float*>(smem), *const s_delta = shares + F::SHARES;
  __syncthreads();
  F::put(shares, wave, l32, h, acc);
  if (h == 0) s_delta[wave * 32 + l32] = delta;
  if (wave == 0 && h == 0 && there) p.stats[0][stat] = keys_lse2;
  __syncthreads();
  const int c0 = t % F::LANES * F::CH;
#pragma unroll 4
  for (int r_out = t / F::LANES; r_out < min(32, packed - r0); r_out += F::ROWS) {
    float x[F::CH];
    F::sum(shares, r_out, c0, x);
    const int i_out = (r0 + r_out) / p.group, head_out = w.head * p.group + (r0 + r_out - i_out * p.group);
    if (c0 == 0) p.stats[1][(int64_t)(first + i_out) * p.heads + head_out] = ((s_delta[r_out] + s_delta[32 + r_out]) + (s_delta[64 + r_out] + s_delta[96 + r_out])) * kAttnKeysUnit<DT>;
    const int64_t row_out = p.map ? p.map[first + i_out] : first + i_out;
    F::write(static_cast<T*>(p.dq) + row_out * p.dq_stride + (int64_t)head_out * p.d, c0, p.d, x, p.scale);
  }
}

template <int DT, int DP, int VEC> __global__ __launch_bounds__(64 * kFewWaves, DP > 64 || (DT == kF32 && VEC < 2) ? 1 : 2) void attn_few_keys_kernel(const AttnParams p) {
  using F = AttnFew<DT, DP, VEC>;
  using A = typename F::A;
  using T = typename A::T;
  extern __shared__ __align__(16) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, l32 = lane & 31;

  const AttnWork w = attn_work(p);
  const int n = w.item.rows, first = w.item.first, group = p.group;
  const int j0 = w.item.tile * 32, j = j0 + l32;
  const bool there = j < n;
  const int64_t row = there ? (p.map ? p.map[first + j] : first + j) : 0;
  const AttnSpan mine = attn_rows(p, there ? j : 0, n), from = attn_rows(p, j0, n), to = attn_rows(p, min(j0 + 32, n) - 1, n);
  // packed rows
  const int r_begin = from.lo * group / 32 * 32, blocks = ((to.hi + 1) * group - r_begin + 31) / 32, own = (blocks - wave + kFewWaves - 1) / kFewWaves;
  const int lo = there ? mine.lo * group : 0x40000000;
  const unsigned span = there ? (mine.hi - mine.lo + 1) * group - 1 : 0;
  const int all_lo = to.lo * group, all_hi = (from.hi + 1) * group - 1;      // rows that see all of the keys

  const T* const q_base = static_cast<const T*>(p.q) + (int64_t)w.head * group * p.d;
  const T* const g_base = static_cast<const T*>(p.d_o) + (int64_t)w.head * group * p.d;
  const int64_t g_stride = (int64_t)p.heads * p.d;
  const unsigned lds = attn_lds(smem) + wave * F::WAVE;
  auto row0 = [&](int b) { return r_begin + (wave + kFewWaves * b) * 32; };
  auto request = [&](const T* base, int64_t stride, int r0, int rows, unsigned at) {
    // packed row l32 of the tile, and its place among the rows that were looked up
    const int rem = __builtin_amdgcn_readfirstlane(r0 % group), past = (int)((unsigned)(rem + l32) * p.magic >> 20), row = __shfl(rows, past);
    const T* const own_row = row < 0 ? nullptr : base + row * stride + (rem + l32 - past * group) * p.d;
    auto place = [=](int r) { return few_of<VEC == 1 && A::RB >= 256>(own_row, r); };
    A::template request<32, 64, VEC>(lds + at, few_width(p), place, lane);
  };
  // lse (in exponents of 2) of the first half's lanes, delta of the second's
  auto request_stats = [&](int r0) {
    const int at = r0 + l32, i = at / group;
    const float* of = p.stats[h] + (int64_t)(first + i) * p.heads + w.head * group + (at - i * group);
    attn_dma4(i < n ? (const void*)of : (const void*)&attn_zeros, lds + 2 * F::TILE);
  };
  int rows = own > 0 ? few_look_up(p, first, row0(0) / group, n) : -1, rows_next = own > 1 ? few_look_up(p, first, row0(1) / group, n) : -1;
  v4i own_f[2][A::KS], (&kf)[A::KS] = own_f[0], (&vf)[A::KS] = own_f[1];
  const T* const own_at[2] = {there ? static_cast<const T*>(p.k) + row * p.k_stride + (int64_t)w.head * p.d : nullptr,
                              there ? static_cast<const T*>(p.v) + row * p.v_stride + (int64_t)w.head * p.d : nullptr};
  few_own<F, VEC>(p, attn_lds(smem), own_at, own_f);
  if (own > 0) {
    request_stats(row0(0));
    request(q_base, p.q_stride, row0(0), rows, 0);
    request(g_base, g_stride, row0(0), rows, F::TILE);
  }
  const float c = p.scale * kAttnLog2e;
  typename A::Along along = A::along(lane);
  typename A::Across across = A::across(lane);
  along.add(lds);
  across.add(lds);
  const unsigned at_stats = lds + 2 * F::TILE + 16 * h;
  typedef __attribute__((address_space(3))) const v4f lds_v4f;
  floatx16 dk[A::DB], dv[A::DB], s, g;
#pragma unroll
  for (int db = 0; db < A::DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) dk[db][v] = dv[db][v] = 0.0f;

  for (int b = 0; b < own; ++b) {
    const bool more = b + 1 < own;
    few_wait<0>();
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = g[v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(s, A::read_along(along, 0, 0, ks), kf[ks]);
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(g, A::read_along(along, F::TILE, 0, ks), vf[ks]);
    const int r0 = row0(b);
    if (r0 < all_lo || r0 + 31 > all_hi || j0 + 32 > n) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = (unsigned)(r0 + 4 * h - lo + (8 * (v >> 2) + (v & 3))) <= span ? s[v] : -INFINITY;
    }
    v4i pf[A::SS], df[A::SS];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const v4f lse2 = *(lds_v4f*)(uint64_t)(at_stats + 32 * a), delta = *(lds_v4f*)(uint64_t)(at_stats + 128 + 32 * a);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = 4 * a + e;
        s[v] = attn_exp2(__builtin_fmaf(s[v], c, -lse2[e]));
        g[v] = attn_keys_ds<DT>(s[v], g[v], delta[e]);
      }
    }
    A::pack(s, pf);
    A::pack(g, df);
#pragma unroll
    for (int ss = 0; ss < A::SS; ++ss)
#pragma unroll
      for (int db = 0; db < A::DB; ++db) A::E::mma(dv[db], A::read_across(across, F::TILE, 0, ss, db), pf[ss]);
    few_read();
    rows = rows_next;
    if (more) {
      request_stats(row0(b + 1));
      request(g_base, g_stride, row0(b + 1), rows, F::TILE);
    }
#pragma unroll
    for (int ss = 0; ss < A::SS; ++ss)
#pragma unroll
      for (int db = 0; db < A::DB; ++db) A::E::mma(dk[db], A::read_across(across, 0, 0, ss, db), df[ss]);
    few_read();
    if (more) {
      request(q_base, p.q_stride, row0(b + 1), rows, 0);
      rows_next = b + 2 < own ? few_look_up(p, first, row0(b + 2) / group, n) : -1;
    }
  }

  float* const shares = reinterpret_cast<float*>(smem);
  const int c0 = t % F::LANES * F::CH;
  auto join = [&](const floatx16 (&acc)[A::DB], void* out, int64_t stride, float factor) {
    __syncthreads();
    F::put(shares, wave, l32, h, acc);
    __syncthreads();
#pragma unroll 4
    for (int j_out = t / F::LANES; j_out < min(32, n - j0); j_out += F::ROWS) {
      float x[F::CH];
      F::sum(shares, j_out, c0, x);
      const int64_t row_out = p.map ? p.map[first + j0 + j_out] : first + j0 + j_out;
      F::write(static_cast<T*>(out) + row_out * stride + (int64_t)w.head * p.d, c0, p.d, x, factor);
    }
  };
  join(dv, p.dv, p.dv_stride, kAttnKeysUnit<DT>);
  join(dk, p.dk, p.dk_stride, p.scale);
}

template <int DT> hipError_t attn_few_launch(int what, const AttnParams& p, int vec, hipStream_t s) {
  auto start = [&](auto width, auto level) {
    constexpr int DP = decltype(width)::value, VEC = decltype(level)::value, lds = AttnFew<DT, DP, VEC>::LDS;
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    if constexpr (DT == kF32) {
      if (what == kAttnForward) return attn_start(attn_few_forward_kernel<DT, DP, VEC>, 64 * kFewWaves, lds, p, s);
    }
    if (what == kAttnBackwardQ) return attn_start(attn_few_rows_kernel<DT, DP, VEC>, 64 * kFewWaves, lds, p, s);
    return attn_start(attn_few_keys_kernel<DT, DP, VEC>, 64 * kFewWaves, lds, p, s);
  };
  auto of_level = [&](auto level) { return p.d <= 64 ? start(attn_c<64>, level) : start(attn_c<128>, level); };
  if (vec == 2) return of_level(attn_c<2>);
  if constexpr (DT != kF32) {
    if (vec == 0) return of_level(attn_c<0>);
  }
  return of_level(attn_c<1>);
}

}  // namespace sc
