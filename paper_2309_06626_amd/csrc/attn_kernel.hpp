// Attention over packed sequences of kept rows: forward pass and gradients.
//
//   s_ij = scale q_i . k_j of the keys that row i sees,  p = exp(s - lse_i),  o_i = sum_j p_ij v_j
//   D_i = do_i . o_i,  ds = p (do_i . v_j - D_i),  dq_i = scale sum_j ds k_j,  dk_j = scale sum_i ds q_i,  dv_j = sum_i p do_i
//
// Query heads that share a key-value head are rows of one matrix: packed row r of a sequence is head r % group of its row r / group, so that a
// tile of keys serves all of them, and a key's gradient is a sum over rows that one wavefront makes.
//
// Bound by the matrix cores and, under full load, by power.  A wavefront's 32 rows (or keys) are a column of the products, one a lane: softmax
// needs one exchange between the halves of the wavefront, and the results of a product are the operand of the next one where they lie.
// Gradients take seven products in place of the five that sums over keys and rows at once would, which needed atomics, whose order
// changes results, or the scores in memory.  Measured, bf16, heads of 128: 8 192 causal rows of 32 heads 483 to 502 us (1 090 to 1 140 TFLOP/s
// at 1.9 to 2.1 GHz, matrix pipes busy 53 to 57 % of cycles, the vector unit as much of them; the library's large product 1 440 to 1 560); a
// step more evenly shared between the two units took 4 % fewer cycles, as much time at a lower clock.  4 x 2 048 rows, 16 heads, gradients:
// queries 111 to 123 (840), keys and values 165 to 181 (790).
#pragma once
#include "attn_params.hpp"
#include "attn_tile.hpp"

#include <math.h>

namespace sc {

constexpr float kAttnLog2e = 1.4426950408889634f;
// a row's lse, and what is taken off in the exponent of 2: in 64 bits, because the error of either is one of all the row's probabilities.  A row
// whose scores are all -infinity has none: less 0, in place of less its lse, they are 0.
template <int DT> __device__ __forceinline__ float attn_lse(float shift, float sum) {
  if constexpr (DT == kF16) return (float)(((double)shift + kAttnUp) * 0.6931471805599453 + (double)__builtin_logf(__builtin_amdgcn_ldexpf(sum, -kAttnUp)));
  return (float)((double)shift * 0.6931471805599453 + (double)__builtin_logf(sum));
}
__device__ __forceinline__ float attn_lse2(float lse, int up = 0) { return (float)((lse == -INFINITY ? 0.0 : (double)lse * 1.4426950408889634) - up); }

// The keys' gradients take probabilities as operands.  f16's are formed 2^14 times as large, so that those down to 2^-28 keep their digits and those
// to 2^-39 are not lost (65 536 rows with 2^-25 each are 2^-9 of their gradients); their lse and delta are written for it, dv is divided by it.
template <int DT> constexpr int kAttnKeysUp = DT == kF16 ? 14 : 0;
template <int DT> constexpr float kAttnKeysUnit = DT == kF16 ? 0x1p-14f : 1.0f;
// gradient of a score: p (do . v - delta)
template <int DT> __device__ __forceinline__ float attn_keys_ds(float p, float g, float delta) {
  return p * (DT == kF16 ? __builtin_fmaf(g, kAttnKeysUnit<DT>, -delta) : g - delta);
}

template <int N> constexpr std::integral_constant<int, N> attn_c{};
template <int I, int N, class Fn> __device__ __forceinline__ void attn_for(Fn&& f) {
  if constexpr (I < N) {
    f(attn_c<I>);
    attn_for<I + 1, N>(f);
  }
}

// How rows are read, the VEC of the kernels: by entries (0), 4 bytes (1) or 16 (2); plain ones, besides, are of 64 or 128 channels and follow
// each other at a distance that offsets of 32 bits span.
constexpr int kAttnPlain = 3;

// Consecutive workgroups go round the eight dies.  Where the key-value heads are a multiple of eight, each die takes heads of its own, whose
// keys and values stay in its L2; otherwise heads are neighbours.  Items come with the longest first.
struct AttnWork { AttnItem item; int head; };
__device__ __forceinline__ AttnWork attn_work(const AttnParams& p) {
  int item, head;
  const int b = blockIdx.x;
  if (p.kv_heads % 8 == 0) {
    const int i = b >> 3;
    head = (b & 7) + 8 * (i / p.n_items);
    item = i % p.n_items;
  } else {
    head = b % p.kv_heads;
    item = b / p.kv_heads;
  }
  return {p.items[item], head};
}

// The workgroups behind those of the items write the zeros of dropped rows, a wavefront a row.  True for such a one.
template <int NW> __device__ __forceinline__ bool attn_zeros_of_dropped(const AttnParams& p) {
  const int block = (int)blockIdx.x - p.n_items * p.kv_heads;
  if (block < 0) return false;
  for (int64_t r = (int64_t)block * NW + (threadIdx.x >> 6); r < p.zeros.rows; r += (int64_t)p.zeros.blocks * NW) {
    if (p.zeros.slot && p.zeros.slot[r] >= 0) continue;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      unsigned char* const row = static_cast<unsigned char*>(p.zeros.out[k]) + r * p.zeros.stride[k];
      if (p.zeros.vec) {
        for (int64_t i = (threadIdx.x & 63) * 16; i < p.zeros.width[k]; i += 1024) *reinterpret_cast<v4i*>(row + i) = v4i{0, 0, 0, 0};
      } else {
        for (int64_t i = (threadIdx.x & 63) * 2; i < p.zeros.width[k]; i += 128) *reinterpret_cast<uint16_t*>(row + i) = 0;
      }
    }
  }
  return true;
}

// Keys that row i of a sequence of n rows sees: lo .. hi.
struct AttnSpan { int lo, hi; };
__device__ __forceinline__ AttnSpan attn_keys(const AttnParams& p, int i, int n) {
  AttnSpan s = {0, n - 1};
  if (p.window) {
    s.lo = i >= p.window ? i - p.window + 1 : 0;
    if (p.window <= n - 1 - i) s.hi = i + p.window - 1;
  }
  if (p.causal) s.hi = i;
  return s;
}
// Rows that see key j.
__device__ __forceinline__ AttnSpan attn_rows(const AttnParams& p, int j, int n) {
  AttnSpan s = {0, n - 1};
  if (p.window) {
    if (p.window <= n - 1 - j) s.hi = j + p.window - 1;
    s.lo = j >= p.window ? j - p.window + 1 : 0;
  }
  if (p.causal) s.lo = j;
  return s;
}

// Rows of the tensors that hold kept rows first + j0 .. + 63 of a sequence of n, a lane each (-1: none).  Asked for a tile ahead: a look-up at
// the place where it is taken would wait for all transfers on their way.
__device__ __forceinline__ int attn_look_up(const AttnParams& p, int first, int j0, int n) {
  const int j = j0 + (threadIdx.x & 63);
  if (j >= n) return -1;
  return p.map ? p.map[first + j] : first + j;
}

// ---- forward ---------------------------------------------------------------------------------------------------------------------------
// A wavefront has 32 packed rows, one a lane and half; keys pass by in tiles.  While the matrix unit multiplies the keys of one tile, the
// vector unit takes the exponentials of the tile before, and while it multiplies their values, the maximum of this one (one after the
// other, with operands read as they are taken: 1 106 us for the 8 192 rows above; side by side 710; with the probabilities held where they are
// formed and sums moved to the values' half 478).  Two tiles of keys and two of values lie in LDS: what is asked for behind one meeting is
// there at the next.
template <int DT, int DP, int NW, int TK, int VEC>
__global__ __launch_bounds__(64 * NW, DP > 64 && (DT == kF32 || (VEC < 2 && NW == 4)) ? 1 : 2) void attn_forward_kernel(const AttnParams p) {
  using A = AttnTile<DT, DP>;
  using T = typename A::T;
  constexpr bool PLAIN = VEC == kAttnPlain;
  constexpr int LOADS = PLAIN ? 2 : VEC, NT = 64 * NW, KB = TK / 32;
  constexpr int TILE = TK * A::RB;                     // LDS: two tiles of keys, two of values
  extern __shared__ __align__(16) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, l32 = lane & 31;

  if (attn_zeros_of_dropped<NW>(p)) return;
  const AttnWork w = attn_work(p);
  const int n = w.item.rows, first = w.item.first, packed = n * p.group;
  const int r0 = w.item.tile * 32 * NW, r_wave = r0 + wave * 32, r = r_wave + l32;
  const bool there = r < packed, any = r_wave < packed;
  const int i = there ? r / p.group : 0, head = w.head * p.group + (there ? r - i * p.group : 0);
  const int64_t row = p.map ? p.map[first + i] : first + i;
  const AttnSpan mine = attn_keys(p, i, n);
  // of the whole wavefront and workgroup: rows are in ascending order, and so are both ends of what they see
  const AttnSpan from = attn_keys(p, any ? r_wave / p.group : 0, n), to = attn_keys(p, any ? (min(r_wave + 32, packed) - 1) / p.group : 0, n);
  const int k_begin = attn_keys(p, r0 / p.group, n).lo / TK * TK;
  const int k_end = attn_keys(p, (min(r0 + 32 * NW, packed) - 1) / p.group, n).hi + 1;
  const int tiles = (k_end - k_begin + TK - 1) / TK;
  // visible: key - lo <= span as unsigned; rows that do not exist see nothing
  const int lo = there ? mine.lo : 0x40000000;
  const unsigned span = there ? mine.hi - mine.lo : 0;

  const T* const k_base = static_cast<const T*>(p.k) + (int64_t)w.head * p.d;
  const T* const v_base = static_cast<const T*>(p.v) + (int64_t)w.head * p.d;
  const unsigned lds = attn_lds(smem);
  // rows that follow each other have their offsets worked out once; the end of a sequence takes the general way
  const auto off = A::template offsets<TK, NT>(PLAIN ? p.k_stride : 0);
  auto request = [&](const T* base, int64_t stride, int tile, int rows, unsigned at) {
    const int k0 = k_begin + tile * TK;
    if (PLAIN && k0 + TK <= n) {
      A::template request_rows<TK, NT>(lds + at, base + (first + k0) * stride, off);
    } else {
      A::template request<TK, NT, LOADS>(lds + at, p.d, [=](int r) -> const T* {
        if constexpr (PLAIN) return k0 + r < n ? base + (first + k0 + r) * stride : nullptr;
        const int row = __shfl(rows, r);
        return row < 0 ? nullptr : base + row * stride;
      });
    }
  };
  int rows_k = 0, rows_v = 0;                          // rows of the next tile of keys, and of values
  auto look_up = [&](int tile) {
    if constexpr (!PLAIN) rows_k = attn_look_up(p, first, k_begin + tile * TK, n);
  };
  auto request_k = [&](int tile, unsigned at) { request(k_base, p.k_stride, tile, rows_k, at); };
  auto request_v = [&](int tile, unsigned at) { request(v_base, p.v_stride, tile, rows_v, at); };
  look_up(0);

  request_k(0, 0);
  rows_v = rows_k;
  request_v(0, 2 * TILE);
  v4i qf[A::KS];
  A::template read_row<LOADS>(static_cast<const T*>(p.q) + row * p.q_stride + (int64_t)head * p.d, p.d, h, there, qf);
  const float c = p.scale * kAttnLog2e;
  typename A::Along along = A::along(lane);
  typename A::Across across = A::across(lane);
  along.add(lds);
  across.add(lds);
  floatx16 acc[A::DB], s_even[KB], s_odd[KB];
#pragma unroll
  for (int db = 0; db < A::DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.0f;
  float m = -INFINITY, sum = 0.0f, shift = 0.0f;       // m is a maximum times c, as it was rounded

  auto scores = [&](floatx16 (&s)[KB], auto parity) {
    constexpr unsigned at = decltype(parity)::value * TILE;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[b][v] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < A::KS; ++ks) A::E::mma(s[b], A::read_along(along, at, b, ks), qf[ks]);
    }
  };
  auto hide = [&](floatx16 (&s)[KB], int tile) {       // what a row does not see
    const int k0 = k_begin + tile * TK;
    if (k0 >= to.lo && k0 + TK - 1 <= from.hi && r_wave + 32 <= packed) return;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[b][v] = (unsigned)(k0 + 4 * h - lo + (32 * b + 8 * (v >> 2) + (v & 3))) <= span ? s[b][v] : -INFINITY;
  };
  auto weights = [&](floatx16 (&s)[KB], v4i (&pf)[KB][A::SS]) {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[b][v] = attn_exp2(__builtin_fmaf(s[b][v], c, -shift));
      A::pack(s[b], pf[b]);
    }
  };
  auto add_up = [&](const floatx16 (&s)[KB], auto from, auto to) {      // blocks from .. to, by themselves first: one weight after the other is lost beside a large sum
    constexpr int B0 = decltype(from)::value, B1 = decltype(to)::value;
    if constexpr (B0 == B1) return;
    float part[4] = {s[B0 % KB][0], s[B0 % KB][1], s[B0 % KB][2], s[B0 % KB][3]};
#pragma unroll
    for (int b = B0; b < B1; ++b)
#pragma unroll
      for (int v = b == B0 ? 4 : 0; v < 16; ++v) part[v & 3] += s[b][v];
    sum += (part[0] + part[1]) + (part[2] + part[3]);
  };
  auto values = [&](const v4i (&pf)[KB][A::SS], auto parity) {
    constexpr unsigned at = (2 + decltype(parity)::value) * TILE;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int ss = 0; ss < A::SS; ++ss)
#pragma unroll
        for (int db = 0; db < A::DB; ++db) A::E::mma(acc[db], A::read_across(across, at, b, ss, db), pf[b][ss]);
  };
  auto maximum = [&](const floatx16 (&s)[KB]) {
    float part[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) part[v & 3] = fmaxf(part[v & 3], s[b][v]);
    return fmaxf(attn_max_halves(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]))) * c, m);
  };
  auto rescale = [&](float most) {
    // (a maximum that grew by less than 2^8 stays, as is published of such kernels: weights of up to 256 are as good as those of up to 1)
    if (attn_any(most > m + 8.0f)) {
      const float next = attn_shift<DT == kF16>(most), less = m == -INFINITY ? 0.0f : attn_exp2(shift - next);
      shift = next;
      sum *= less;
#pragma unroll
      for (int db = 0; db < A::DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[db][v] *= less;
      m = most;
    }
  };
  // blocks whose weights are added up beside the scores, the others beside the values: as the vector unit has room and registers last
  constexpr int EARLY = VEC >= 2 && DP > 64 ? 0 : KB;
  // An order of the instructions between two of these points: LDS reads ahead of the products that take them, vector work between.
  auto ahead = [&](auto products, auto reads, auto first, auto vector, auto trans) {
    if constexpr (DT != kF32) {
      constexpr int N = decltype(products)::value, R = decltype(reads)::value, F = decltype(first)::value;
      __builtin_amdgcn_sched_group_barrier(0x100, F, 0);
      attn_for<0, N>([&](auto i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        constexpr int left = R - F - decltype(i)::value * (R / N);
        if constexpr (left > 0) __builtin_amdgcn_sched_group_barrier(0x100, left < R / N ? left : R / N, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, decltype(vector)::value, 0);
        if constexpr (decltype(trans)::value > 0) __builtin_amdgcn_sched_group_barrier(0x400, decltype(trans)::value, 0);
      });
    }
  };
  // Scores of tile `tile` (of parity P) into `now`, while `before` becomes weights of the values of the tile before it.
  auto step = [&](floatx16 (&before)[KB], floatx16 (&now)[KB], int tile, auto parity) {
    constexpr int P = decltype(parity)::value;
    attn_meet<0>();                                    // keys of this tile and values of the one before are here, and everybody is this far
    if (tile + 1 < tiles) request_k(tile + 1, (1 - P) * TILE);
    request_v(tile, (2 + P) * TILE);
    rows_v = rows_k;
    look_up(tile + 2);
    v4i pf[KB][A::SS];
    __builtin_amdgcn_sched_barrier(0);
    scores(now, parity);
    weights(before, pf);
    add_up(before, attn_c<0>, attn_c<EARLY>);
    asm volatile("" : "+v"(sum));                      // (formed here, not where they are taken)
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int ss = 0; ss < A::SS; ++ss) asm volatile("" : "+v"(pf[b][ss]));
    ahead(attn_c<KB * A::KS>, attn_c<KB * A::KS>, attn_c<3>, attn_c<EARLY ? 40 / A::KS : 24 / A::KS>, attn_c<16 / A::KS>);
    __builtin_amdgcn_sched_barrier(0);
    hide(now, tile);
    __builtin_amdgcn_sched_barrier(0);
    values(pf, attn_c<1 - P>);
    add_up(before, attn_c<EARLY>, attn_c<KB>);
    const float most = maximum(now);
    ahead(attn_c<KB * A::SS * A::DB>, attn_c<2 * KB * A::SS * A::DB>, attn_c<6>, attn_c<EARLY ? 8 / A::DB : 16 / A::DB>, attn_c<0>);
    __builtin_amdgcn_sched_barrier(0);
    rescale(most);
  };
  auto finish = [&](floatx16 (&before)[KB], auto parity) {
    v4i pf[KB][A::SS];
    attn_meet<0>();
    weights(before, pf);
    values(pf, parity);
    add_up(before, attn_c<0>, attn_c<KB>);
  };
  look_up(1);
  attn_meet<0>();
  if (tiles > 1) request_k(1, TILE);
  rows_v = rows_k;
  look_up(2);
  scores(s_even, attn_c<0>);
  hide(s_even, 0);
  rescale(maximum(s_even));
  int tile = 1;
  for (; tile + 1 < tiles; tile += 2) {
    step(s_even, s_odd, tile, attn_c<1>);
    step(s_odd, s_even, tile + 1, attn_c<0>);
  }
  if (tile < tiles) {
    step(s_even, s_odd, tile, attn_c<1>);
    finish(s_odd, attn_c<1>);
  } else {
    finish(s_even, attn_c<0>);
  }
  sum = attn_add_halves(sum);
  // (the row's place is worked out again: registers are short in between)
  int again = threadIdx.x;
  asm volatile("" : "+v"(again));
  const int r_out = r_wave + (again & 31);
  if (r_out >= packed) return;
  const int i_out = r_out / p.group, head_out = w.head * p.group + (r_out - i_out * p.group);
  const int64_t row_out = p.map ? p.map[first + i_out] : first + i_out;
  sum = attn_total(m, sum);
  const float per = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;      // (NaN stays)
  if (p.lse && again % 64 < 32) p.lse[(int64_t)(first + i_out) * p.heads + head_out] = sum == 0.0f ? -INFINITY : attn_lse<DT>(shift, sum);
  T* const out = static_cast<T*>(p.out) + (row_out * p.heads + head_out) * p.d;
#pragma unroll
  for (int db = 0; db < A::DB; ++db) A::template write_16<LOADS>(out, 32 * db + 16 * ((again >> 5) & 1), p.d, acc[db], per);
}

// ---- gradients ---------------------------------------------------------------------------------------------------------------------------
// Both kernels go in steps of 32 rows of what passes by.  While the matrix unit forms the scores and the products with the result's gradient of
// the next step, the vector unit makes probabilities and gradients of scores of this one; then those are multiplied.  Tiles (one or two
// steps) lie in three places in LDS: one whose second half is still multiplied, the next, and one on its way.

// Orders of the instructions of a step.  Products of scores: N, a read of LDS each (FIRST others before, MORE behind, of the products that
// follow), and the vector unit's work beside them.  Products across: N, two reads each, of which FIRST have been there before.
template <int N, int FIRST, int MORE, int VECTOR> __device__ __forceinline__ void attn_order_scores() {
  __builtin_amdgcn_sched_group_barrier(0x100, FIRST + 3, 0);
  attn_for<0, N>([&](auto at) {
    constexpr int i = decltype(at)::value;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, i + 3 < N ? 1 : (MORE + 2) / 3, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, VECTOR, 0);
    __builtin_amdgcn_sched_group_barrier(0x400, 16 / N, 0);
  });
}
template <int N, int FIRST> __device__ __forceinline__ void attn_order_across() {
  attn_for<0, N>([&](auto at) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (decltype(at)::value + FIRST < N) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
  });
}
template <int N> __device__ __forceinline__ void attn_keep(v4i (&f)[N]) {      // what has been formed by here stays formed here
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i]));
}

// Gradient of the queries: a wavefront has 32 packed rows, one a lane and half; keys and values pass by.
template <int DT, int DP, int NW, int VEC>
__global__ __launch_bounds__(64 * NW, DT == kF32 || (DP > 64 && NW == 4) ? 1 : 2) void attn_rows_kernel(const AttnParams p) {
  using A = AttnTile<DT, DP>;
  using T = typename A::T;
  constexpr bool PLAIN = VEC == kAttnPlain;
  constexpr int LOADS = PLAIN ? 2 : VEC, NT = 64 * NW, HALVES = DT == kF32 ? 1 : 2, TK = 32 * HALVES;
  constexpr int TILE = TK * A::RB, STAGE = 2 * TILE;
  extern __shared__ __align__(16) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, l32 = lane & 31;

  if (attn_zeros_of_dropped<NW>(p)) return;
  const AttnWork w = attn_work(p);
  const int n = w.item.rows, first = w.item.first, packed = n * p.group;
  const int r0 = w.item.tile * 32 * NW, r_wave = r0 + wave * 32, r = r_wave + l32;
  const bool there = r < packed, any = r_wave < packed;
  const int i = there ? r / p.group : 0, head = w.head * p.group + (there ? r - i * p.group : 0);
  const int64_t row = p.map ? p.map[first + i] : first + i;
  const AttnSpan mine = attn_keys(p, i, n);
  // of the whole wavefront and workgroup: rows are in ascending order, and so are both ends of what they see
  const AttnSpan from = attn_keys(p, any ? r_wave / p.group : 0, n), to = attn_keys(p, any ? (min(r_wave + 32, packed) - 1) / p.group : 0, n);
  const int k_begin = attn_keys(p, r0 / p.group, n).lo / TK * TK;
  const int k_end = attn_keys(p, (min(r0 + 32 * NW, packed) - 1) / p.group, n).hi + 1;
  const int tiles = (k_end - k_begin + TK - 1) / TK;
  // visible: key - lo <= span as unsigned; rows that do not exist see nothing
  const int lo = there ? mine.lo : 0x40000000;
  const unsigned span = there ? mine.hi - mine.lo : 0;

  const T* const k_base = static_cast<const T*>(p.k) + (int64_t)w.head * p.d;
  const T* const v_base = static_cast<const T*>(p.v) + (int64_t)w.head * p.d;
  const unsigned lds = attn_lds(smem);
  const auto off = A::template offsets<TK, NT>(PLAIN ? p.k_stride : 0);
  int rows = PLAIN ? 0 : attn_look_up(p, first, k_begin, n);      // of the next tile
  auto request = [&](int tile, unsigned stage) {
    const int k0 = k_begin + tile * TK;
    if (PLAIN && k0 + TK <= n) {
      A::template request_rows<TK, NT>(lds + stage, k_base + (first + k0) * p.k_stride, off);
      A::template request_rows<TK, NT>(lds + stage + TILE, v_base + (first + k0) * p.k_stride, off);
    } else {
      auto place = [&](const T* base, int64_t stride) {
        return [=](int r) -> const T* {
          if constexpr (PLAIN) return k0 + r < n ? base + (first + k0 + r) * stride : nullptr;
          const int row = __shfl(rows, r);
          return row < 0 ? nullptr : base + row * stride;
        };
      };
      A::template request<TK, NT, LOADS>(lds + stage, p.d, place(k_base, p.k_stride));
      __builtin_amdgcn_sched_barrier(0);
      A::template request<TK, NT, LOADS>(lds + stage + TILE, p.d, place(v_base, p.v_stride));
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (!PLAIN) rows = attn_look_up(p, first, k0 + TK, n);
  };
  request(0, 0);

  v4i qf[A::KS], gf[A::KS];
  A::template read_row<LOADS>(static_cast<const T*>(p.q) + row * p.q_stride + (int64_t)head * p.d, p.d, h, there, qf);
  const float c = p.scale * kAttnLog2e;
  float lse2 = 0.0f, delta = 0.0f;
  {
    const int64_t at = (row * p.heads + head) * p.d;
    A::template read_row<LOADS>(static_cast<const T*>(p.d_o) + at, p.d, h, there, gf);
    v4i of[A::KS];
    A::template read_row<LOADS>(static_cast<const T*>(p.o) + at, p.d, h, there, of);
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) {
      T a[A::V], b[A::V];
      __builtin_memcpy(a, &gf[ks], 16);
      __builtin_memcpy(b, &of[ks], 16);
#pragma unroll
      for (int e = 0; e < A::V; ++e) delta += (float)a[e] * (float)b[e];
    }
    delta = attn_add_halves(delta);
    const int64_t stat = (int64_t)(first + i) * p.heads + head;
    lse2 = there ? attn_lse2(p.lse[stat]) : 0.0f;
    if (there && h == 0) p.stats[0][stat] = attn_lse2(p.lse[stat], kAttnKeysUp<DT>);      // (for the keys)
  }

  typename A::Along along = A::along(lane);
  typename A::Across across = A::across(lane);
  along.add(lds);
  across.add(lds);
  floatx16 acc[A::DB], s_even, g_even, s_odd, g_odd;
#pragma unroll
  for (int db = 0; db < A::DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.0f;
  // delta again, as sum_j p (do . v_j): what o as it is stored makes of it is off by that tensor's rounding, one error of all the row's
  // gradients of scores.  Here they have to be formed before the sum is there; the keys' gradients have it.
  float part[2] = {0.0f, 0.0f};

  // (the tile that scores are formed of is where `along` points, that of the products across where `across` does)
  auto products = [&](floatx16& s, floatx16& g, auto half) {
    constexpr int H = decltype(half)::value;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = g[v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(s, A::read_along(along, 0, H, ks), qf[ks]);
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(g, A::read_along(along, TILE, H, ks), gf[ks]);
  };
  auto hide = [&](floatx16& s, int k0) {               // what a row does not see
    if (k0 >= to.lo && k0 + 31 <= from.hi && r_wave + 32 <= packed) return;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = (unsigned)(k0 + 4 * h - lo + (8 * (v >> 2) + (v & 3))) <= span ? s[v] : -INFINITY;
  };
  auto form = [&](const floatx16& s, floatx16& g, v4i (&pf)[A::SS]) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float e = attn_exp2(__builtin_fmaf(s[v], c, -lse2));
      part[v & 1] = __builtin_fmaf(e, g[v], part[v & 1]);
      g[v] = e * (g[v] - delta);
    }
    A::pack(g, pf);
  };
  constexpr int EARLY = DT == kF32 || VEC < 2 ? 0 : 2; // operands across that are read before
  auto early = [&](v4i (&of)[EARLY + 1], auto half) {
#pragma unroll
    for (int db = 0; db < EARLY; ++db) of[db] = A::read_across(across, 0, decltype(half)::value, 0, db);
  };
  auto take = [&](const v4i (&pf)[A::SS], const v4i (&of)[EARLY + 1], auto half) {
#pragma unroll
    for (int ss = 0; ss < A::SS; ++ss)
#pragma unroll
      for (int db = 0; db < A::DB; ++db)
        A::E::mma(acc[db], ss == 0 && db < EARLY ? of[db] : A::read_across(across, 0, decltype(half)::value, ss, db), pf[ss]);
  };
  // a step of `half` of a tile, from key k0 on, with the next one's products beside it
  auto step = [&](floatx16& s, floatx16& g, floatx16& s_next, floatx16& g_next, int k0, auto half, auto half_next) {
    v4i pf[A::SS], of[EARLY + 1] = {};
    hide(s, k0);
    __builtin_amdgcn_sched_barrier(0);
    products(s_next, g_next, half_next);
    form(s, g, pf);
    early(of, half);
    if constexpr (DT != kF32) {
      attn_keep(pf);
      attn_keep(of);
      attn_order_scores<2 * A::KS, 0, 2 * EARLY, 80 / (2 * A::KS)>();
    }
    __builtin_amdgcn_sched_barrier(0);
    take(pf, of, half);
    if constexpr (DT != kF32) attn_order_across<A::SS * A::DB, EARLY>();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto last = [&](floatx16& s, floatx16& g, int k0, auto half) {
    v4i pf[A::SS], of[EARLY + 1] = {};
    hide(s, k0);
    form(s, g, pf);
    early(of, half);
    take(pf, of, half);
  };
  unsigned place = 0;                                  // of the tile that `along` points into
  auto turn = [&]() {                                  // on to the next tile
    const unsigned by = place == 2 * STAGE ? 0u - 2 * STAGE : STAGE;
    place += by;
    along.add(by);
    return by;
  };
  attn_meet<0>();
  if (tiles > 1) request(1, STAGE);
  products(s_even, g_even, attn_c<0>);
  int k0 = k_begin, tile = 0;
  if constexpr (HALVES == 2) {
    for (; tile + 1 < tiles; ++tile, k0 += TK) {
      step(s_even, g_even, s_odd, g_odd, k0, attn_c<0>, attn_c<1>);
      attn_meet<0>();                                  // the next tile is here, and nobody is in the one before this any more
      const unsigned by = turn();
      if (tile + 2 < tiles) request(tile + 2, place == 2 * STAGE ? 0 : place + STAGE);
      step(s_odd, g_odd, s_even, g_even, k0 + 32, attn_c<1>, attn_c<0>);
      across.add(by);
    }
    step(s_even, g_even, s_odd, g_odd, k0, attn_c<0>, attn_c<1>);
    last(s_odd, g_odd, k0 + 32, attn_c<1>);
  } else {
    auto one = [&](floatx16& s, floatx16& g, floatx16& s_next, floatx16& g_next) {
      attn_meet<0>();
      const unsigned by = turn();
      if (tile + 2 < tiles) request(tile + 2, place == 2 * STAGE ? 0 : place + STAGE);
      step(s, g, s_next, g_next, k0, attn_c<0>, attn_c<0>);
      across.add(by);
      ++tile;
      k0 += TK;
    };
    while (tile + 2 < tiles) {
      one(s_even, g_even, s_odd, g_odd);
      one(s_odd, g_odd, s_even, g_even);
    }
    if (tile + 1 < tiles) {
      one(s_even, g_even, s_odd, g_odd);
      last(s_odd, g_odd, k0, attn_c<0>);
    } else {
      last(s_even, g_even, k0, attn_c<0>);
    }
  }
  delta = attn_add_halves(part[0] + part[1]);
  // (the row's place is worked out again: registers are short in between)
  int again = threadIdx.x;
  asm volatile("" : "+v"(again));
  const int r_out = r_wave + (again & 31), h_out = (again >> 5) & 1;
  if (r_out >= packed) return;
  const int i_out = r_out / p.group, head_out = w.head * p.group + (r_out - i_out * p.group);
  if (h_out == 0) p.stats[1][(int64_t)(first + i_out) * p.heads + head_out] = delta * kAttnKeysUnit<DT>;
  T* const out = static_cast<T*>(p.dq) + (p.map ? p.map[first + i_out] : first + i_out) * p.dq_stride + (int64_t)head_out * p.d;
#pragma unroll
  for (int db = 0; db < A::DB; ++db) A::template write_16<LOADS>(out, 32 * db + 16 * h_out, p.d, acc[db], p.scale);
}

// Gradients of keys and values: a wavefront has 32 keys, one a lane and half; packed rows of queries and of the result's gradient pass by.
template <int DT, int DP, int VEC>
__global__ __launch_bounds__(64 * kAttnKeyWaves, DP > 64 || DT == kF32 ? 1 : 2) void attn_keys_kernel(const AttnParams p) {
  using A = AttnTile<DT, DP>;
  using T = typename A::T;
  constexpr bool PLAIN = VEC == kAttnPlain;
  constexpr int LOADS = PLAIN ? 2 : VEC, NW = kAttnKeyWaves, NT = 64 * NW, HALVES = DT == kF32 ? 1 : 2, TQ = 32 * HALVES;
  constexpr int TILE = TQ * A::RB, STATS = 2 * TQ * 4, STAGE = 2 * TILE + STATS;
  extern __shared__ __align__(16) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, l32 = lane & 31;

  const AttnWork w = attn_work(p);
  const int n = w.item.rows, first = w.item.first;
  const int j0 = w.item.tile * 32 * NW, j_wave = j0 + wave * 32, j = j_wave + l32;
  const bool there = j < n, any = j_wave < n;
  const int64_t row = there ? (p.map ? p.map[first + j] : first + j) : 0;
  const AttnSpan mine = attn_rows(p, there ? j : 0, n);
  const AttnSpan from = attn_rows(p, any ? j_wave : 0, n), to = attn_rows(p, any ? min(j_wave + 32, n) - 1 : 0, n);
  // packed rows
  const int group = p.group;
  const int r_begin = attn_rows(p, j0, n).lo * group / TQ * TQ, r_end = (attn_rows(p, min(j0 + 32 * NW, n) - 1, n).hi + 1) * group;
  const int tiles = (r_end - r_begin + TQ - 1) / TQ;
  const int lo = there ? mine.lo * group : 0x40000000;
  const unsigned span = there ? (mine.hi - mine.lo + 1) * group - 1 : 0;
  const int all_lo = to.lo * group, all_hi = (from.hi + 1) * group - 1;            // rows that see all of the wavefront's keys

  const T* const q_base = static_cast<const T*>(p.q) + (int64_t)w.head * group * p.d;
  const T* const g_base = static_cast<const T*>(p.d_o) + (int64_t)w.head * group * p.d;
  const unsigned lds = attn_lds(smem);
  const float c = p.scale * kAttnLog2e;
  const int64_t g_stride = (int64_t)p.heads * p.d;
  const auto q_off = A::template offsets<TQ, NT>(PLAIN ? p.q_stride : 0, PLAIN ? group : 1), g_off = A::template offsets<TQ, NT>(PLAIN ? g_stride : 0, PLAIN ? group : 1);
  int rows = PLAIN ? 0 : attn_look_up(p, first, r_begin / group, n);      // of the next tile
  auto request = [&](int tile, unsigned stage) {
    const int r0 = r_begin + tile * TQ, i0 = r0 / group, rem = r0 - i0 * group;
    if (PLAIN && r0 + TQ <= n * group) {
      A::template request_rows<TQ, NT>(lds + stage, q_base + (first + i0) * p.q_stride, q_off);
      A::template request_rows<TQ, NT>(lds + stage + TILE, g_base + (first + i0) * g_stride, g_off);
    } else {
      auto place = [&](const T* base, int64_t stride) {
        return [=, &p](int r) -> const T* {
          const int past = (int)((unsigned)(rem + r) * p.magic >> 20), row = PLAIN ? (i0 + past < n ? first + i0 + past : -1) : __shfl(rows, past);
          return row < 0 ? nullptr : base + row * stride + (rem + r - past * group) * p.d;
        };
      };
      A::template request<TQ, NT, LOADS>(lds + stage, p.d, place(q_base, p.q_stride));
      A::template request<TQ, NT, LOADS>(lds + stage + TILE, p.d, place(g_base, g_stride));
    }
    if constexpr (!PLAIN) rows = attn_look_up(p, first, (r0 + TQ) / group, n);
    // lse of the tile's rows (in exponents of 2), then delta: the first wavefront's transfers
    if (wave == 0) {
#pragma unroll
      for (int part = 0; part < 2 * TQ; part += 64) {
        const int x = part + lane, r = x % TQ, past = (int)((unsigned)(rem + r) * p.magic >> 20), i = i0 + past;
        const float* of = p.stats[x / TQ] + (int64_t)(first + i) * p.heads + w.head * group + (rem + r - past * group);
        attn_dma4(i < n ? (const void*)of : (const void*)&attn_zeros, lds + stage + 2 * TILE + part * 4);
      }
    }
  };
  request(0, 0);

  v4i kf[A::KS], vf[A::KS];
  A::template read_row<LOADS>(static_cast<const T*>(p.k) + row * p.k_stride + (int64_t)w.head * p.d, p.d, h, there, kf);
  A::template read_row<LOADS>(static_cast<const T*>(p.v) + row * p.v_stride + (int64_t)w.head * p.d, p.d, h, there, vf);
  typename A::Along along = A::along(lane);
  typename A::Across across = A::across(lane);
  along.add(lds);
  across.add(lds);
  unsigned at_stats = lds + 2 * TILE + 16 * h;
  floatx16 dk[A::DB], dv[A::DB], s_even, g_even, s_odd, g_odd;
#pragma unroll
  for (int db = 0; db < A::DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) dk[db][v] = dv[db][v] = 0.0f;

  typedef __attribute__((address_space(3))) const v4f lds_v4f;
  // (the tile that scores are formed of is where `along` points, that of the products across where `across` does)
  auto products = [&](floatx16& s, floatx16& g, auto half) {
    constexpr int H = decltype(half)::value;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = g[v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(s, A::read_along(along, 0, H, ks), kf[ks]);
    if constexpr (DT == kF32) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(g, A::read_along(along, TILE, H, ks), vf[ks]);
  };
  auto hide = [&](floatx16& s, int r0) {               // keys that a row does not see
    if (r0 >= all_lo && r0 + 31 <= all_hi && j_wave + 32 <= n) return;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = (unsigned)(r0 + 4 * h - lo + (8 * (v >> 2) + (v & 3))) <= span ? s[v] : -INFINITY;
  };
  struct Stats { v4f lse2[4], delta[4]; };             // of a step's rows
  auto stats_of = [&](auto half) {
    constexpr int H = decltype(half)::value;
    Stats of;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      of.lse2[a] = *(lds_v4f*)(uint64_t)(at_stats + (32 * H + 8 * a) * 4);
      of.delta[a] = *(lds_v4f*)(uint64_t)(at_stats + (TQ + 32 * H + 8 * a) * 4);
    }
    return of;
  };
  auto form = [&](floatx16& s, floatx16& g, const Stats& of, v4i (&pf)[A::SS], v4i (&df)[A::SS]) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s[v] = attn_exp2(__builtin_fmaf(s[v], c, -of.lse2[v >> 2][v & 3]));
      g[v] = attn_keys_ds<DT>(s[v], g[v], of.delta[v >> 2][v & 3]);
    }
    A::pack(s, pf);
    A::pack(g, df);
  };
  constexpr int EARLY = DT == kF32 ? 0 : 1;            // pairs of operands across that are read before
  auto early = [&](v4i (&of)[2 * EARLY + 1], auto half) {
#pragma unroll
    for (int db = 0; db < EARLY; ++db) {
      of[2 * db] = A::read_across(across, TILE, decltype(half)::value, 0, db);
      of[2 * db + 1] = A::read_across(across, 0, decltype(half)::value, 0, db);
    }
  };
  auto take = [&](const v4i (&pf)[A::SS], const v4i (&df)[A::SS], const v4i (&of)[2 * EARLY + 1], auto half) {
    constexpr int H = decltype(half)::value;
#pragma unroll
    for (int ss = 0; ss < A::SS; ++ss) {
      if constexpr (DT == kF32) __builtin_amdgcn_sched_barrier(0);      // (operands are read as they are taken: there is no room for all)
#pragma unroll
      for (int db = 0; db < A::DB; ++db) {
        const bool there = ss == 0 && db < EARLY;
        A::E::mma(dv[db], there ? of[2 * db] : A::read_across(across, TILE, H, ss, db), pf[ss]);
        A::E::mma(dk[db], there ? of[2 * db + 1] : A::read_across(across, 0, H, ss, db), df[ss]);
      }
    }
  };
  auto step = [&](floatx16& s, floatx16& g, floatx16& s_next, floatx16& g_next, int r0, auto half, auto half_next) {
    v4i pf[A::SS], df[A::SS], of[2 * EARLY + 1] = {};
    const Stats of_rows = stats_of(half);
    hide(s, r0);
    __builtin_amdgcn_sched_barrier(0);
    products(s_next, g_next, half_next);
    form(s, g, of_rows, pf, df);
    early(of, half);
    if constexpr (DT != kF32) {
      attn_keep(pf);
      attn_keep(df);
      attn_keep(of);
      attn_order_scores<2 * A::KS, 0, 4 * EARLY, 80 / (2 * A::KS)>();
    }
    __builtin_amdgcn_sched_barrier(0);
    take(pf, df, of, half);
    if constexpr (DT != kF32) attn_order_across<2 * A::SS * A::DB, 2 * EARLY>();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto last = [&](floatx16& s, floatx16& g, int r0, auto half) {
    v4i pf[A::SS], df[A::SS], of[2 * EARLY + 1] = {};
    hide(s, r0);
    form(s, g, stats_of(half), pf, df);
    early(of, half);
    take(pf, df, of, half);
  };
  unsigned place = 0;                                  // of the tile that `along` points into
  auto turn = [&]() {                                  // on to the next tile
    const unsigned by = place == 2 * STAGE ? 0u - 2 * STAGE : STAGE;
    place += by;
    along.add(by);
    return by;
  };
  int r0 = r_begin, tile = 0;
  if constexpr (HALVES == 2) {
    attn_meet<0>();
    if (tiles > 1) request(1, STAGE);
    products(s_even, g_even, attn_c<0>);
    for (; tile + 1 < tiles; ++tile, r0 += TQ) {
      step(s_even, g_even, s_odd, g_odd, r0, attn_c<0>, attn_c<1>);
      attn_meet<0>();                                  // the next tile is here, and nobody is in the one before this any more
      const unsigned by = turn();
      if (tile + 2 < tiles) request(tile + 2, place == 2 * STAGE ? 0 : place + STAGE);
      step(s_odd, g_odd, s_even, g_even, r0 + 32, attn_c<1>, attn_c<0>);
      across.add(by);
      at_stats += by;
    }
    step(s_even, g_even, s_odd, g_odd, r0, attn_c<0>, attn_c<1>);
    last(s_odd, g_odd, r0 + 32, attn_c<1>);
  } else {
    // floats: the products take all of the time, and registers two sets of results do not have
    for (; tile < tiles; ++tile, r0 += TQ) {
      attn_meet<0>();
      if (tile + 1 < tiles) request(tile + 1, place == 2 * STAGE ? 0 : place + STAGE);
      products(s_even, g_even, attn_c<0>);
      __builtin_amdgcn_sched_barrier(0);
      last(s_even, g_even, r0, attn_c<0>);
      const unsigned by = turn();
      across.add(by);
      at_stats += by;
    }
  }
  if (!there) return;
  T* const out_k = static_cast<T*>(p.dk) + row * p.dk_stride + (int64_t)w.head * p.d;
  T* const out_v = static_cast<T*>(p.dv) + row * p.dv_stride + (int64_t)w.head * p.d;
#pragma unroll
  for (int db = 0; db < A::DB; ++db) {
    A::template write_16<LOADS>(out_k, 32 * db + 16 * h, p.d, dk[db], p.scale);
    A::template write_16<LOADS>(out_v, 32 * db + 16 * h, p.d, dv[db], kAttnKeysUnit<DT>);
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------------------------------
template <class Kernel> static hipError_t attn_start(Kernel kernel, int threads, int lds, const AttnParams& p, hipStream_t s) {
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3((unsigned)((int64_t)p.n_items * p.kv_heads + p.zeros.blocks)), dim3(threads), lds, s>>>(p);
  return hipGetLastError();
}

template <int DT, int DP, int VEC> static hipError_t attn_start_width(int what, const AttnParams& p, AttnTiles t, hipStream_t s) {
  using A = AttnTile<DT, DP>;
  constexpr int rows = DT == kF32 ? 32 : 64;                 // of a tile that passes by
  if (what == kAttnBackwardKV) return attn_start(attn_keys_kernel<DT, DP, VEC>, 64 * kAttnKeyWaves, 3 * (2 * rows * A::RB + 2 * rows * 4), p, s);
  auto start = [&](auto waves) {
    constexpr int NW = decltype(waves)::value;
    // (4-byte transfers of eight wavefronts need more registers than there are: entries, where strides alone ask for them)
    constexpr int LOADS = VEC == 1 && NW == 8 ? 0 : VEC;
    if (what == kAttnBackwardQ) return attn_start(attn_rows_kernel<DT, DP, NW, LOADS>, 64 * NW, 6 * rows * A::RB, p, s);
    if constexpr (DT != kF32 && DP == 64 && NW == 4) {
      if (t.keys == 32) return attn_start(attn_forward_kernel<DT, DP, NW, 32, VEC>, 64 * NW, 4 * 32 * A::RB, p, s);
    }
    return attn_start(attn_forward_kernel<DT, DP, NW, rows, VEC>, 64 * NW, 4 * rows * A::RB, p, s);
  };
  if constexpr (DT != kF32) {
    if (t.waves == 8) return start(attn_c<8>);
  }
  return start(attn_c<4>);
}

template <int DT> hipError_t attn_launch(int what, const AttnParams& p, AttnTiles t, int vec, hipStream_t s) {
  auto start = [&](auto level) {
    constexpr int VEC = decltype(level)::value;
    return p.d <= 64 ? attn_start_width<DT, 64, VEC>(what, p, t, s) : attn_start_width<DT, 128, VEC>(what, p, t, s);
  };
  if (vec == 2) {
    const int64_t most = AttnTile<DT, 64>::kMostStride;
    const bool plain = !p.map && (p.d == 64 || p.d == 128) &&
                       (what == kAttnBackwardKV ? (DT == kF32 ? 32 : 64) % p.group == 0 && p.q_stride <= most && (int64_t)p.heads * p.d <= most
                                                : p.k_stride == p.v_stride && p.k_stride <= most);
    return plain ? start(attn_c<kAttnPlain>) : start(attn_c<2>);
  }
  if constexpr (DT != kF32) {
    if (vec == 0) return start(attn_c<0>);
  }
  return start(attn_c<1>);
}

}  // namespace sc
