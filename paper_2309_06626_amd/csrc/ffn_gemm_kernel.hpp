// Products of the gated feed-forward block: C[i][j] = sum_k P[i][k] Q[j][k] in tiles of BM x BN on the matrix cores, with the
// block's activation, gating and row maps in the loads and the epilogue.
//
// Bound by the matrix cores, and under full load by power: 8 192 x 5 632 -> 2 048 in bf16 145 to 157 us (1 200 to 1 300 TFLOP/s, matrix
// pipes busy 83 % of cycles at 1.6 to 1.9 GHz; the library's product 131, 89 %), gated 8 192 x 2 048 -> 2 x 5 632 with what backward needs
// 358 to 383, hidden gradient 278 to 300, input gradient 280 to 300, weight gradients 372 to 440 (two) and 190 to 223.  Tiles of 256 x 256
// need the fewest bytes an operation from LDS and L2; the smaller ones fill the compute units where there are few tiles.
// Floats: 8 192 x 512 -> 4 096 187 TFLOP/s, 132 on the float matrix instruction.
#pragma once
#include "ffn_act.hpp"
#include "ffn_params.hpp"
#include "ffn_saved.hpp"
#include "mma_common.hpp"

namespace sc {

// ---- LDS tiles ------------------------------------------------------------------------------------------------------------------
// 128 bytes of k a row of an operand along k (64 entries of 16 bits, 32 floats); an operand across k has as many rows of k.
// A 16-byte group lies at its index XOR a key of its row, so that the lanes that read together touch every bank once.
template <int EB> struct FfnTile {
  static constexpr int BK = 128 / EB, V = 16 / EB, STEPS = 4, KSTEP = BK / STEPS;
  // (row >> 1) & 7: a 16-byte read serves lanes 0-3, 12-15, 20-23 and 24-27 of a wavefront together (and their like); they then touch
  // every bank once, for consecutive rows (P) as for those of ffn_q_order (Q): 4.0 cycles a read, 6.7 with row & 7, 24 without a key
  static __device__ __forceinline__ int key_along(int row) { return (row >> 1) & 7; }
  // GROUPS 16-byte groups a row
  template <int GROUPS> static __device__ __forceinline__ int key_across(int k) {
    if constexpr (EB == 2) return GROUPS >= 16 ? ((k & 3) << 2) | ((k >> 1) & 1) : ((k >> 1) & 1) << 2;
    return ((k >> 2) & 1) << 3;
  }
};

// A 32 x 32 block of results leaves 16 registers a lane: with the Q rows of a block read in this order, they are 16 consecutive
// columns of the lane's row.
__device__ __forceinline__ int ffn_q_order(int r) { return ((r >> 2) & 1) * 16 + (r >> 3) * 4 + (r & 3); }

constexpr int kFfnList = 4096;      // rows of the contraction whose list entries lie in LDS
static __device__ __align__(16) v4i ffn_zeros = {0, 0, 0, 0};      // what is read beyond an operand's end

// 16 bytes a lane from memory into LDS at base + 16 lane.  Written out, because the compiler would let every later LDS read wait
// for all transfers in flight; their arrival is waited for at the barriers below.  The base goes through m0, which the compiler writes (it
// has to know what m0 holds), a wait state before the transfer.
__device__ __forceinline__ void ffn_dma16(const void* src, unsigned lds_base) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(lds_base), "v"(src));
}

// Eight floats of a row in bf16 parts.  Cutting off keeps 8 bits a part, and what is left over is exact: hi + mid + lo is the float (of
// numbers from 2^-102 on: what lies below 2^-126 is lost; infinities become infinity - infinity).
struct FfnParts { v4i part[3]; };
__device__ __forceinline__ FfnParts ffn_parts(v4i first, v4i second) {
  unsigned bits[3][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float left = __builtin_bit_cast(float, e < 4 ? first[e] : second[e - 4]);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      bits[k][e] = __builtin_bit_cast(unsigned, left);
      if (k < 2) left -= __builtin_bit_cast(float, bits[k][e] & 0xffff0000u);
    }
  }
  FfnParts p;
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) p.part[k][i] = (int)__builtin_amdgcn_perm(bits[k][2 * i + 1], bits[k][2 * i], 0x07060302u);
  return p;
}
template <class E> __device__ __forceinline__ void ffn_mma(floatx16& acc, const v4i& q, const v4i& p) { E::mma(acc, q, p); }
template <class E> __device__ __forceinline__ void ffn_mma(floatx16& acc, const FfnParts& q, const FfnParts& p) {
  using B = Elem<kBF16>;      // the smallest products first
  B::mma(acc, q.part[2], p.part[0]);
  B::mma(acc, q.part[0], p.part[2]);
  B::mma(acc, q.part[1], p.part[1]);
  B::mma(acc, q.part[1], p.part[0]);
  B::mma(acc, q.part[0], p.part[1]);
  B::mma(acc, q.part[0], p.part[0]);
}

template <int I, int N, class Fn> __device__ __forceinline__ void ffn_for(Fn&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    ffn_for<I + 1, N>(f);
  }
}

// As store_block_pairs, of 16 columns that lie as they are stored: two lanes trade pieces, so that they write 32 bytes of one row each time.
template <typename T>
__device__ __forceinline__ void ffn_store_pairs(const v4i (&pk)[sizeof(T)], int row, int c0, T* y, int c_out) {
  constexpr int GC = 16 / (int)sizeof(T), PIECES = 16 / GC;
  const bool odd = threadIdx.x & 1;
  auto other = [](int v) { return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, false); };   // quad_perm [1, 0, 3, 2]
  const int theirs = other(row);
  const int row0 = odd ? theirs : row, row1 = odd ? row : theirs;
  T* const y0 = y + ((int64_t)row0 * c_out + c0 + (odd ? GC : 0));
  T* const y1 = y + ((int64_t)row1 * c_out + c0 + (odd ? GC : 0));
#pragma unroll
  for (int q = 0; q < PIECES; q += 2) {
    v4i first, second;       // the pieces of the even and of the odd lane's row
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int got = other(odd ? pk[q][i] : pk[q + 1][i]);
      first[i] = odd ? got : pk[q][i];
      second[i] = odd ? pk[q + 1][i] : got;
    }
    const bool inside = c0 + q * GC + (odd ? GC : 0) < c_out;
    if (inside && row0 >= 0) sc_store16(reinterpret_cast<v4i*>(y0 + q * GC), first);
    if (inside && row1 >= 0) sc_store16(reinterpret_cast<v4i*>(y1 + q * GC), second);
  }
}

template <int DT, bool P_ALONG, bool Q_ALONG, int WHAT, int BM, int BN, int WAVES_M, int WAVES_N, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N, 2) void ffn_gemm_kernel(const FfnGemm p) {
  using E = Elem<DT>;
  using T = typename E::T;
  constexpr int EB = sizeof(T);
  using L = FfnTile<EB>;
  constexpr int V = L::V, BK = L::BK;
  constexpr int W = WAVES_M * WAVES_N, NT = 64 * W;
  // a tile is two halves of P's rows by two halves of Q's; a wavefront has MB x NB blocks of 32 x 32 in each quadrant
  constexpr int PM = BM / 2, PN = BN / 2;
  constexpr int MB = PM / WAVES_M / 32, NB = PN / WAVES_N / 32;
  constexpr int JP = PM * 8 / NT, JQ = PN * 8 / NT;            // transfers of 16 bytes a lane and half tile
  constexpr int P_PIECE = PM * 128, Q_PIECE = PN * 128, STAGE = 2 * (P_PIECE + Q_PIECE);
  // half h of stage s in LDS, the halves of an operand within 64 KB of each other: one address a lane, the rest is in the instructions
  auto at_p = [](int h, int s) constexpr { return (2 * h + s) * P_PIECE; };
  auto at_q = [](int h, int s) constexpr { return 4 * P_PIECE + (2 * h + s) * Q_PIECE; };
  constexpr bool GATED = WHAT == kFfnUp;                       // the halves of Q: gate and up weights of the same columns
  constexpr int COLS = GATED ? PN : BN;                        // result columns of a tile
  static_assert(2 * JP + 3 * JQ <= 63, "the counts of transfers below");
  extern __shared__ __align__(16) unsigned char smem[];

  constexpr std::integral_constant<int, 0> c0{};
  constexpr std::integral_constant<int, 1> c1{};
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave / WAVES_N, wn = wave % WAVES_N;
  const int l32 = lane & 31, h = lane >> 5;

  // consecutive workgroups go round the eight dies: renumbered so that a die has neighbouring tiles, `group` tiles high
  const int tiles = p.m_tiles * p.n_tiles, total = tiles * p.batch * p.splits;
  const int per_xcd = (total + 7) >> 3;
  int at = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_xcd || at >= total) return;
  const int part = at / tiles;
  at -= part * tiles;
  const int z = part / p.splits, split = part - z * p.splits;
  const int band = at / (p.group * p.n_tiles), in_band = at - band * p.group * p.n_tiles;
  const int high = min(p.group, p.m_tiles - band * p.group);
  const int m0 = (band * p.group + in_band % high) * BM, n0 = (in_band / high) * COLS;

  // K tiles of this workgroup: every segment is a whole number of tiles, the last one padded with zeros
  const int n_last = p.n - 1;
  const bool q_listed = p.q_rows != nullptr;
  const int seg_tiles = (p.k + BK - 1) / BK, all_tiles = seg_tiles * p.segments;
  const int kt_lo = (int)((int64_t)all_tiles * split / p.splits), kt_hi = (int)((int64_t)all_tiles * (split + 1) / p.splits);

  // ---- loads ----
  // 16-byte group s of a half of an operand's tile: along k, row s / PPR, across k, row s / PPR of k
  constexpr int P_PPR = (P_ALONG ? 128 : PM * EB) / 16, Q_PPR = (Q_ALONG ? 128 : PN * EB) / 16;
  const int p_row = t / P_PPR, q_row = t / Q_PPR;              // of transfer 0
  constexpr int P_NEXT = NT / P_PPR, Q_NEXT = NT / Q_PPR;      // rows from transfer to transfer
  // first entry, within the row, of the group that belongs at place u of row r of the tile
  auto entry = [](auto along, auto ppr, int u, int r) -> int {
    const int key = decltype(along)::value ? L::key_along(r) : L::template key_across<decltype(ppr)::value>(r);
    return (u ^ key) * V;
  };
  // held in scalar registers: a load of a kernel argument between the products would have to wait for the operands on their way
  const T *p0 = static_cast<const T*>(p.p[P_ALONG ? 0 : z]), *p1 = static_cast<const T*>(p.p[p.segments > 1]);
  const T *q0 = static_cast<const T*>(p.q[0]), *q1 = static_cast<const T*>(p.q[p.segments > 1 || GATED]);
  int64_t ldp = p.ldp, ldq = p.ldq;
  int k_end = p.k;
  const void* zeros = &ffn_zeros;
  asm volatile("" : "+s"(p0), "+s"(p1), "+s"(q0), "+s"(q1), "+s"(ldp), "+s"(ldq), "+s"(k_end), "+s"(zeros));
  // along: k of the lane's group, and its rows from the start of the operand; rows beyond the end: results that are not stored.
  // across: result row / column of the group in either half (beyond the end: any that exists; a row is whole groups long)
  const int p_k0 = entry(std::bool_constant<P_ALONG>{}, std::integral_constant<int, P_PPR>{}, t % P_PPR, p_row);
  const int q_k0 = entry(std::bool_constant<Q_ALONG>{}, std::integral_constant<int, Q_PPR>{}, t % Q_PPR, q_row);
  int p_at[2], q_at[2];
  int64_t p_off[2][P_ALONG ? JP : 1], q_off[2][Q_ALONG ? JQ : 1];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    p_at[h] = P_ALONG ? p_k0 : min(p_k0 + m0 + h * PM, (int)ldp - V);
    q_at[h] = Q_ALONG ? q_k0 : min(q_k0 + n0 + h * PN, (int)ldq - V);
    if constexpr (P_ALONG) {
#pragma unroll
      for (int j = 0; j < JP; ++j) {
        const int i = min(m0 + h * PM + p_row + j * P_NEXT, p.m - 1);
        p_off[h][j] = (p.p_rows ? (int64_t)p.p_rows[i] : i) * ldp + p_k0;
      }
    }
    if constexpr (Q_ALONG) {
#pragma unroll
      for (int j = 0; j < JQ; ++j) q_off[h][j] = min(n0 + (GATED ? 0 : h * PN) + q_row + j * Q_NEXT, n_last) * ldq + q_k0;
    }
  }
  // rows of the contraction that stand for others: a stretch of the list at a time in LDS (a look-up in memory would have to wait
  // for the transfers before it)
  constexpr bool LISTED = WHAT == kFfnWGrad;
  int32_t* const s_list = reinterpret_cast<int32_t*>(smem + 2 * STAGE);
  const int32_t* const list = LISTED ? (p.p_rows ? p.p_rows : p.q_rows) : nullptr;
  int list_base = 0;
  auto stretch = [&](int kt) {      // called by all
    list_base = kt * BK;
    for (int i = t; i < kFfnList && list_base + i < p.k; i += NT) s_list[i] = list[list_base + i];
  };

  const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char*)smem;
  int listed_row[JP > JQ ? JP : JQ];                           // of the tile asked for next; the halves share them
  auto look_up = [&](int kt) {
    if constexpr (LISTED) {
      if (!list) return;
      const int first = kt * BK + (q_listed ? q_row : p_row), next = q_listed ? Q_NEXT : P_NEXT;
#pragma unroll
      for (int j = 0; j < (JP > JQ ? JP : JQ); ++j)
        if ((j < JP && j < JQ) || j < (q_listed ? JQ : JP)) listed_row[j] = s_list[min(first + j * next, p.k - 1) - list_base];
    }
  };
  // What the transfers of a K tile share, worked out once: whole groups go straight into LDS, zeros beyond the end of k.
  struct Ask { const T *p, *q[2]; int k0; };
  auto prepare = [&](int kt) -> Ask {
    const int seg = kt >= seg_tiles, k0 = (kt - seg * seg_tiles) * BK;
    Ask a;
    a.k0 = k0;
    a.p = (seg ? p1 : p0) + (P_ALONG ? k0 : 0);
    a.q[0] = (!GATED && seg ? q1 : q0) + (Q_ALONG ? k0 : 0);
    a.q[1] = GATED ? q1 + k0 : a.q[0];
    return a;
  };
  const unsigned to = lds0 + wave * 1024;
  auto request_p = [&](const Ask& a, auto half, auto stage, auto which) {
    constexpr int h = decltype(half)::value, j = decltype(which)::value;
    const T* src;
    bool in;
    if constexpr (P_ALONG) {
      src = a.p + p_off[h][j];
      in = a.k0 + p_k0 < k_end;
    } else {
      const int k = a.k0 + p_row + j * P_NEXT;
      in = k < k_end;
      src = a.p + p_at[h] + (LISTED && list && !q_listed ? listed_row[j] : k) * ldp;
    }
    ffn_dma16(in ? (const void*)src : zeros, to + at_p(h, decltype(stage)::value) + j * NT * 16);
  };
  auto request_q = [&](const Ask& a, auto half, auto stage, auto which) {
    constexpr int h = decltype(half)::value, j = decltype(which)::value;
    const T* src;
    bool in;
    if constexpr (Q_ALONG) {
      src = a.q[h] + q_off[h][j];
      in = a.k0 + q_k0 < k_end;
    } else {
      const int k = a.k0 + q_row + j * Q_NEXT;
      in = k < k_end;
      src = a.q[h] + q_at[h] + (LISTED && q_listed ? listed_row[j] : k) * ldq;
    }
    ffn_dma16(in ? (const void*)src : zeros, to + at_q(h, decltype(stage)::value) + j * NT * 16);
  };
  // ---- operands of the matrix instructions, from LDS ----
  // 32 rows of a half of an operand and KSTEP entries of k.  A lane's addresses in half 0 of stage 0: along k one for every step (the
  // keys differ), across k one for every block of 32 rows; the rest is an offset in the instruction.
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) const v4i lds_v4i;
  typedef __attribute__((address_space(3))) const int lds_int;
  auto lane_address = [&](auto along, auto is_q, auto rows, int r0, int i) -> unsigned {
    constexpr int BR = decltype(rows)::value;
    constexpr bool Q = decltype(is_q)::value;
    if constexpr (decltype(along)::value) {
      const int r = r0 + (Q ? ffn_q_order(l32) : l32);
      return r * 128 + (((2 * i + h) ^ L::key_along(r)) << 4);
    } else if constexpr (EB == 2) {
      // within 16 lanes the transposing read gives lane j element t of source lane 4 t + j / 4, entry j % 4: source lane s
      // points at row s / 4 of k, columns of the four lanes from 4 (s % 4) on
      const int l16 = lane & 15, k = 8 * h + (l16 >> 2), r = 16 * ((lane >> 4) & 1) + 4 * (l16 & 3);
      const int c = r0 + 32 * i + (Q ? ffn_q_order(r) : r);
      return k * (BR * 2) + (((c >> 3) ^ L::template key_across<BR / V>(k)) << 4) + (c & 7) * 2;
    } else {
      const int k = 4 * h, c = r0 + 32 * i + (Q ? ffn_q_order(l32) : l32);
      return k * (BR * 4) + (((c >> 2) ^ L::template key_across<BR / V>(k)) << 4) + (c & 3) * 4;
    }
  };
  constexpr int P_ADDR = P_ALONG ? L::STEPS : MB, Q_ADDR = Q_ALONG ? L::STEPS : NB;
  unsigned p_addr[P_ADDR], q_addr[Q_ADDR];
#pragma unroll
  for (int i = 0; i < P_ADDR; ++i) {
    p_addr[i] = lds0 + lane_address(std::bool_constant<P_ALONG>{}, std::false_type{}, std::integral_constant<int, PM>{}, wm * MB * 32, i);
    asm volatile("" : "+v"(p_addr[i]));      // (kept as it is, so that what is added to it goes into the instructions)
  }
#pragma unroll
  for (int i = 0; i < Q_ADDR; ++i) {
    q_addr[i] = lds0 + at_q(0, 0) +
                lane_address(std::bool_constant<Q_ALONG>{}, std::true_type{}, std::integral_constant<int, PN>{}, wn * NB * 32, i);
    asm volatile("" : "+v"(q_addr[i]));
  }
  auto fragment = [&](auto along, auto rows, auto step, const auto& addr, int b, unsigned at) -> v4i {
    constexpr int BR = decltype(rows)::value, ks = decltype(step)::value;
    if constexpr (decltype(along)::value) {
      return *(lds_v4i*)(uint64_t)(addr[ks] + at + b * 32 * 128);
    } else if constexpr (EB == 2) {
      const unsigned a = addr[b] + at + ks * L::KSTEP * BR * 2;
      struct { s16x4 lo, hi; } both = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uint64_t)a),
                                       __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uint64_t)(a + 4 * BR * 2))};
      return __builtin_bit_cast(v4i, both);
    } else {
      v4i f;
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = *(lds_int*)(uint64_t)(addr[b] + at + (ks * L::KSTEP + e) * BR * 4);
      return f;
    }
  };

  floatx16 acc[2 * MB][2 * NB];
#pragma unroll
  for (int mi = 0; mi < 2 * MB; ++mi)
#pragma unroll
    for (int ni = 0; ni < 2 * NB; ++ni)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[mi][ni][v] = 0.0f;

  // operands: one half of P, both of Q, and the first half of Q of the next tile (the first and the third change places from tile to tile).
  // Floats are multiplied in three bf16 parts (x = hi + mid + lo, exactly: 3 x 8 bits) on the 16-bit instruction, six of the nine products; the
  // other three are below 2^-21 of the whole.  What is read waits as it is until it is taken apart, once for all its products.
  constexpr bool PARTS = DT == kF32;
  constexpr int GROUPS = PARTS ? 2 : L::STEPS;                 // groups of instructions over a tile's k
  using Operand = std::conditional_t<PARTS, FfnParts, v4i>;
  Operand pf[GROUPS][MB], qf[3][GROUPS][NB];
  v4i p_raw[PARTS ? L::STEPS : 1][MB], q_raw[PARTS ? L::STEPS : 1][NB];
  auto read_p = [&](auto stage, auto half, auto step) {
    constexpr int ks = decltype(step)::value;
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      const v4i f = fragment(std::bool_constant<P_ALONG>{}, std::integral_constant<int, PM>{}, step, p_addr, b,
                             at_p(decltype(half)::value, decltype(stage)::value));
      if constexpr (PARTS) p_raw[ks][b] = f;
      else pf[ks][b] = f;
    }
  };
  auto read_q = [&](auto stage, auto half, auto into, auto step) {
    constexpr int ks = decltype(step)::value;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const v4i f = fragment(std::bool_constant<Q_ALONG>{}, std::integral_constant<int, PN>{}, step, q_addr, b,
                             at_q(decltype(half)::value, decltype(stage)::value) - at_q(0, 0));
      if constexpr (PARTS) q_raw[ks][b] = f;
      else qf[decltype(into)::value][ks][b] = f;
    }
  };
  auto settle_p = [&]() {
    if constexpr (PARTS) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int b = 0; b < MB; ++b) pf[g][b] = ffn_parts(p_raw[2 * g][b], p_raw[2 * g + 1][b]);
    }
  };
  auto settle_q = [&](auto into) {
    if constexpr (PARTS) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int b = 0; b < NB; ++b) qf[decltype(into)::value][g][b] = ffn_parts(q_raw[2 * g][b], q_raw[2 * g + 1][b]);
    }
  };
  // the products of a quadrant with Q in registers `set`; then(ks) behind those of a step of k
  auto quadrant = [&](auto half_p, auto half_q, auto set, auto&& then) {
    constexpr int hp = decltype(half_p)::value, hq = decltype(half_q)::value;
    ffn_for<0, GROUPS>([&](auto group) {
      constexpr int g = decltype(group)::value;
#pragma unroll
      for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int c = 0; c < NB; ++c) ffn_mma<E>(acc[hp * MB + b][hq * NB + c], qf[decltype(set)::value][g][c], pf[g][b]);
      if constexpr (!PARTS) {
        __builtin_amdgcn_sched_barrier(0);
        then(group);
        __builtin_amdgcn_sched_barrier(0);
      } else if constexpr (g == 0) {                           // all reads behind the first half, which hides them
        __builtin_amdgcn_sched_barrier(0);
        ffn_for<0, L::STEPS>(then);
        __builtin_amdgcn_sched_barrier(0);
      }
    });
  };
  // all transfers but the youngest N have landed, for every wavefront, and all have come this far
  auto meet = [&](auto youngest) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(youngest)::value) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  constexpr int STRETCH = kFfnList / BK;                       // K tiles of a stretch of the list
  auto renew_list = [&](int kt) {                              // called by all, before anything of K tile kt is asked for
    if constexpr (LISTED) {
      if (list && (kt - kt_lo) % STRETCH == 0) {
        __syncthreads();
        stretch(kt);
        __syncthreads();
      }
    }
  };
  // Two K tiles in LDS, each in four halves.  The quadrants of a tile are multiplied in the order (P0, Q0), (P0, Q1), (P1, Q1),
  // (P1, Q0).  The operands of a quadrant are read from LDS one or two quadrants before, into registers that are free by then, and a
  // half's place in LDS is taken by the same half of the tile after next as soon as it is in everybody's registers: wavefronts meet
  // twice a tile, behind the first quadrant and behind the third, and a transfer has four to five quadrants (2 000 to 2 500 cycles for
  // tiles of 256) to arrive.  64 KB take 1.1 us to arrive in a compute unit that has nothing else to do.
  //   quadrant    1          2          3              4
  //   reads       Q1         P1         Q0, next tile  P0, next tile
  //   asks for    P1, next   Q0, after  P0, after      Q1, after next
  if (kt_lo < kt_hi) {
    const int last = kt_hi - 1;
    const std::integral_constant<int, 2> c2{};
    auto all_p = [&](const Ask& a, auto half, auto stage) { ffn_for<0, JP>([&](auto j) { request_p(a, half, stage, j); }); };
    auto all_q = [&](const Ask& a, auto half, auto stage) { ffn_for<0, JQ>([&](auto j) { request_q(a, half, stage, j); }); };
    renew_list(kt_lo);
    look_up(kt_lo);
    Ask a = prepare(kt_lo);
    all_q(a, c0, c0);
    all_p(a, c0, c0);
    all_q(a, c1, c0);
    all_p(a, c1, c0);
    look_up(min(kt_lo + 1, last));
    a = prepare(min(kt_lo + 1, last));
    all_q(a, c0, c1);
    all_p(a, c0, c1);
    all_q(a, c1, c1);
    meet(std::integral_constant<int, 2 * JP + 3 * JQ>{});
    ffn_for<0, L::STEPS>([&](auto ks) { read_q(c0, c0, c0, ks); read_p(c0, c0, ks); });
    settle_q(c0);
    settle_p();
    meet(std::integral_constant<int, 2 * JP + 2 * JQ>{});
    auto some = [&](auto ks, auto all, auto&& request) {       // transfers behind a step
      constexpr int n = decltype(all)::value, each = (n + L::STEPS - 1) / L::STEPS, lo = decltype(ks)::value * each;
      ffn_for<(lo < n ? lo : n), (lo + each < n ? lo + each : n)>(request);
    };
    constexpr std::integral_constant<int, JP> all_of_p{};
    constexpr std::integral_constant<int, JQ> all_of_q{};
    // tile kt in `stage`, its first half of Q in registers `now`, that of the next tile goes into `next`
    auto tile = [&](int kt, auto stage, auto other, auto now, auto next) {
      // a: the next tile's
      quadrant(c0, c0, now, [&](auto ks) {
        read_q(stage, c1, c1, ks);
        some(ks, all_of_p, [&](auto j) { request_p(a, c1, other, j); });
      });
      settle_q(c1);
      meet(std::integral_constant<int, 2 * JP + JQ>{});
      // (behind the last tiles the last one again, which nobody reads: the counts stay, and a branch would cost registers)
      const int ahead = min(kt + 2, last);
      if (kt + 2 <= last) renew_list(ahead);
      look_up(ahead);
      a = prepare(ahead);
      quadrant(c0, c1, c1, [&](auto ks) {
        read_p(stage, c1, ks);
        some(ks, all_of_q, [&](auto j) { request_q(a, c0, stage, j); });
      });
      settle_p();
      quadrant(c1, c1, c1, [&](auto ks) {
        read_q(other, c0, next, ks);
        some(ks, all_of_p, [&](auto j) { request_p(a, c0, stage, j); });
      });
      settle_q(next);
      meet(std::integral_constant<int, 2 * JP + JQ>{});
      quadrant(c1, c0, now, [&](auto ks) {
        read_p(other, c0, ks);
        some(ks, all_of_q, [&](auto j) { request_q(a, c1, stage, j); });
      });
      settle_p();
    };
    for (int kt = kt_lo;;) {
      tile(kt, c0, c1, c0, c2);
      if (++kt == kt_hi) break;
      tile(kt, c1, c0, c2, c0);
      if (++kt == kt_hi) break;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing may still be on its way into LDS when the workgroup ends
  }

  // ---- results: the lane has row l32 of a block, its columns 16 h .. 16 h + 15 ----
  const int n = p.n, m = p.m;
  // rows of any length, and rows for the next product, whole groups with zeros behind the last column; row < 0: none
  auto store = [&](T* c, int64_t ldc, int row, int col, const floatx16& v) {
    if constexpr (WHOLE) {
      store_block_pairs<DT, false>(v, row, false, col, c, nullptr, 0, (int)ldc);
    } else if (row >= 0) {
      T out[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) out[e] = E::from_float(v[e]);
      T* const dst = c + (int64_t)row * ldc + col;
      if (col + 16 <= n) {
        __builtin_memcpy(dst, out, sizeof(out));
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (col + e < n) dst[e] = out[e];
      }
    }
  };
  auto store_operand = [&](T* c, int64_t ldc, int row, int col, const floatx16& v) {
    floatx16 out = v;
    if constexpr (!WHOLE) {
#pragma unroll
      for (int e = 0; e < 16; ++e) out[e] = col + e < n ? v[e] : 0.0f;
    }
    store_block_pairs<DT, false>(out, row, false, col, c, nullptr, 0, (int)ldc);
  };
  // 16 columns of a row of `saved`, as they lie
  using Saved = FfnSaved<T>;
  using U = typename Saved::U;
  constexpr int PLANES = Saved::PLANES, PER = Saved::PER;
  struct Raw { v4i g[PLANES][16 / V]; };
  auto load16 = [&](int row, int col) {
    Raw raw;
    const int64_t at = (int64_t)row * n + col;
#pragma unroll
    for (int plane = 0; plane < PLANES; ++plane) {
      const U* s = static_cast<const U*>(p.saved) + (int64_t)plane * m * n + at;
#pragma unroll
      for (int g = 0; g < 16 / V; ++g) {
        const int have = row < 0 ? 0 : n - col - g * V;
        raw.g[plane][g] = v4i{0, 0, 0, 0};
        if (have >= V) {
          __builtin_memcpy(&raw.g[plane][g], s + g * V, 16);
        } else if (!WHOLE) {
          U e[V];
#pragma unroll
          for (int i = 0; i < V; ++i) e[i] = i < have ? s[g * V + i] : U(0);
          __builtin_memcpy(&raw.g[plane][g], e, 16);
        }
      }
    }
    return raw;
  };
  auto save16 = [&](int row, int col, const floatx16& gate, const floatx16& up) {
    unsigned words[PLANES][16 / PER];
#pragma unroll
    for (int w = 0; w < 16 / PER; ++w) {
      float g[PER], u[PER];
#pragma unroll
      for (int e = 0; e < PER; ++e) g[e] = gate[w * PER + e], u[e] = up[w * PER + e];
      unsigned one[PLANES];
      Saved::keep_word(g, u, one);
#pragma unroll
      for (int plane = 0; plane < PLANES; ++plane) words[plane][w] = one[plane];
    }
#pragma unroll
    for (int plane = 0; plane < PLANES; ++plane) {
      U* const to = static_cast<U*>(p.saved) + (int64_t)plane * m * n;
      if constexpr (WHOLE) {
        v4i pieces[sizeof(U)];
        __builtin_memcpy(pieces, words[plane], sizeof(pieces));
        ffn_store_pairs<U>(pieces, row, col, to, n);
      } else if (row >= 0) {
        U* const dst = to + (int64_t)row * n + col;
        if (col + 16 <= n) {
          __builtin_memcpy(dst, words[plane], sizeof(words[plane]));
        } else {
          U one[16];
          __builtin_memcpy(one, words[plane], sizeof(one));
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (col + e < n) dst[e] = one[e];
        }
      }
    }
  };
  if (p.splits > 1) {                                          // sums of this part: [batch, or gate and up][splits][m][pitch]
    const int pitch = (n + 3) & ~3;
#pragma unroll
    for (int mi = 0; mi < 2 * MB; ++mi) {
      const int row = m0 + mi / MB * PM + (wm * MB + mi % MB) * 32 + l32;
#pragma unroll
      for (int ni = 0; ni < 2 * NB; ++ni) {
        const int col = n0 + (GATED ? 0 : ni / NB * PN) + (wn * NB + ni % NB) * 32 + 16 * h;
        float* const dst = p.partial + (((int64_t)(GATED ? ni / NB : z) * p.splits + split) * m + row) * pitch + col;
        if (row < m && col + 16 <= pitch) {
          __builtin_memcpy(dst, &acc[mi][ni], 64);
        } else if (row < m) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (col + e < pitch) dst[e] = acc[mi][ni][e];
        }
      }
    }
    return;
  }
  int own_row = l32;
  auto row_of = [&](int mi) {
    const int i = m0 + mi / MB * PM + (wm * MB + mi % MB) * 32 + own_row;
    return i < m ? i : -1;
  };
  auto col_of = [&](int ni) { return n0 + ni / NB * PN + (wn * NB + ni % NB) * 32 + 16 * h; };
  if constexpr (WHAT == kFfnGateGrad) {
    // a block's rows of gate and up are asked for a block ahead
    Raw next = load16(row_of(0), col_of(0));
    ffn_for<0, 4 * MB * NB>([&](auto block) {
      constexpr int b = decltype(block)::value, mi = b / (2 * NB), ni = b % (2 * NB), after = b + 1 < 4 * MB * NB ? b + 1 : b;
      const Raw raw = next;
      asm volatile("" : "+v"(own_row));                        // (no addresses kept from block to block: registers)
      if constexpr (after != b) next = load16(row_of(after / (2 * NB)), col_of(after % (2 * NB)));
      unsigned words[PLANES][16 / PER];
      __builtin_memcpy(words, &raw, sizeof(words));
      T dg[16], du[16], hidden[16];                            // (converted at once: half as many registers)
      ffn_act_kind(p.activation, [&](auto kind) {
#pragma unroll
        for (int w = 0; w < 16 / PER; ++w) {
          unsigned one[PLANES];
#pragma unroll
          for (int plane = 0; plane < PLANES; ++plane) one[plane] = words[plane][w];
          float g[PER], u[PER];
          Saved::back_word(one, g, u);
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            const int e = w * PER + i;
            float a, da;
            ffn_act_of<decltype(kind)::value, T>(g[i], a, da);
            const bool in = WHOLE || col_of(ni) + e < n;
            dg[e] = E::from_float(in ? acc[mi][ni][e] * u[i] * da : 0.0f);
            du[e] = E::from_float(in ? acc[mi][ni][e] * a : 0.0f);
            hidden[e] = E::from_float(in ? a * u[i] : 0.0f);
          }
        }
      });
      auto leave = [&](void* c, const T (&v)[16]) {
        v4i pieces[sizeof(T)];
        __builtin_memcpy(pieces, v, sizeof(pieces));
        ffn_store_pairs<T>(pieces, row_of(mi), col_of(ni), static_cast<T*>(c), (int)p.ldc);
      };
      leave(p.c[0], dg);
      leave(p.c[1], du);
      if (p.hidden) leave(p.hidden, hidden);
    });
    return;
  }
#pragma unroll
  for (int mi = 0; mi < 2 * MB; ++mi) {
    const int row = row_of(mi);
    int out_row = row;
    if (row >= 0 && p.c_rows) out_row = p.c_rows[row];
#pragma unroll
    for (int ni = 0; ni < (GATED ? NB : 2 * NB); ++ni) {
      const int col = col_of(ni);
      if constexpr (WHAT == kFfnUp) {
        floatx16 hidden;
        ffn_act_kind(p.activation, [&](auto kind) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float a, da;
            ffn_act_of<decltype(kind)::value, T>(acc[mi][ni][e], a, da);
            hidden[e] = a * acc[mi][ni + NB][e];
          }
        });
        store_operand(static_cast<T*>(p.c[0]), p.ldc, row, col, hidden);
        if (p.saved) save16(row, col, acc[mi][ni], acc[mi][ni + NB]);
      } else {
        store(static_cast<T*>(p.c[z]), p.ldc, out_row, col, acc[mi][ni]);
      }
    }
  }
}

template <int DT, bool P_ALONG, bool Q_ALONG, int WHAT, int BM, int BN, int WAVES_M, int WAVES_N, bool WHOLE>
hipError_t ffn_launch_tile(FfnGemm g, hipStream_t s) {
  auto kernel = ffn_gemm_kernel<DT, P_ALONG, Q_ALONG, WHAT, BM, BN, WAVES_M, WAVES_N, WHOLE>;
  constexpr int cols = WHAT == kFfnUp ? BN / 2 : BN;
  g.m_tiles = (g.m + BM - 1) / BM;
  g.n_tiles = (g.n + cols - 1) / cols;
  g.group = 8;
  const bool listed = WHAT == kFfnWGrad && (g.p_rows || g.q_rows);
  const int lds = (BM + BN) * 256 + (listed ? kFfnList * 4 : 0);
  static std::atomic<uint64_t> told{0};
  const hipError_t e = ffn_allow_lds(reinterpret_cast<const void*>(kernel), (BM + BN) * 256 + kFfnList * 4, told);
  if (e != hipSuccess) return e;
  const int64_t total = (int64_t)g.m_tiles * g.n_tiles * g.batch * g.splits;
  kernel<<<dim3((unsigned)((total + 7) / 8 * 8)), dim3(64 * WAVES_M * WAVES_N), lds, s>>>(g);
  return hipGetLastError();
}

template <int DT, bool P_ALONG, bool Q_ALONG, int WHAT, bool WHOLE>
hipError_t ffn_launch_rows(const FfnGemm& g, int tile, hipStream_t s) {
  if constexpr (DT != kF32) {
    if (tile == 1) return ffn_launch_tile<DT, P_ALONG, Q_ALONG, WHAT, 256, 256, 2, 4, WHOLE>(g, s);
    if (tile == 2) return ffn_launch_tile<DT, P_ALONG, Q_ALONG, WHAT, 256, 128, 4, 2, WHOLE>(g, s);
  }
  return ffn_launch_tile<DT, P_ALONG, Q_ALONG, WHAT, 128, 128, 2, 2, WHOLE>(g, s);
}
template <int DT, bool P_ALONG, bool Q_ALONG, int WHAT>
hipError_t ffn_launch_what(const FfnGemm& g, int tile, bool whole, hipStream_t s) {
  return whole ? ffn_launch_rows<DT, P_ALONG, Q_ALONG, WHAT, true>(g, tile, s) : ffn_launch_rows<DT, P_ALONG, Q_ALONG, WHAT, false>(g, tile, s);
}

template <int DT> hipError_t ffn_launch_type(FfnProduct what, const FfnGemm& g, int tile, bool whole, hipStream_t s) {
  switch (what) {
    case kFfnUp: return ffn_launch_what<DT, true, true, kFfnUp>(g, tile, whole, s);
    case kFfnDown: return ffn_launch_what<DT, true, true, kFfnDown>(g, tile, whole, s);
    case kFfnGateGrad: return ffn_launch_what<DT, true, false, kFfnGateGrad>(g, tile, whole, s);
    case kFfnInGrad: return ffn_launch_what<DT, true, false, kFfnInGrad>(g, tile, whole, s);
    case kFfnWGrad: return ffn_launch_what<DT, false, false, kFfnWGrad>(g, tile, whole, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace sc
