// Tiles of rows in LDS and the operands of the matrix instructions that the attention kernels take from them.
//
// A tile is a number of rows of DP channels (a head's channels, padded with zeros), as they lie in memory.  Every tile is read in one or
// both of two ways, as the first operand of a 32 x 32 product:
//   along    rows of the tile are rows of the operand, the contraction goes over the channels  (S' = K Q', dP' = V dO')
//   across   channels are rows of the operand, the contraction goes over the tile's rows       (O' = V' P', dQ' = K' dS')
// The results of a product along leave a lane one column and the rows 8 a + 4 h + i of 32 (h: half of the wavefront).  Across, a
// lane's entries of the contraction are taken in that same order, so that results of the first product, rounded, are the second operand of
// the next one without leaving their lane.
#pragma once
#include "mma_common.hpp"

#include <math.h>
#include <type_traits>

namespace sc {

static __device__ __align__(16) v4i attn_zeros = {0, 0, 0, 0};      // what is read beyond a tile's end

// 16 (4) bytes a lane from memory into LDS at base + 16 (4) lane.  Written out, because the compiler would let every later LDS read wait
// for all transfers in flight; their arrival is waited for in attn_meet.  The base goes through m0, which the compiler writes (it has to
// know what m0 holds), a wait state before the transfer.
__device__ __forceinline__ void attn_dma16(const void* src, unsigned lds_base) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(lds_base), "v"(src) : "memory");
}
__device__ __forceinline__ void attn_dma4(const void* src, unsigned lds_base) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" ::"{m0}"(lds_base), "v"(src) : "memory");
}

// the same with a base that all lanes share and 32-bit offsets
__device__ __forceinline__ void attn_dma16(const void* base, unsigned offset, unsigned lds_base) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(lds_base), "v"(offset), "s"(base) : "memory");
}

// All of this wavefront's transfers but the youngest N have landed and its LDS accesses are done; then the same holds for all.
template <int N> __device__ __forceinline__ void attn_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ unsigned attn_lds(const void* p) {
  return (unsigned)(unsigned long long)(__attribute__((address_space(3))) const unsigned char*)p;
}

__device__ __forceinline__ float attn_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bool attn_any(bool b) { return __builtin_amdgcn_ballot_w64(b) != 0; }

// f16 holds numbers from 2^-24 on, those below 2^-14 with fewer digits, up to 65 504.  Weights that become operands of it are therefore formed 2^6 times
// as large: with the 2^8 by which a maximum that stays may be passed, the largest are 2^14, and those down to 2^-31 of the largest are not lost
// (100 000 of 2^-25 beside it are 0.3 % of their sum).
constexpr int kAttnUp = 6;
// What is taken off in the exponent of 2, m being what the largest score so far became there: 0 where nothing has been seen, so that every term is 0.
// (An m in whose rounding the 2^6 would be lost stays as it is.)
template <bool UP> __device__ __forceinline__ float attn_shift(float m) {
  return m == -INFINITY ? 0.0f : UP && fabsf(m) < 0x1p20f ? m - kAttnUp : m;
}

// A row's sum of weights, m being what its largest score became as an exponent.  No weight at all is a row that sees nothing but scores of -infinity;
// with any other m the score, as it was scaled, left a float's range, and the row is lost.
__device__ __forceinline__ float attn_total(float m, float sum) { return sum == 0.0f && m != -INFINITY ? __builtin_nanf("") : sum; }

// a value and that of the lane in the other half of the wavefront, in the same order in both
__device__ __forceinline__ void attn_halves(float v, float& low, float& high) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  low = __builtin_bit_cast(float, (unsigned)r[0]);
  high = __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float attn_max_halves(float v) { float a, b; attn_halves(v, a, b); return fmaxf(a, b); }
__device__ __forceinline__ float attn_add_halves(float v) { float a, b; attn_halves(v, a, b); return a + b; }

// A 32 x 32 block of results leaves 16 registers a lane: with the rows of the first operand read in this order, they are 16 consecutive
// ones, from 16 h on.
__device__ __forceinline__ int attn_order(int r) { return ((r >> 2) & 1) * 16 + (r >> 3) * 4 + (r & 3); }

template <int DT, int DP> struct AttnTile {
  using E = Elem<DT>;
  using T = typename E::T;
  static constexpr int EB = (int)sizeof(T), V = 16 / EB;
  static constexpr int RB = DP * EB;            // bytes of a row
  static constexpr int GROUPS = RB / 16;        // 16-byte groups of a row
  static constexpr int KS = RB / 32;            // products of a contraction over the channels
  static constexpr int SS = EB;                 // products of a contraction over 32 rows
  static constexpr int DB = DP / 32;            // blocks of 32 channels

  // A row's group g lies at g XOR key(row).  Along, the lanes that are served together (0-3, 12-15, 20-23, 24-27 and their like) read 16
  // rows, whose keys differ in all of the low bits; across, four rows are read together whose keys differ in bits 2 and 3 (64 bytes apart).
  static __device__ __forceinline__ int key(int row) {
    if constexpr (EB == 2) return GROUPS >= 16 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    else return (((row >> 2) & 1) << 3) | ((row & 3) << 1) | ((row >> 3) & 1);
  }

  // Lane addresses within a tile, worked out once; what depends on the block of 32 rows is an offset.
  template <int N> struct Lanes {
    unsigned at[N];
    // the tiles' base, kept as it is, so that what is added to it goes into the instructions
    __device__ __forceinline__ void add(unsigned base) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        at[i] += base;
        asm volatile("" : "+v"(at[i]));
      }
    }
  };
  typedef Lanes<KS> Along;
  typedef Lanes<EB == 2 ? 2 * DB : 16> Across;

  static __device__ __forceinline__ Along along(int lane) {
    Along a;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) a.at[ks] = (lane & 31) * RB + (((2 * ks + (lane >> 5)) ^ key(lane & 31)) << 4);
    return a;
  }
  static __device__ __forceinline__ Across across(int lane) {
    Across a;
    const int h = lane >> 5;
    if constexpr (EB == 2) {
      // within 16 lanes the transposing read gives lane j element t of source lane 4 t + j / 4, entry j % 4: source lane s points at
      // row s / 4 of four, channels of the four lanes from 4 (s % 4) on
      const int l16 = lane & 15;
#pragma unroll
      for (int i = 0; i < 2 * DB; ++i) {
        const int row = 8 * (i & 1) + 4 * h + (l16 >> 2), c = 32 * (i >> 1) + attn_order(16 * ((lane >> 4) & 1) + 4 * (l16 & 3));
        a.at[i] = row * RB + (((c >> 3) ^ key(row)) << 4) + (c & 7) * 2;
      }
    } else {
      // channel 32 db + order of row 8 ss + 4 h + e; db and ss count by their low bits, the rest is an offset
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int e = i & 3, ss = (i >> 2) & 1, c = 32 * (i >> 3) + attn_order(lane & 31), row = 8 * ss + 4 * h + e;
        a.at[i] = (4 * h + e) * RB + (((c >> 2) ^ key(row)) << 4) + (c & 3) * 4;
      }
    }
    return a;
  }

  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) const v4i lds_v4i;
  typedef __attribute__((address_space(3))) const int lds_int;

  // rows 32 b .. of the tile at `tile`, channels of product ks
  static __device__ __forceinline__ v4i read_along(const Along& a, unsigned tile, int b, int ks) {
    return *(lds_v4i*)(uint64_t)(a.at[ks] + (tile + b * 32 * RB));
  }
  // channels 32 db .. as rows; the rows 32 b + ... of the tile of product ss
  static __device__ __forceinline__ v4i read_across(const Across& a, unsigned tile, int b, int ss, int db) {
    if constexpr (EB == 2) {
      const unsigned at = tile + (b * 32 + ss * 16) * RB;
      struct { s16x4 lo, hi; } both = {
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uint64_t)(a.at[2 * db] + at)),
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uint64_t)(a.at[2 * db + 1] + at))};
      return __builtin_bit_cast(v4i, both);
    } else {
      v4i f;
      const unsigned at = tile + (b * 32 + ss * 8) * RB + 256 * (db >> 1);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = *(lds_int*)(uint64_t)(a.at[8 * (db & 1) + 4 * (ss & 1) + e] + at);
      return f;
    }
  }

  // results of a block, rounded, as second operand of the SS products across
  static __device__ __forceinline__ void pack(const floatx16& p, v4i (&f)[SS]) {
    T r[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) r[v] = E::from_float(p[v]);
    __builtin_memcpy(f, r, sizeof(r));
  }

  // a lane's share of a row in memory (channel groups 2 ks + h), as second operand of the products along; zeros beyond d
  template <int VEC> static __device__ __forceinline__ void read_row(const T* row, int d, int h, bool there, v4i (&f)[KS]) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) f[ks] = group<VEC>(row, (2 * ks + h) * V, d, there);
  }
  template <int VEC> static __device__ __forceinline__ v4i group(const T* row, int c, int d, bool there) {
    v4i g = {0, 0, 0, 0};
    if constexpr (VEC == 2) {
      if (there && c < d) g = *reinterpret_cast<const v4i*>(row + c);
    } else if (d >= V) {
      // whatever the alignment; a group that the row ends in is that of the row's end, moved down (entry by entry the training of 16 x 512 rows, 16
      // heads of 63 in f16, took 290 us in place of 162)
      const int at = min(c, d - V);
      if (there && c < d) __builtin_memcpy(&g, row + at, 16);
      if (d % V) {
        const int down = (c - at) * EB;
        if (EB == 2) {
#pragma unroll
          for (int i = 0; i < 4; ++i) g[i] = down & 2 ? (int)((unsigned)g[i] >> 16 | (unsigned)(i < 3 ? g[i < 3 ? i + 1 : i] : 0) << 16) : g[i];
        }
        g = down & 4 ? v4i{g[1], g[2], g[3], 0} : g;
        g = down & 8 ? v4i{g[2], g[3], 0, 0} : g;
        if (c >= d) g = v4i{0, 0, 0, 0};
      }
    } else {
      T e[V];
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = there && c + i < d ? row[c + i] : T(0);
      __builtin_memcpy(&g, e, 16);
    }
    return g;
  }

  // 16 channels from c0 on of a row, from a lane's results
  template <int VEC> static __device__ __forceinline__ void write_16(T* row, int c0, int d, const floatx16& o, float factor) {
    T r[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) r[v] = E::from_float(o[v] * factor);
    if constexpr (VEC == 2) {
      v4i g[EB];
      __builtin_memcpy(g, r, sizeof(r));
#pragma unroll
      for (int i = 0; i < EB; ++i)
        if (c0 + i * V < d) *reinterpret_cast<v4i*>(row + c0 + i * V) = g[i];
    } else {
#pragma unroll
      for (int i = 0; i < EB; ++i) write_group(row, c0 + i * V, d, r + i * V);
    }
  }
  // a 16-byte group whatever the alignment, of which the row may hold a part
  static __device__ __forceinline__ void write_group(T* row, int c, int d, const T* r) {
    if (c + V <= d) {
      __builtin_memcpy(row + c, r, 16);
    } else {
#pragma unroll
      for (int v = 0; v < V - 1; ++v)
        if (c + v < d) row[c + v] = r[v];
    }
  }

  // The same of rows of DP channels, `group` of them together and such groups `stride` entries apart: offsets of a lane's transfers, worked out
  // once, from the first row.
  template <int ROWS, int NT> struct Offsets { unsigned at[ROWS * GROUPS / NT]; };
  template <int ROWS, int NT> static __device__ __forceinline__ Offsets<ROWS, NT> offsets(int64_t stride, int group = 1, int t = threadIdx.x) {
    Offsets<ROWS, NT> o;
#pragma unroll
    for (int j = 0; j < ROWS * GROUPS / NT; ++j) {
      const int at = j * NT + t, r = at / GROUPS;
      o.at[j] = (unsigned)(r / group * (int)stride * EB + r % group * RB + ((at % GROUPS) ^ key(r)) * 16);
    }
    return o;
  }
  static constexpr int64_t kMostStride = (1 << 23) / EB;      // entries: offsets within 128 rows fit 31 bits
  template <int ROWS, int NT>
  static __device__ __forceinline__ void request_rows(unsigned tile, const T* first, const Offsets<ROWS, NT>& o) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int j = 0; j < ROWS * GROUPS / NT; ++j) attn_dma16(first, o.at[j], tile + (j * NT + wave * 64) * 16);
  }

  // Transfer of ROWS rows by NT lanes: `place(r)` is the row's address in memory, null for a row of zeros.
  template <int ROWS, int NT> static constexpr int transfers() { return ROWS * GROUPS / NT; }
  template <int ROWS, int NT, int VEC, class Place>
  static __device__ __forceinline__ void request(unsigned tile, int d, Place&& place, int t = threadIdx.x) {
    constexpr int J = ROWS * GROUPS / NT;
    static_assert(J >= 1 && ROWS * GROUPS % NT == 0, "whole transfers");
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    // (a wavefront that transfers alone has many addresses: eight at a time, and code that is read once costs as much as what it does: written
    // out, the gradients of 8 x 137 rows, 10 heads of 41 floats, took 90 us in place of 84)
    constexpr int TRANSFERS = VEC == 1 ? 4 * J : J, STEP = NT == 64 && TRANSFERS > 8 ? 8 : TRANSFERS;
    if constexpr (VEC == 1) {      // 4 bytes a lane
      constexpr int WORDS = RB / 4, PER = 4 / EB;
#pragma unroll 1
      for (int j0 = 0; j0 < TRANSFERS; j0 += STEP) {
        const void* from[STEP];
#pragma unroll
        for (int j = 0; j < STEP; ++j) {
          const int at = (j0 + j) * NT + t, r = at / WORDS, word = at % WORDS, c = (((word >> 2) ^ key(r)) << 2 | (word & 3)) * PER;
          const T* row = place(r);
          from[j] = row && c < d ? (const void*)(row + c) : (const void*)&attn_zeros;
        }
#pragma unroll
        for (int j = 0; j < STEP; ++j) attn_dma4(from[j], tile + ((j0 + j) * NT + wave * 64) * 4);
        if constexpr (STEP < TRANSFERS) __builtin_amdgcn_sched_barrier(0);
      }
      return;
    }
#pragma unroll
    for (int j0 = 0; j0 < TRANSFERS; j0 += STEP) {
      const T* from[STEP];
#pragma unroll
      for (int j = 0; j < STEP; ++j) from[j] = place(((j0 + j) * NT + t) / GROUPS);
#pragma unroll
      for (int j = 0; j < STEP; ++j) {
        const int at = (j0 + j) * NT + t, g = (at % GROUPS) ^ key(at / GROUPS);
        if constexpr (VEC == 2) {
          attn_dma16(from[j] && g * V < d ? (const void*)(from[j] + g * V) : (const void*)&attn_zeros, tile + ((j0 + j) * NT + wave * 64) * 16);
        } else {
          *(__attribute__((address_space(3))) v4i*)(uint64_t)(tile + at * 16) = group<0>(from[j], g * V, d, from[j] != nullptr);
        }
      }
      if constexpr (STEP < TRANSFERS) __builtin_amdgcn_sched_barrier(0);
    }
  }
};

}  // namespace sc
