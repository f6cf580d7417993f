// Attention of single tokens over a paged cache of keys and values.
//
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q . k_j,  m = max s_j, over the first `length` rows of the sequence
//
// A workgroup takes the query heads of one key-value head (up to 32 of them) and a stretch of the sequence, of which its wavefronts take every
// fourth tile of 32 keys each, on their own: keys by heads are one 32 x 32 product, whose results, rounded, are an operand of the next.
// Maximum, sum and result of the wavefronts are joined in LDS, those of the stretches by a second launch, both in a fixed order.
//
// Bound by memory: a tile is 16 KB of 16-bit entries for 16 products, of whose columns a group of query heads fills some.  Entries go straight
// into LDS, where a wavefront has two tiles of keys and two of values, of which three are on their way (of floats above 64 channels one of each, asked
// for when both have been multiplied).  Measured, 8 key-value heads in bf16: 64 sequences of 4 096 to 8 192 rows 288 us with heads of 128 (5.6 TB/s;
// a plain copy 6.3), 152 of 64 (5.3), one of 100 000 rows 79 (5.2) and 44 (4.7); in floats, of the 64 sequences, 640 (5.0) and 442 (3.6).  Codes go
// through registers, where they are widened; 33 sequences of up to 4 000 rows, 4 heads: 28.3 us (2.5 TB/s), bound by the longest stretch's chain of
// widening, products and exponentials.
#pragma once
#include "attn_tile.hpp"
#include "decode_params.hpp"

#include <math.h>

namespace sc {

// 8-bit codes as entries of the type: whole numbers up to 127 are exact in it.
__device__ __forceinline__ void decode_widen(v4i codes, float (&out)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) out[i] = (float)(int8_t)(codes[i >> 2] >> (8 * (i & 3)));
}
// A byte below a half's 0x64 is 1 024 and the byte: code + 128 of these bytes, two at a time, less 1 152.
__device__ __forceinline__ void decode_widen(v4i codes, _Float16 (&out)[16]) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned bytes = (unsigned)codes[i] ^ 0x80808080u;
    const f16x2 less = {(_Float16)1152, (_Float16)1152};
    const f16x2 low = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, bytes, 0x04010400u)) - less;
    const f16x2 high = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, bytes, 0x04030402u)) - less;
    out[4 * i] = low[0];
    out[4 * i + 1] = low[1];
    out[4 * i + 2] = high[0];
    out[4 * i + 3] = high[1];
  }
}

// power of two at or below x (of normal numbers), and 1 / x of such a power
__device__ __forceinline__ float decode_pow2(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, x) & 0x7f800000u); }
__device__ __forceinline__ float decode_per(float pow2) { return __builtin_bit_cast(float, 0x7f000000u - __builtin_bit_cast(unsigned, pow2)); }

// What a lane holds of a row of q, as f16: in units of a power of two, so that the largest entry is between 2^13 and 2^14 (none is lost that
// is not below 2^-37 of it).  Returns the unit.
template <class From, class To, int KS> __device__ __forceinline__ float decode_narrow(const v4i (&from)[KS], v4i (&to)[KS]) {
  float x[KS][8], most = 0.0f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    From e[8];
    __builtin_memcpy(e, &from[ks], 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[ks][i] = (float)e[i];
      most = fmaxf(most, fabsf(x[ks][i]));
    }
  }
  most = attn_max_halves(most);
  const int up = most > 0.0f && most <= 3.4e38f ? min(14 - __builtin_amdgcn_frexp_expf(most), 100) : 0;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    To e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = (To)__builtin_amdgcn_ldexpf(x[ks][i], up);
    __builtin_memcpy(&to[ks], e, 16);
  }
  return __builtin_amdgcn_ldexpf(1.0f, -up);
}

template <int DT, int DP, bool BITS8>
__global__ __launch_bounds__(64 * kDecodeWaves, BITS8 && DT != kF32 ? 2 : 1) void decode_kernel(const DecodeParams p) {
  using IO = typename Elem<DT>::T;                             // of q and o
  constexpr int CT = BITS8 && DT == kBF16 ? kF16 : DT;         // codes are multiplied in f16, which they are widened to in the fewest operations
  using A = AttnTile<CT, DP>;
  using T = typename A::T;
  constexpr int TILE = 32 * A::RB, STAGES = BITS8 || A::RB > 256 ? 1 : 2, SCALES = 2 * 32 * 4;
  constexpr int LDS_WAVE = 2 * TILE * STAGES;
  constexpr int J = TILE / 1024;                               // transfers of 16 bytes a lane and tile
  extern __shared__ __align__(16) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, l32 = lane & 31;
  unsigned b = blockIdx.x;
  const int split = b % p.splits;
  b /= p.splits;
  const int head = b % p.kv_heads;                             // key-value head
  b /= p.kv_heads;
  const int block = b % p.blocks;                              // 32 query heads of it
  const int64_t row = b / p.blocks;

  // the keys of this stretch
  const int64_t most = (int64_t)p.table_width << p.shift;
  const int64_t length = p.lengths[row] < most ? p.lengths[row] : most;
  const int64_t begin = p.window && length > p.window ? length - p.window : 0;
  const int64_t first_tile = begin / 32, all_tiles = length > begin ? (length + 31) / 32 - first_tile : 0;
  int64_t per = (all_tiles + p.splits - 1) / p.splits;
  per = per < kDecodeWaves ? kDecodeWaves : per;
  const int64_t lo_tile = first_tile + split * per;
  const int tiles = (int)(split * per >= all_tiles ? 0 : all_tiles - split * per < per ? all_tiles - split * per : per);
  const int mine = tiles > wave ? (tiles - wave + kDecodeWaves - 1) / kDecodeWaves : 0;      // tiles of this wavefront

  // pages of the stretch, in LDS
  int32_t* const s_pages = reinterpret_cast<int32_t*>(smem + kDecodeWaves * (LDS_WAVE + SCALES));
  const int64_t first_page = (lo_tile * 32) >> p.shift;
  if (tiles) {
    const int64_t end = (lo_tile + tiles) * 32 < length ? (lo_tile + tiles) * 32 : length;
    const int count = min((int)(((end - 1) >> p.shift) - first_page) + 1, kDecodePages);      // (as many as there are, by the choice of splits)
    for (int i = t; i < count; i += 64 * kDecodeWaves) s_pages[i] = p.table[row * p.table_width + first_page + i];
  }
  const int group = p.heads / p.kv_heads, col = block * 32 + l32, q_head = head * group + col;
  const bool there = col < group;
  v4i qf[A::KS];
  float c = p.scale * 1.4426950408889634f;                     // of a product of q and k; of this lane's row
  {
    using Q = AttnTile<DT, DP>;
    v4i f[Q::KS];
    const IO* const q = static_cast<const IO*>(p.q) + (row * p.heads + (there ? q_head : 0)) * p.d;
    if (p.vec) Q::template read_row<2>(q, p.d, h, there, f);
    else Q::template read_row<0>(q, p.d, h, there, f);
    if constexpr (CT != DT) {
      c = fminf(fmaxf(c * decode_narrow<IO, T>(f, qf), 1e-37f), 3e38f);      // (neither 0 nor infinite, whatever the scale: scores are, times it)
    } else {
#pragma unroll
      for (int ks = 0; ks < A::KS; ++ks) qf[ks] = f[ks];
    }
  }
  __syncthreads();

  const unsigned lds = attn_lds(smem) + wave * (LDS_WAVE + SCALES), at_scales = lds + LDS_WAVE;
  // row of the cache that holds key l32 of a tile, or -1: beyond the length or the window, or on a page that is not there
  auto cache_row = [&](int i) -> int {
    const int64_t key = (lo_tile + wave + (int64_t)i * kDecodeWaves) * 32 + l32;
    if (key < begin || key >= length) return -1;
    const int page = s_pages[(key >> p.shift) - first_page];
    if ((unsigned)page >= (unsigned)p.pages) return -1;
    return (((unsigned)page * p.kv_heads + head) << p.shift) + (int)(key & ((1 << p.shift) - 1));
  };
  const unsigned char *const k_pages = static_cast<const unsigned char*>(p.k_pages), *const v_pages = static_cast<const unsigned char*>(p.v_pages);
  // entries as they are: straight into LDS
  const bool near = p.shift >= 5 && p.row_bytes == A::RB;      // a tile whose rows are all there is one piece of memory
  const auto off = A::template offsets<32, 64>(DP, 1, lane);
  auto request = [&](const unsigned char* pages, unsigned at, int at_row) {
    if (near && __ballot(at_row < 0) == 0) {
      const int64_t of = __builtin_amdgcn_readfirstlane(at_row);
#pragma unroll
      for (int j = 0; j < J; ++j) attn_dma16(pages + of * A::RB, off.at[j], at + j * 1024);
      return;
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int place = j * 64 + lane, r = place / A::GROUPS, g = (place % A::GROUPS) ^ A::key(r);
      const int64_t of = __shfl(at_row, r);
      const bool in = of >= 0 && g * 16 < p.row_bytes;
      attn_dma16(in ? (const void*)(pages + of * p.row_bytes + g * 16) : (const void*)&attn_zeros, at + j * 1024);
    }
  };
  auto request_k = [&](int i, int at_row) { request(k_pages, lds + (i % STAGES) * TILE, at_row); };
  auto request_v = [&](int i, int at_row) { request(v_pages, lds + (STAGES + i % STAGES) * TILE, at_row); };
  // codes: into registers, widened on the way to LDS
  constexpr int CG = DP / 16, CJ = BITS8 ? 32 * CG / 64 : 1;   // 16-byte groups of a row, and transfers of a tile
  struct Codes { v4i k[CJ], v[CJ]; float k_scale, v_scale; };
  auto fetch = [&](int at_row) -> Codes {
    Codes c;
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      const int place = j * 64 + lane, r = place / CG, g = place % CG;
      const int64_t of = __shfl(at_row, r);
      c.k[j] = c.v[j] = v4i{0, 0, 0, 0};
      if (of >= 0 && g * 16 < p.row_bytes) {
        c.k[j] = *reinterpret_cast<const v4i*>(k_pages + of * p.row_bytes + g * 16);
        c.v[j] = *reinterpret_cast<const v4i*>(v_pages + of * p.row_bytes + g * 16);
      }
    }
    c.k_scale = at_row >= 0 ? p.k_scales[at_row] : 0.0f;
    c.v_scale = at_row >= 0 ? p.v_scales[at_row] : 0.0f;
    return c;
  };
  auto widen = [&](const Codes& c) {
    if constexpr (BITS8) {
#pragma unroll
      for (int j = 0; j < CJ; ++j) {
        const int place = j * 64 + lane, r = place / CG, g = place % CG;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          T e[16];
          decode_widen(k ? c.v[j] : c.k[j], e);
          v4i w[A::EB];
          __builtin_memcpy(w, e, sizeof(e));
#pragma unroll
          for (int i = 0; i < A::EB; ++i)
            *(__attribute__((address_space(3))) v4i*)(uint64_t)(lds + k * TILE * STAGES + r * A::RB + (((g * A::EB + i) ^ A::key(r)) << 4)) = w[i];
        }
      }
      *(__attribute__((address_space(3))) float*)(uint64_t)(at_scales + lane * 4) = h ? c.v_scale : c.k_scale;
    }
  };

  typename A::Along along = A::along(lane);
  typename A::Across across = A::across(lane);
  // Floats of one stage: the tiles stay where they are, and their places go into the lanes' addresses (worked out at every read, they and what is read
  // were waited for one by one: 64 sequences of 4 096 to 8 192 rows, 8 heads of 128 floats, 643 us in place of 735 to 830).  Codes of 16-bit types have
  // no registers for it (28.3 and 30.6 us).
  constexpr bool FIXED = STAGES == 1 && sizeof(T) == 4;
  if constexpr (FIXED) {
    along.add(lds);
    across.add(lds);
  }
  floatx16 acc[A::DB];
#pragma unroll
  for (int db = 0; db < A::DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.0f;
  constexpr bool UP = DT == kF16 && !BITS8;                    // (the weights of codes are taken in units)
  float m = -INFINITY, sum = 0.0f, shift = 0.0f;               // m is a maximum times c, as it was rounded
  float unit = 0.0f, peak = 0.0f;                              // of codes in f16: acc is in units of it, see below

  typedef __attribute__((address_space(3))) const v4f lds_v4f;
  // Entries as they are: with two places for keys and two for values, whatever is in LDS is asked for again as soon as it has been multiplied, so
  // that three transfers of a tile are on their way all the time.  All but the youngest of them have landed, when N are waited for:
  auto wait = [&](int on_their_way) {
    if (on_their_way >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * J <= 63 ? 3 * J : 63) : "memory");
    else if (on_their_way == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * J <= 63 ? 2 * J : 63) : "memory");
    else if (on_their_way == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(J) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  };
  int rows[3] = {-1, -1, -1};                                  // of this tile and of the two behind it
  if (mine > 0) rows[0] = cache_row(0);
  if (mine > 1) rows[1] = cache_row(1);
  Codes codes;
  if constexpr (BITS8) {
    if (mine > 0) codes = fetch(rows[0]);
  } else if constexpr (STAGES > 1) {
    if (mine > 0) {
      request_k(0, rows[0]);
      request_v(0, rows[0]);
    }
    if (mine > 1) {
      request_k(1, rows[1]);
      request_v(1, rows[1]);
    }
  }
  for (int i = 0; i < mine; ++i) {
    const int left = mine - 1 - i;                             // tiles behind this one
    const uint64_t seen = __ballot(rows[0] >= 0);
    rows[2] = left > 1 ? cache_row(i + 2) : -1;
    if constexpr (BITS8) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the tile before is in registers)
      widen(codes);
      if (left > 0) codes = fetch(rows[1]);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    } else if constexpr (STAGES == 1) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      request_k(i, rows[0]);
      request_v(i, rows[0]);
      wait(0);
    } else {
      wait(left > 0 ? 3 : 1);
    }
    const unsigned at_k = FIXED ? 0 : lds + (i % STAGES) * TILE, at_v = FIXED ? TILE : lds + (STAGES + i % STAGES) * TILE;
    floatx16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < A::KS; ++ks) A::E::mma(s, A::read_along(along, at_k, 0, ks), qf[ks]);
    if constexpr (!BITS8 && STAGES > 1) {
      if (left > 1) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        request_k(i + 2, rows[2]);
      }
    }
    if constexpr (BITS8) {
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const v4f k_scale = *(lds_v4f*)(uint64_t)(at_scales + (8 * a + 4 * h) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * a + e] *= k_scale[e];
      }
    }
    const unsigned keys = (unsigned)seen;                      // (both halves hold the same 32)
    if (keys != 0xffffffffu) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = keys >> (8 * (v >> 2) + 4 * h + (v & 3)) & 1 ? s[v] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) top = fmaxf(top, s[v]);
    top = fmaxf(attn_max_halves(top) * c, m);
    // (a maximum that grew by less than 2^8 stays: weights of up to 256 are as good as those of up to 1)
    float less = 1.0f;
    auto rescale = [&]() {
#pragma unroll
      for (int db = 0; db < A::DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[db][v] *= less;
    };
    if (attn_any(top > m + 8.0f)) {
      const float next = attn_shift<UP>(top);
      less = m == -INFINITY ? 0.0f : attn_exp2(shift - next);
      shift = next;
      m = top;
      sum *= less;
      if constexpr (!BITS8) rescale();
    }
    float part[4];                                             // (one weight after the other is lost beside a large sum)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s[v] = attn_exp2(__builtin_fmaf(s[v], c, -shift));
      part[v & 3] = v < 4 ? s[v] : part[v & 3] + s[v];
    }
    sum += (part[0] + part[1]) + (part[2] + part[3]);
    if constexpr (BITS8) {
      // weights of the codes: p times the value's scale
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const v4f v_scale = *(lds_v4f*)(uint64_t)(at_scales + (32 + 8 * a + 4 * h) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * a + e] *= v_scale[e];
      }
      if constexpr (CT == kF16) {
        // in f16 in units of a power of two, 2^-6 to 2^-14 of this head's largest one so far (not of the largest scale, whose row may have no weight), so
        // that they keep their digits whatever the values' size, and those down to 2^-30 of the largest are not lost
        float big = s[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) big = fmaxf(big, s[v]);
        peak = fmaxf(peak * less, attn_max_halves(big));
        if (attn_any(peak > unit * 0x1p14f || less != 1.0f)) {
          const float next = decode_pow2(fminf(fmaxf(peak, 0x1p-119f), 0x1p127f)) * 0x1p-6f;
          less = less * unit * decode_per(next);      // (0 at first)
          unit = next;
        }
        const float per_unit = decode_per(unit);
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] *= per_unit;
      }
      if (attn_any(less != 1.0f)) rescale();
    }
    v4i pf[A::SS];
    A::pack(s, pf);
    if constexpr (!BITS8 && STAGES > 1) wait(left > 1 ? 3 : 2 * left);
#pragma unroll
    for (int ss = 0; ss < A::SS; ++ss)
#pragma unroll
      for (int db = 0; db < A::DB; ++db) A::E::mma(acc[db], A::read_across(across, at_v, 0, ss, db), pf[ss]);
    if constexpr (!BITS8 && STAGES > 1) {
      if (left > 1) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        request_v(i + 2, rows[2]);
      }
    }
    rows[0] = rows[1];
    rows[1] = rows[2];
  }
  if constexpr (BITS8 && CT == kF16) {
#pragma unroll
    for (int db = 0; db < A::DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[db][v] *= unit;
  }
  sum = attn_add_halves(sum);

  // the wavefronts' shares: [wave][column][DP] results, [wave][column] maxima and sums
  __syncthreads();
  const int cols = group - block * 32 < 32 ? group - block * 32 : 32;
  float* const s_acc = reinterpret_cast<float*>(smem);
  float* const s_max = s_acc + kDecodeWaves * 32 * DP;
  float* const s_sum = s_max + kDecodeWaves * 32;
  if (there) {
#pragma unroll
    for (int db = 0; db < A::DB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v4f part;
#pragma unroll
        for (int e = 0; e < 4; ++e) part[e] = acc[db][4 * q + e];
        *reinterpret_cast<v4f*>(s_acc + (wave * 32 + l32) * DP + 32 * db + 16 * h + 4 * q) = part;
      }
    if (h == 0) {
      s_max[wave * 32 + l32] = m == -INFINITY ? m : shift;
      s_sum[wave * 32 + l32] = sum;
    }
  }
  __syncthreads();
  for (int at = t; at < cols * DP; at += 64 * kDecodeWaves) {
    const int q = at / DP, ch = at % DP;
    float top = s_max[q];
#pragma unroll
    for (int w = 1; w < kDecodeWaves; ++w) top = fmaxf(top, s_max[w * 32 + q]);
    float all = 0.0f, out = 0.0f;
#pragma unroll
    for (int w = 0; w < kDecodeWaves; ++w) {
      const float sw = s_sum[w * 32 + q];
      if (sw == 0.0f) continue;
      const float f = attn_exp2(s_max[w * 32 + q] - top);
      all += sw * f;
      out += s_acc[(w * 32 + q) * DP + ch] * f;
    }
    const int64_t head_row = row * p.heads + head * group + block * 32 + q;
    if (p.splits == 1) {
      all = attn_total(top, all);
      if (ch < p.d) static_cast<IO*>(p.o)[head_row * p.d + ch] = Elem<DT>::from_float(all == 0.0f ? 0.0f : out / all);
    } else {
      p.part_o[(head_row * p.splits + split) * DP + ch] = out;
      if (ch == 0) {
        p.part_m[(head_row * p.splits + split) * 2] = top;
        p.part_m[(head_row * p.splits + split) * 2 + 1] = all;
      }
    }
  }
}

// The stretches' shares of a head, in a fixed order: eight teams of lanes take every eighth one each, four channels a lane.
template <int DT, int DP> __global__ __launch_bounds__(2 * DP) void decode_join_kernel(const DecodeParams p) {
  using T = typename Elem<DT>::T;
  constexpr int LANES = DP / 4, TEAMS = 8;
  __shared__ v4f s_out[TEAMS][LANES];
  __shared__ float s_all[TEAMS];
  const int64_t head_row = blockIdx.x;
  const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
  const float* const stat = p.part_m + head_row * p.splits * 2;
  float top = -INFINITY;
#pragma unroll 8
  for (int s = 0; s < p.splits; ++s) top = fmaxf(top, stat[2 * s]);
  float all = 0.0f;
  v4f out = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = team; s < p.splits; s += TEAMS) {
    const float sum = stat[2 * s + 1], f = sum == 0.0f ? 0.0f : attn_exp2(stat[2 * s] - top);
    const v4f part = *reinterpret_cast<const v4f*>(p.part_o + (head_row * p.splits + s) * DP + 4 * lane);
    all += sum * f;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] += part[e] * f;
  }
  s_out[team][lane] = out;
  if (lane == 0) s_all[team] = all;
  __syncthreads();
  if (team != 0) return;
#pragma unroll
  for (int i = 1; i < TEAMS; ++i) {
    all += s_all[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] += s_out[i][lane][e];
  }
  all = attn_total(top, all);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (4 * lane + e < p.d) static_cast<T*>(p.o)[head_row * p.d + 4 * lane + e] = Elem<DT>::from_float(all == 0.0f ? 0.0f : out[e] / all);
}

template <int DT, int DP, bool BITS8> static hipError_t decode_start(const DecodeParams& p, hipStream_t s) {
  using A = AttnTile<BITS8 && DT == kBF16 ? kF16 : DT, DP>;
  constexpr int wave = 2 * 32 * A::RB * (BITS8 || A::RB > 256 ? 1 : 2) + 2 * 32 * 4, join = kDecodeWaves * 32 * (DP + 2) * 4;
  constexpr int lds = (kDecodeWaves * wave + kDecodePages * 4) > join ? kDecodeWaves * wave + kDecodePages * 4 : join;
  static_assert(lds <= 160 * 1024, "LDS of a compute unit");
  auto kernel = decode_kernel<DT, DP, BITS8>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3((unsigned)(p.rows * p.blocks * p.kv_heads * p.splits)), dim3(64 * kDecodeWaves), lds, s>>>(p);
  if (p.splits > 1) decode_join_kernel<DT, DP><<<dim3((unsigned)(p.rows * p.heads)), dim3(2 * DP), 0, s>>>(p);
  return hipGetLastError();
}

template <int DT> hipError_t decode_launch(const DecodeParams& p, bool bits8, hipStream_t s) {
  if (p.d <= 64) return bits8 ? decode_start<DT, 64, true>(p, s) : decode_start<DT, 64, false>(p, s);
  return bits8 ? decode_start<DT, 128, true>(p, s) : decode_start<DT, 128, false>(p, s);
}

}  // namespace sc
