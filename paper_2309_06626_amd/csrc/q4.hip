// Products of a few rows with weights in 4 bits: y[r][n] = sum_k x[r][k] (code[n][k] - zero[n][g]) scale[n][g], g = k / group.
//
// Bound by reading the weights once: n k / 2 bytes and 4 bytes a group of every output.  What follows from that:
//   * matrix instructions although there are few rows: 16 outputs x 32 columns of codes times 32 columns x 16 rows take one 16-cycle
//     instruction, against hundreds of vector operations, and cost the same for 1 and for 16 rows;
//   * codes become operands without arithmetic: OR-ed into the mantissa of 128 (bf16) or 1024 (f16) they are exactly 128 + code.  With
//     B that number, sum_k x (code - zero) = sum_k x (B + code) - (B + zero) sum_k x; the second sum comes from the matrix unit too (a
//     left operand of ones leaves it in every lane that needs it).  Both are sums of a group in float, where B costs 7 (10) of 24 bits;
//   * scales act on a group's sums, four outputs a lane, and not on the codes;
//   * the plan lays codes out in the order in which lanes take them: 16 outputs x 128 columns are 1 KB, read by one wavefront at once,
//     its dword j the columns 32 j + 8 (lane / 16) .. + 7, in the nibble order that one AND-OR a pair undoes;
//   * a workgroup has 16 outputs and eight or sixteen wavefronts, which share the columns; their sums meet in LDS, in order.
// Measured, bf16, one row: 4 096 -> 4 096 3.9 us (2.3 TB/s, most of it a launch), 11 264 -> 4 096 8.0 (3.1 TB/s), gated 4 096 -> 11 264 14.3
// (3.6 TB/s).  More rows read x again in every workgroup: the gated block 4 096 -> 11 264 -> 4 096 takes 21 us for 1 row, 23 for 8, 30 for
// 16 and 115 for 64.
#include "../../include/sparse_block.h"
#include "ffn_act.hpp"
#include "mma_common.hpp"

#include <initializer_list>
#include <new>

struct sc_q4 {
  sc_q4_desc desc;
  int32_t gated, activation;
  const void* codes[2];
  const void* scales[2];
};

namespace sc {

void note_hip_error(int32_t code);

constexpr int kQ4MostRows = 64;      // of a workgroup; more rows take more workgroups, which read the weights again

template <int DT> struct Q4Elem;
template <> struct Q4Elem<kBF16> {
  static constexpr unsigned BIAS = 0x43004300u, ONES = 0x3f803f80u;
  static constexpr float B = 128.0f;
  static __device__ __forceinline__ v4f mma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Q4Elem<kF16> {
  static constexpr unsigned BIAS = 0x64006400u, ONES = 0x3c003c00u;
  static constexpr float B = 1024.0f;
  static __device__ __forceinline__ v4f mma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

// codes [n][ceil(k / 2)] -> [n / 16][k / 128][lane][4] dwords; beyond n and k codes are 0
__global__ __launch_bounds__(256) void q4_codes_kernel(const uint8_t* __restrict__ codes, int n, int k, int blocks, int64_t dwords,
                                                       unsigned* __restrict__ out) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= dwords) return;
  const int j = at & 3, lane = (int)(at >> 2) & 63;
  const int64_t unit = at >> 8;
  const int row = (int)(unit / blocks) * 16 + (lane & 15), col = (int)(unit % blocks) * 128 + 32 * j + 8 * (lane >> 4);
  const int64_t pitch = (k + 1) / 2;
  unsigned v = 0;
  if (row < n) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = col + e;
      if (c < k) {
        const unsigned code = codes[(int64_t)row * pitch + (c >> 1)] >> ((c & 1) * 4) & 15u;
        v |= code << ((e & 1) * 16 + (e >> 1) * 4);      // elements 0, 1 in bits 0-3 of the halves, 2, 3 in bits 4-7, ...
      }
    }
  }
  out[at] = v;
}

// scales and zeros [n][groups] -> [n / 16][groups of whole blocks][n % 16 / 4][4 scales, 4 zeros]; beyond n and k a scale is 0
template <typename T>
__global__ __launch_bounds__(256) void q4_scales_kernel(const T* __restrict__ scales, const T* __restrict__ zeros, int n, int groups,
                                                        int all_groups, int64_t count, T* __restrict__ out) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= count) return;
  const int i = at & 3, is_zero = (int)(at >> 2) & 1, quad = (int)(at >> 3) & 3;
  const int64_t unit = at >> 5;
  const int g = (int)(unit % all_groups);
  const int64_t row = unit / all_groups * 16 + quad * 4 + i;
  T v = T(0);
  if (row < n && g < groups) v = !is_zero ? scales[row * groups + g] : zeros ? zeros[row * groups + g] : T(8.0f);
  out[at] = v;
}

struct Q4Params {
  const void *x, *codes[2], *scales[2];
  void* y;
  int64_t rows;
  int32_t k, n, blocks, groups, activation;
};

// GROUP columns share a scale; MT tiles of 16 rows; MATS 2: act(x gate') (x up'); AHEAD blocks of 128 columns asked for at once
template <int DT, int GROUP, int MT, int MATS, int WAVES, int AHEAD>
__global__ __launch_bounds__(64 * WAVES) void q4_kernel(const Q4Params p) {
  using Q = Q4Elem<DT>;
  using T = typename Elem<DT>::T;
  constexpr int PER = GROUP / 32, GPB = 4 / PER;      // matrix instructions a group, groups a block of 128 columns
  extern __shared__ float q4_sum[];                   // [WAVES][MATS][MT][64][4]
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int col = lane & 15, kg = lane >> 4;
  const int64_t row0 = (int64_t)blockIdx.y * kQ4MostRows;
  const int tile = blockIdx.x;

  const v4i* codes[MATS];
  const v4i* scales[MATS];
#pragma unroll
  for (int m = 0; m < MATS; ++m) {
    codes[m] = static_cast<const v4i*>(p.codes[m]) + (int64_t)tile * p.blocks * 64 + lane;
    scales[m] = static_cast<const v4i*>(p.scales[m]) + (int64_t)tile * p.groups * 4 + kg;
  }
  const T* x[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t r = row0 + 16 * i + col;            // a row that is not there: the first one again, whose results are not stored
    x[i] = static_cast<const T*>(p.x) + (r < p.rows ? r : 0) * p.k + 8 * kg;
  }
  const v4i ones = {(int)Q::ONES, (int)Q::ONES, (int)Q::ONES, (int)Q::ONES};

  v4f acc[MATS][MT];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[m][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  struct Block { v4i w[MATS], sz[MATS][GPB], x[MT][4]; };
  auto ask = [&](int b, Block& k) {
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      k.w[m] = codes[m][(int64_t)b * 64];
#pragma unroll
      for (int g = 0; g < GPB; ++g) k.sz[m][g] = scales[m][((int64_t)b * GPB + g) * 4];
    }
    if ((b + 1) * 128 <= p.k) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) __builtin_memcpy(&k.x[i][j], x[i] + b * 128 + 32 * j, 16);
    } else {                                          // the rows end within this block
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = b * 128 + 32 * j, left = p.k - c - 8 * kg;
          k.x[i][j] = v4i{0, 0, 0, 0};
          if (left >= 8) {
            __builtin_memcpy(&k.x[i][j], x[i] + c, 16);
          } else if (left > 0) {
            T e[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) e[u] = u < left ? x[i][c + u] : T(0);
            __builtin_memcpy(&k.x[i][j], e, 16);
          }
        }
    }
  };
  auto add = [&](const Block& k) {
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      v4f sum[MATS][MT], xs[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        xs[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int m = 0; m < MATS; ++m) sum[m][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      }
#pragma unroll
      for (int j = g * PER; j < (g + 1) * PER; ++j) {
#pragma unroll
        for (int i = 0; i < MT; ++i) xs[i] = Q::mma(ones, k.x[i][j], xs[i]);
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
          const unsigned c = (unsigned)k.w[m][j];
          v4i a;
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] = (int)((c >> (4 * e) & 0x000f000fu) | Q::BIAS);
#pragma unroll
          for (int i = 0; i < MT; ++i) sum[m][i] = Q::mma(a, k.x[i][j], sum[m][i]);
        }
      }
#pragma unroll
      for (int m = 0; m < MATS; ++m) {
        T e[8];
        __builtin_memcpy(e, &k.sz[m][g], 16);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float s = (float)e[q], z = Q::B + (float)e[4 + q];
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[m][i][q] += s * (sum[m][i][q] - z * xs[i][q]);
        }
      }
    }
  };
  int b = wave;
  for (; b + (AHEAD - 1) * WAVES < p.blocks; b += AHEAD * WAVES) {
    Block k[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) ask(b + u * WAVES, k[u]);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) add(k[u]);
  }
  if constexpr (AHEAD > 1) {
    for (; b < p.blocks; b += WAVES) {
      Block k;
      ask(b, k);
      add(k);
    }
  }
  v4f* const mine = reinterpret_cast<v4f*>(q4_sum) + wave * (MATS * MT * 64) + lane;
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int i = 0; i < MT; ++i) mine[(m * MT + i) * 64] = acc[m][i];
  __syncthreads();
  // value v of a tile: lane v / 4 of the accumulators, output 4 (lane / 16) + v % 4, row lane % 16
  for (int at = t; at < MT * 256; at += 64 * WAVES) {
    const int n16 = at & 15, r = at >> 4;      // outputs of one row next to each other
    const int word = ((r >> 4) * 64 + (n16 >> 2) * 16 + (r & 15)) * 4 + (n16 & 3);
    float v[MATS];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      v[m] = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v[m] += q4_sum[(w * MATS + m) * (MT * 256) + word];
    }
    const int n = tile * 16 + n16;
    const int64_t row = row0 + r;
    if (n < p.n && row < p.rows) {
      float out = v[0];
      if constexpr (MATS == 2) {
        float a, da;
        ffn_act<T>(p.activation, v[0], a, da);
        out = a * v[1];
      }
      static_cast<T*>(p.y)[row * p.n + n] = (T)out;
    }
  }
}

template <int DT, int GROUP, int MT, int MATS, int WAVES, int AHEAD> static void q4_launch(const Q4Params& p, hipStream_t s) {
  constexpr int lds = WAVES * MATS * MT * 1024;
  static_assert(lds <= 65536, "no more than any kernel may have");
  const dim3 grid((unsigned)((p.n + 15) / 16), (unsigned)((p.rows + kQ4MostRows - 1) / kQ4MostRows));
  q4_kernel<DT, GROUP, MT, MATS, WAVES, AHEAD><<<grid, dim3(64 * WAVES), lds, s>>>(p);
}
// Sixteen wavefronts where there are no more than two workgroups a compute unit: they ask for as much at once as twice as many workgroups.
template <int DT, int GROUP, int MATS> static void q4_launch_rows(const Q4Params& p, hipStream_t s) {
  constexpr int AHEAD = MATS == 2 ? 1 : 2;      // of sixteen wavefronts: registers
  if (p.rows <= 16) {
    if (p.n <= 512 * 16) q4_launch<DT, GROUP, 1, MATS, 16, AHEAD>(p, s);
    else q4_launch<DT, GROUP, 1, MATS, 8, 2>(p, s);
  } else if (p.rows <= 32) {
    q4_launch<DT, GROUP, 2, MATS, 8, 1>(p, s);
  } else {
    q4_launch<DT, GROUP, 4, MATS, 8, 1>(p, s);
  }
}
template <int DT, int MATS> static void q4_launch_group(int group, const Q4Params& p, hipStream_t s) {
  if (group == 32) q4_launch_rows<DT, 32, MATS>(p, s);
  else if (group == 64) q4_launch_rows<DT, 64, MATS>(p, s);
  else q4_launch_rows<DT, 128, MATS>(p, s);
}

// ---- host ---------------------------------------------------------------------------------------------------------------------
static int q4_blocks(const sc_q4_desc& d) { return (d.k + 127) / 128; }
static int q4_groups(const sc_q4_desc& d) { return q4_blocks(d) * (128 / d.group); }
static int64_t q4_tiles(const sc_q4_desc& d) { return (d.n + 15) / 16; }
static size_t q4_code_bytes(const sc_q4_desc& d) { return (size_t)q4_tiles(d) * q4_blocks(d) * 1024; }
static size_t q4_scale_bytes(const sc_q4_desc& d) { return (size_t)q4_tiles(d) * q4_groups(d) * 64; }

static sc_status check_q4(const sc_q4_desc* d) {
  if (!d) return SC_ERR_NULL;
  if (d->dtype != SC_F16 && d->dtype != SC_BF16) return SC_ERR_UNSUPPORTED;
  if (d->group != 32 && d->group != 64 && d->group != 128) return SC_ERR_UNSUPPORTED;
  if (d->k < 1 || d->n < 1 || d->k > (1 << 24) || d->n > (1 << 24)) return SC_ERR_BAD_SHAPE;
  return SC_OK;
}

static sc_status q4_lay_out(const sc_q4_desc& d, const uint8_t* codes, const void* scales, const void* zeros, unsigned char* at,
                            hipStream_t s) {
  const int64_t dwords = (int64_t)(q4_code_bytes(d) / 4), count = (int64_t)(q4_scale_bytes(d) / 2);
  const int groups = (d.k + d.group - 1) / d.group;
  q4_codes_kernel<<<dim3((unsigned)((dwords + 255) / 256)), dim3(256), 0, s>>>(codes, d.n, d.k, q4_blocks(d), dwords,
                                                                              reinterpret_cast<unsigned*>(at));
  unsigned char* const to = at + q4_code_bytes(d);
  const dim3 grid((unsigned)((count + 255) / 256));
  if (d.dtype == SC_BF16)
    q4_scales_kernel<__bf16><<<grid, dim3(256), 0, s>>>((const __bf16*)scales, (const __bf16*)zeros, d.n, groups, q4_groups(d), count,
                                                       reinterpret_cast<__bf16*>(to));
  else
    q4_scales_kernel<_Float16><<<grid, dim3(256), 0, s>>>((const _Float16*)scales, (const _Float16*)zeros, d.n, groups, q4_groups(d),
                                                         count, reinterpret_cast<_Float16*>(to));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

static sc_status q4_plan(const sc_q4_desc* d, int gated, int activation, const uint8_t* const codes[2], const void* const scales[2],
                         const void* const zeros[2], void* workspace, size_t workspace_bytes, void* stream, sc_q4** out) {
  if (!out) return SC_ERR_NULL;
  *out = nullptr;
  size_t need = 0;
  sc_status st = sparse_q4_workspace_bytes(d, gated, &need);
  if (st != SC_OK) return st;
  if (activation < SC_ACT_SILU || activation > SC_ACT_GELU_TANH) return SC_ERR_UNSUPPORTED;
  if (!workspace) return SC_ERR_NULL;
  uintptr_t low = (uintptr_t)workspace;
  for (int m = 0; m <= gated; ++m) {
    if (!codes[m] || !scales[m]) return SC_ERR_NULL;
    low |= (uintptr_t)codes[m] | (uintptr_t)scales[m] | (uintptr_t)zeros[m];
  }
  if (workspace_bytes < need) return SC_ERR_WORKSPACE;
  if (low & 15) return SC_ERR_ALIGN;
  sc_q4* plan = new (std::nothrow) sc_q4;
  if (!plan) return SC_ERR_HIP;
  plan->desc = *d;
  plan->gated = gated;
  plan->activation = activation;
  unsigned char* at = static_cast<unsigned char*>(workspace);
  for (int m = 0; m <= gated; ++m) {
    st = q4_lay_out(*d, codes[m], scales[m], zeros[m], at, static_cast<hipStream_t>(stream));
    if (st != SC_OK) {
      delete plan;
      return st;
    }
    plan->codes[m] = at;
    plan->scales[m] = at + q4_code_bytes(*d);
    at += q4_code_bytes(*d) + q4_scale_bytes(*d);
  }
  *out = plan;
  return SC_OK;
}

}  // namespace sc

extern "C" {

sc_status sparse_q4_workspace_bytes(const sc_q4_desc* desc, int32_t gated, size_t* bytes) {
  if (!bytes) return SC_ERR_NULL;
  *bytes = 0;
  const sc_status st = sc::check_q4(desc);
  if (st != SC_OK) return st;
  *bytes = (gated ? 2 : 1) * (sc::q4_code_bytes(*desc) + sc::q4_scale_bytes(*desc));
  return SC_OK;
}

sc_status sparse_q4_plan(const sc_q4_desc* desc, const uint8_t* codes_dev, const void* scales_dev, const void* zeros_dev,
                         void* workspace_dev, size_t workspace_bytes, void* hip_stream, sc_q4** out) {
  const uint8_t* const codes[2] = {codes_dev, nullptr};
  const void* const scales[2] = {scales_dev, nullptr};
  const void* const zeros[2] = {zeros_dev, nullptr};
  return sc::q4_plan(desc, 0, SC_ACT_SILU, codes, scales, zeros, workspace_dev, workspace_bytes, hip_stream, out);
}

sc_status sparse_q4_plan_gated(const sc_q4_desc* desc, int32_t activation, const uint8_t* gate_codes_dev,
                               const void* gate_scales_dev, const void* gate_zeros_dev, const uint8_t* up_codes_dev,
                               const void* up_scales_dev, const void* up_zeros_dev, void* workspace_dev, size_t workspace_bytes,
                               void* hip_stream, sc_q4** out) {
  const uint8_t* const codes[2] = {gate_codes_dev, up_codes_dev};
  const void* const scales[2] = {gate_scales_dev, up_scales_dev};
  const void* const zeros[2] = {gate_zeros_dev, up_zeros_dev};
  return sc::q4_plan(desc, 1, activation, codes, scales, zeros, workspace_dev, workspace_bytes, hip_stream, out);
}

sc_status sparse_q4_run(const sc_q4* plan, int64_t rows, const void* x_dev, void* y_dev, void* hip_stream) {
  if (!plan) return SC_ERR_NULL;
  if (rows < 0 || rows > 65535 * (int64_t)sc::kQ4MostRows) return SC_ERR_BAD_SHAPE;
  if (rows > 0 && (!x_dev || !y_dev)) return SC_ERR_NULL;
  if (((uintptr_t)x_dev | (uintptr_t)y_dev) & 15) return SC_ERR_ALIGN;
  if (rows == 0) return SC_OK;
  sc::Q4Params p = {};
  p.x = x_dev;
  p.y = y_dev;
  for (int m = 0; m < 2; ++m) {
    p.codes[m] = plan->gated || m == 0 ? plan->codes[m] : nullptr;
    p.scales[m] = plan->gated || m == 0 ? plan->scales[m] : nullptr;
  }
  p.rows = rows;
  p.k = plan->desc.k;
  p.n = plan->desc.n;
  p.blocks = sc::q4_blocks(plan->desc);
  p.groups = sc::q4_groups(plan->desc);
  p.activation = plan->activation;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool bf16 = plan->desc.dtype == SC_BF16;
  if (plan->gated) {
    if (bf16) sc::q4_launch_group<sc::kBF16, 2>(plan->desc.group, p, s);
    else sc::q4_launch_group<sc::kF16, 2>(plan->desc.group, p, s);
  } else {
    if (bf16) sc::q4_launch_group<sc::kBF16, 1>(plan->desc.group, p, s);
    else sc::q4_launch_group<sc::kF16, 1>(plan->desc.group, p, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { sc::note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

void sparse_q4_destroy(sc_q4* plan) { delete plan; }

}  // extern "C"
