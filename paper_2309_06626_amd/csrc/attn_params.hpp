// What the attention kernels are told of a call.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sc {

struct AttnItem {      // a workgroup's share: a tile of a sequence
  int32_t first, rows; // the sequence's first kept row, and how many it has
  int32_t tile, pad;
};

struct AttnZeros {                     // dropped rows of up to three dense outputs
  const int32_t* slot;                 // null: every row is dropped
  int64_t rows;
  void* out[3];
  int64_t stride[3], width[3];         // bytes
  int32_t blocks, vec;                 // workgroups that write them (0: none); whole 16-byte groups
};

struct AttnParams {
  const void *q, *k, *v, *o, *d_o;
  void *out, *dq, *dk, *dv;
  int64_t q_stride, k_stride, v_stride, dq_stride, dk_stride, dv_stride;      // entries from row to row; o and d_o are [rows][heads][d]
  float* lse;                          // [kept][heads]
  float* stats[2];                     // of the backward pass, as the keys' gradients take them: lse in exponents of 2, and delta
  const int32_t* map;                  // row of the tensors that holds a kept row; null: row r is kept row r
  const AttnItem* items;
  int32_t n_items, heads, kv_heads, group, d;
  int32_t causal, window;              // window 0: none
  uint32_t magic;                      // ceil(2^20 / group)
  float scale;
  AttnZeros zeros;
};

struct AttnTiles {
  int32_t waves;                       // wavefronts of a workgroup, 32 packed rows each; 1: four that share 32
  int32_t keys;                        // of a tile that passes by (forward)
};

// vec: rows are whole 16-byte groups (2), 4-byte ones (1) or neither (0)
template <int DT> hipError_t attn_launch(int what, const AttnParams& p, AttnTiles t, int vec, hipStream_t s);
template <int DT> hipError_t attn_few_launch(int what, const AttnParams& p, int vec, hipStream_t s);

constexpr int kAttnKeyWaves = 4;                            // wavefronts of a workgroup of the keys' gradients, 32 keys each
enum { kAttnForward, kAttnBackwardQ, kAttnBackwardKV };

}  // namespace sc
