// What the attention kernels are told of a call.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sc {

struct AttnItem {      // a workgroup's share: a tile of a sequence
  int32_t first, rows; // the sequence's first kept row, and how many it has
  int32_t tile, pad;
};

struct AttnParams {
  const void *q, *k, *v, *o, *d_o;
  void *out, *dq, *dk, *dv;
  int64_t q_stride, k_stride, v_stride, dq_stride, dk_stride, dv_stride;      // entries from row to row; o and d_o are [rows][heads][d]
  float* lse;                          // [kept][heads]
  float* stats[2];                     // the same of the backward pass: lse in exponents of 2, and delta
  const int32_t* map;                  // row of the tensors that holds a kept row; null: row r is kept row r
  const AttnItem* items;
  int32_t n_items, heads, kv_heads, group, d;
  int32_t causal, window;              // window 0: none
  uint32_t magic;                      // ceil(2^20 / group)
  float scale;
};

// waves: wavefronts of a workgroup; vec: all rows are whole 16-byte groups
template <int DT> hipError_t attn_launch(int what, const AttnParams& p, int waves, bool vec, hipStream_t s);

constexpr int kAttnKeyWaves = 4;                            // wavefronts of a workgroup of the keys' gradients, 32 keys each
enum { kAttnForward, kAttnBackwardQ, kAttnBackwardKV };

}  // namespace sc
