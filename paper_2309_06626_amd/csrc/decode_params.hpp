// What the kernels of single tokens are told of a call.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sc {

constexpr int kDecodeWaves = 4;         // wavefronts of a workgroup
constexpr int kDecodePages = 2048;      // entries of the page table that a workgroup holds (two with codes fit a compute unit's LDS)

struct DecodeParams {
  const void *q, *k_pages, *v_pages;
  const float *k_scales, *v_scales;
  void* o;
  const int32_t *table, *lengths;
  float *part_o, *part_m;              // [rows][heads][splits][DP], and of maximum and sum
  int64_t rows, table_width;
  int32_t heads, kv_heads, d, pages, shift, row_bytes, window, splits, blocks, vec;
  float scale;
};

template <int DT> hipError_t decode_launch(const DecodeParams& p, bool bits8, hipStream_t s);

}  // namespace sc
