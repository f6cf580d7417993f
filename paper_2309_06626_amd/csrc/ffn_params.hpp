// Host-side description of the products of the gated feed-forward block, and the launchers of each element type.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

namespace sc {

// C[i][j] = sum_k P[i][k] Q[j][k].  An operand is "along k" (its rows are those of the result, k runs within them) or "across k"
// (its rows are those of the contraction).
enum FfnProduct : int32_t {
  kFfnUp = 0,       // P along, Q = gate and up weights along: hidden = act(P Wg') * (P Wu'), and with `saved` the two products
  kFfnDown = 1,     // P along, Q along
  kFfnGateGrad = 2, // P along, Q across: the product is the gradient of the hidden rows; leaves those of gate and up, and hidden again
  kFfnInGrad = 3,   // P along, Q across, two pairs of operands summed
  kFfnWGrad = 4     // P across, Q across, one or two P with results of their own
};

// Rows of operands are whole 16-byte groups, with zeros behind the last entry; so are the rows that a product leaves for the next one.
struct FfnGemm {
  const void* p[2];
  const void* q[2];
  int64_t ldp, ldq;            // elements from row to row
  const int32_t* p_rows;       // row of p that row i (of the result, or of the contraction) stands for; null: i
  const int32_t* q_rows;
  int32_t m, n, k;             // result rows and columns, contraction
  int32_t segments;            // pairs (p[s], q[s]) whose products are summed
  int32_t batch;               // results c[z] of p[z] with q[0]
  void* c[2];
  int64_t ldc;                 // (of kFfnUp's and kFfnGateGrad's results: whole groups)
  const int32_t* c_rows;       // row of c that receives result row i; null: i
  void* saved;                 // [3][m][n], see FfnSaved.  kFfnUp: written, may be null.  kFfnGateGrad: read
  void* hidden;                // kFfnGateGrad: like c; null where it is not wanted
  int32_t activation;
  int32_t splits;              // parts of the contraction, each with its sums in `partial`
  float* partial;              // [batch, or gate and up][splits][m][n up to a multiple of 4]
  // set by the launcher
  int32_t m_tiles, n_tiles, group;
};

// tile: index into the launcher's list of tile shapes; whole: rows of `saved` and of all results are whole groups too
hipError_t ffn_launch_bf16(FfnProduct what, const FfnGemm& g, int tile, bool whole, hipStream_t s);
hipError_t ffn_launch_f16(FfnProduct what, const FfnGemm& g, int tile, bool whole, hipStream_t s);
hipError_t ffn_launch_f32(FfnProduct what, const FfnGemm& g, int tile, bool whole, hipStream_t s);

// kFfnUp (gated) and kFfnDown for a few rows
hipError_t ffn_few_bf16(bool gated, const FfnGemm& g, bool whole, hipStream_t s);
hipError_t ffn_few_f16(bool gated, const FfnGemm& g, bool whole, hipStream_t s);
hipError_t ffn_few_f32(bool gated, const FfnGemm& g, bool whole, hipStream_t s);

// Kernels with more than 64 KB of LDS have to say so, once on each device.
inline hipError_t ffn_allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& told) {
  if (bytes <= 65536) return hipSuccess;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (told.load(std::memory_order_relaxed) & bit)) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) told.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

}  // namespace sc
