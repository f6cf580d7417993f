// Kept rows of a token mask: ascending row list and the slot of every row in it.
//
// Two launches: workgroups count the kept bytes of their kRowsPart rows, then each adds up the counts before its own and writes its
// share of both lists, ranks within a wavefront from the ballot.  Memory moved: the mask twice, 4 bytes a row and 4 a kept row; 12 544 rows
// take 5 and 5 us, which are two launches and a round trip each, and the synchronisation that brings the count to the host.
#include "rows.hpp"

#include "../../include/sparse_block.h"

#include <new>

namespace sc {

void note_hip_error(int32_t code);

constexpr int kRowsPart = 4096, kRowsThreads = 256, kRowsTurns = kRowsPart / kRowsThreads;

__global__ __launch_bounds__(kRowsThreads) void rows_count_kernel(const uint8_t* __restrict__ mask, int64_t rows,
                                                                  int32_t* __restrict__ counts) {
  __shared__ int s_wave[kRowsThreads / 64];
  const int64_t base = (int64_t)blockIdx.x * kRowsPart;
  int kept = 0;
#pragma unroll
  for (int u = 0; u < kRowsTurns; ++u) {
    const int64_t r = base + u * kRowsThreads + threadIdx.x;
    kept += __popcll(__ballot(r < rows && mask[r] != 0));
  }
  if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = kept;
  __syncthreads();
  if (threadIdx.x == 0) {
    int all = 0;
#pragma unroll
    for (int w = 0; w < kRowsThreads / 64; ++w) all += s_wave[w];
    counts[1 + blockIdx.x] = all;
  }
}

// counts[0] receives the number of kept rows
__global__ __launch_bounds__(kRowsThreads) void rows_list_kernel(const uint8_t* __restrict__ mask, int64_t rows,
                                                                 int32_t* __restrict__ counts, int32_t* __restrict__ row_idx,
                                                                 int32_t* __restrict__ slot) {
  __shared__ int s_sum[kRowsThreads / 64], s_wave[kRowsTurns][kRowsThreads / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int before = 0;
  for (int i = t; i < (int)blockIdx.x; i += kRowsThreads) before += counts[1 + i];
#pragma unroll
  for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
  if (lane == 0) s_sum[wave] = before;
  const int64_t base = (int64_t)blockIdx.x * kRowsPart;
  unsigned long long ballots[kRowsTurns];
#pragma unroll
  for (int u = 0; u < kRowsTurns; ++u) {
    const int64_t r = base + u * kRowsThreads + t;
    ballots[u] = __ballot(r < rows && mask[r] != 0);
    if (lane == 0) s_wave[u][wave] = __popcll(ballots[u]);
  }
  __syncthreads();
  int at = 0;
#pragma unroll
  for (int w = 0; w < kRowsThreads / 64; ++w) at += s_sum[w];
#pragma unroll
  for (int u = 0; u < kRowsTurns; ++u) {
    int mine = at;
#pragma unroll
    for (int w = 0; w < kRowsThreads / 64; ++w) {
      if (w < wave) mine += s_wave[u][w];
      at += s_wave[u][w];
    }
    const int64_t r = base + u * kRowsThreads + t;
    const int rank = mine + __popcll(ballots[u] & ((1ull << lane) - 1));
    if (r < rows) {
      const bool keep = ballots[u] >> lane & 1;
      slot[r] = keep ? rank : -1;
      if (keep) row_idx[rank] = (int32_t)r;
    }
  }
  if (blockIdx.x == gridDim.x - 1 && t == 0) counts[0] = at;
}

// zeros in the dropped rows of a dense output (no slots: all are); one wavefront a row
__global__ __launch_bounds__(256) void rows_zero_kernel(const int32_t* __restrict__ slot, int64_t rows, int64_t row_bytes,
                                                        unsigned char* __restrict__ out) {
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += (int64_t)gridDim.x * 4) {
    if (slot && slot[r] >= 0) continue;
    unsigned char* row = out + r * row_bytes;
    typedef int v4 __attribute__((ext_vector_type(4)));
    if (row_bytes % 16 == 0) {
      for (int64_t i = (threadIdx.x & 63) * 16; i < row_bytes; i += 1024) *reinterpret_cast<v4*>(row + i) = v4{0, 0, 0, 0};
    } else {
      for (int64_t i = (threadIdx.x & 63) * 2; i < row_bytes; i += 128) *reinterpret_cast<uint16_t*>(row + i) = 0;
    }
  }
}

hipError_t rows_zero_dropped(const sc_rows* set, int64_t row_bytes, void* out, hipStream_t s) {
  if (!set || set->kept == set->rows || row_bytes == 0) return hipSuccess;
  const int64_t want = (set->rows + 3) / 4, most = 1 << 22;      // a launch has fewer than 2^32 lanes
  rows_zero_kernel<<<dim3((unsigned)(want < most ? want : most)), dim3(256), 0, s>>>(set->kept ? set->slot : nullptr, set->rows, row_bytes,
                                                                                  static_cast<unsigned char*>(out));
  return hipGetLastError();
}

static size_t rows_up(size_t n) { return (n + 255) & ~(size_t)255; }
static int64_t rows_parts(int64_t rows) { return (rows + kRowsPart - 1) / kRowsPart; }

static sc_status build(sc_rows* set, const uint8_t* mask, hipStream_t s) {
  set->kept = 0;      // and nothing is kept if this fails, whatever became of the lists
  if (set->rows == 0) return SC_OK;
  const unsigned parts = (unsigned)rows_parts(set->rows);
  rows_count_kernel<<<dim3(parts), dim3(kRowsThreads), 0, s>>>(mask, set->rows, set->counts);
  rows_list_kernel<<<dim3(parts), dim3(kRowsThreads), 0, s>>>(mask, set->rows, set->counts, set->row_idx, set->slot);
  hipError_t e = hipGetLastError();
  int32_t kept = 0;
  if (e == hipSuccess) e = hipMemcpyAsync(&kept, set->counts, sizeof(kept), hipMemcpyDeviceToHost, s);
  if (e == hipSuccess) e = hipStreamSynchronize(s);
  if (e != hipSuccess) { note_hip_error((int32_t)e); return SC_ERR_HIP; }
  set->kept = kept;
  return SC_OK;
}

}  // namespace sc

extern "C" {

sc_status sparse_rows_workspace_bytes(int64_t rows, size_t* bytes) {
  if (!bytes) return SC_ERR_NULL;
  *bytes = 0;
  if (rows < 0 || rows > 0x7fffffff) return SC_ERR_BAD_SHAPE;
  *bytes = 2 * sc::rows_up((size_t)rows * 4) + sc::rows_up((size_t)(1 + sc::rows_parts(rows)) * 4);
  return SC_OK;
}

sc_status sparse_rows_plan(const uint8_t* mask_dev, int64_t rows, void* workspace_dev, size_t workspace_bytes, void* hip_stream,
                           sc_rows** out) {
  if (!out) return SC_ERR_NULL;
  *out = nullptr;
  size_t need = 0;
  sc_status st = sparse_rows_workspace_bytes(rows, &need);
  if (st != SC_OK) return st;
  if ((!mask_dev && rows > 0) || !workspace_dev) return SC_ERR_NULL;
  if (workspace_bytes < need) return SC_ERR_WORKSPACE;
  if ((uintptr_t)workspace_dev & 15) return SC_ERR_ALIGN;
  sc_rows* set = new (std::nothrow) sc_rows;
  if (!set) return SC_ERR_HIP;
  unsigned char* w = static_cast<unsigned char*>(workspace_dev);
  set->rows = rows;
  set->row_idx = reinterpret_cast<int32_t*>(w);
  set->slot = reinterpret_cast<int32_t*>(w + sc::rows_up((size_t)rows * 4));
  set->counts = reinterpret_cast<int32_t*>(w + 2 * sc::rows_up((size_t)rows * 4));
  st = sc::build(set, mask_dev, static_cast<hipStream_t>(hip_stream));
  if (st != SC_OK) {
    delete set;
    return st;
  }
  *out = set;
  return SC_OK;
}

sc_status sparse_rows_set_mask(sc_rows* set, const uint8_t* mask_dev, void* hip_stream) {
  if (!set || (!mask_dev && set->rows > 0)) return SC_ERR_NULL;
  return sc::build(set, mask_dev, static_cast<hipStream_t>(hip_stream));
}

sc_status sparse_rows_info(const sc_rows* set, int64_t* rows, int64_t* kept, const int32_t** row_idx_dev, const int32_t** slot_dev) {
  if (!set) return SC_ERR_NULL;
  if (rows) *rows = set->rows;
  if (kept) *kept = set->kept;
  if (row_idx_dev) *row_idx_dev = set->row_idx;
  if (slot_dev) *slot_dev = set->slot;
  return SC_OK;
}

void sparse_rows_destroy(sc_rows* set) { delete set; }

}  // extern "C"
