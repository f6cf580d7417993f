// The kept rows of a mask, as the block operators use them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

struct sc_rows {
  int64_t rows, kept;    // with kept = 0 the lists are not looked at
  int32_t* row_idx;      // [kept] ascending
  int32_t* slot;         // [rows] position in row_idx, or -1
  int32_t* counts;       // [0] kept, [1 ..] kept rows of each part
};

namespace sc {
// +0.0 in every dropped row of a dense tensor; nothing where no row is dropped
hipError_t rows_zero_dropped(const sc_rows* set, int64_t row_bytes, void* out, hipStream_t s);
}  // namespace sc
