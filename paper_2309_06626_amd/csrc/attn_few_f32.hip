// Attention kernels of few rows, of one element type.
#include "attn_few.hpp"

namespace sc {
template hipError_t attn_few_launch<kF32>(int what, const AttnParams& p, int vec, hipStream_t s);
}  // namespace sc
