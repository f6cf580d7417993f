// Attention kernels of one element type.
#include "attn_kernel.hpp"

namespace sc {
template hipError_t attn_launch<kF32>(int what, const AttnParams& p, AttnTiles t, int vec, hipStream_t s);
}  // namespace sc
