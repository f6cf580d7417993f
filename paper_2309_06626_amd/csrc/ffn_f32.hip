// Products of the gated feed-forward block: f32 operands.
#include "ffn_gemm_kernel.hpp"

namespace sc {
hipError_t ffn_launch_f32(FfnProduct what, const FfnGemm& g, int tile, bool aligned, hipStream_t s) {
  return ffn_launch_type<kF32>(what, g, tile, aligned, s);
}
}  // namespace sc
