// Products of the gated feed-forward block: f16 operands.
#include "ffn_few_kernel.hpp"
#include "ffn_gemm_kernel.hpp"

namespace sc {
hipError_t ffn_launch_f16(FfnProduct what, const FfnGemm& g, int tile, bool whole, hipStream_t s) {
  return ffn_launch_type<kF16>(what, g, tile, whole, s);
}
hipError_t ffn_few_f16(bool gated, const FfnGemm& g, bool whole, hipStream_t s) { return ffn_few_type<kF16>(gated, g, whole, s); }
}  // namespace sc
