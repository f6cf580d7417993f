// Products of the gated feed-forward block: bf16 operands.
#include "ffn_few_kernel.hpp"
#include "ffn_gemm_kernel.hpp"

namespace sc {
hipError_t ffn_launch_bf16(FfnProduct what, const FfnGemm& g, int tile, bool whole, hipStream_t s) {
  return ffn_launch_type<kBF16>(what, g, tile, whole, s);
}
hipError_t ffn_few_bf16(bool gated, const FfnGemm& g, bool whole, hipStream_t s) { return ffn_few_type<kBF16>(gated, g, whole, s); }
}  // namespace sc
