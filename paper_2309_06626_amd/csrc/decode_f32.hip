// Kernels of single tokens, of one element type.
#include "decode_kernel.hpp"

namespace sc {
template hipError_t decode_launch<kF32>(const DecodeParams& p, bool bits8, hipStream_t s);
}  // namespace sc
