#include "rotary_kernels.inc"

namespace aa {
hipError_t launch_rotary_bf16(const RotaryArgs& a, const RotaryShape& s, RotaryMode mode, int chunk, int blocks, hipStream_t st) {
  return dispatch<ElemBF16>(a, s, mode, chunk, blocks, st);
}
}  // namespace aa
