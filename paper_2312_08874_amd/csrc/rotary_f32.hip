#include "rotary_kernels.inc"

namespace aa {
hipError_t launch_rotary_f32(const RotaryArgs& a, const RotaryShape& s, RotaryMode mode, int chunk, int blocks, hipStream_t st) {
  return dispatch<ElemF32>(a, s, mode, chunk, blocks, st);
}
}  // namespace aa
