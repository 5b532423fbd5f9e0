#include "rotary_kernels.inc"

namespace aa {
hipError_t launch_rotary_bf16(const RotaryArgs& a, int ve, const RotaryPlan& p, RotaryMode mode, hipStream_t st) {
  return dispatch<ElemBF16>(a, ve, p, mode, st);
}
}  // namespace aa
