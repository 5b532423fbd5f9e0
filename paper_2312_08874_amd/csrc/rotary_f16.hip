#include "rotary_kernels.inc"

namespace aa {
hipError_t launch_rotary_f16(const RotaryArgs& a, int ve, const RotaryPlan& p, RotaryMode mode, hipStream_t st) {
  return dispatch<ElemF16>(a, ve, p, mode, st);
}
}  // namespace aa
