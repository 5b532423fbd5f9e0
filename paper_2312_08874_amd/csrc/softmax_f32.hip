#include "softmax_kernels.inc"

namespace aa {
hipError_t launch_softmax_f32(const SoftmaxArgs& a, SoftmaxPass pass, int tiles, hipStream_t st) {
  return dispatch_forward<ElemF32>(a, pass, tiles, st);
}
}  // namespace aa
