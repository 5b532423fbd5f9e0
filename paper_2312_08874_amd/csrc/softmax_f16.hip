#include "softmax_kernels.inc"

namespace aa {
hipError_t launch_softmax_f16(const SoftmaxArgs& a, SoftmaxPass pass, int tiles, hipStream_t st) {
  return dispatch_forward<ElemF16>(a, pass, tiles, st);
}
}  // namespace aa
