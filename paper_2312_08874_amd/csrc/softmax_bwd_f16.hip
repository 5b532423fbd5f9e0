#include "softmax_bwd_kernels.inc"

namespace aa {
hipError_t launch_softmax_bwd_f16(const SoftmaxArgs& a, SoftmaxPass pass, int tiles, hipStream_t st) {
  return dispatch_backward<ElemF16>(a, pass, tiles, st);
}
}  // namespace aa
