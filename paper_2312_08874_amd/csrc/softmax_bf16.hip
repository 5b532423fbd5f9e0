#include "softmax_kernels.inc"

namespace aa {
hipError_t launch_softmax_bf16(const SoftmaxArgs& a, SoftmaxPass pass, int tiles, hipStream_t st) {
  return dispatch_forward<ElemBF16>(a, pass, tiles, st);
}
}  // namespace aa
