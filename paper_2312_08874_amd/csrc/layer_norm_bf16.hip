#include "layer_norm_kernels.inc"

namespace aa {
hipError_t launch_layer_norm_bf16(const NormArgs& a, const NormShape& s, bool back, void* dw, void* db, hipStream_t st) {
  return dispatch_norm<ElemBF16>(a, s, back, dw, db, st);
}
}  // namespace aa
