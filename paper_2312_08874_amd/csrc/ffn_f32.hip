#include "kernels.h"

#include "ffn_kernels.inc"

namespace aa {
hipError_t launch_ffn_product_f32(const FfnProduct& a, FfnForm form, FfnEpilogue epi, const FfnTile& t, hipStream_t st) {
  return product<ElemF32>(a, form, epi, t, st);
}
}  // namespace aa
