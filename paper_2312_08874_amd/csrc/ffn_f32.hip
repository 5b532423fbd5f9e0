#include "kernels.h"

#include "ffn_rows_kernels.inc"

namespace aa {
hipError_t launch_ffn_product_f32(const FfnGroup& g, FfnForm form, FfnEpilogue epi, int rows, int cols, hipStream_t st) {
  return product<ElemF32>(g, form, epi, rows, cols, st);
}
hipError_t launch_ffn_rows_f32(const FfnRows& a, bool gate, int waves, hipStream_t st) { return rows_product<ElemF32>(a, gate, waves, st); }
}  // namespace aa
