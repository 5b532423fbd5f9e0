#include "kernels.h"

#include "ffn_rows_kernels.inc"

namespace aa {
hipError_t launch_ffn_product_bf16(const FfnGroup& g, FfnForm form, FfnEpilogue epi, int rows, int cols, hipStream_t st) {
  return product<ElemBF16>(g, form, epi, rows, cols, st);
}
hipError_t launch_ffn_rows_bf16(const FfnRows& a, bool gate, int waves, hipStream_t st) { return rows_product<ElemBF16>(a, gate, waves, st); }
}  // namespace aa
