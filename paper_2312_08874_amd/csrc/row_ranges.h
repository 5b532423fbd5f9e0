// Tensors of rows as the C-ABI layer checks them: what of their memory a call touches, and whether two of them meet.
#pragma once
#include "../../include/agent_attn.h"

namespace aa {

struct Range {
  const void* p;
  size_t bytes;
  size_t pitch = 0, row = 0;      // rows of `row` bytes, `pitch` apart; 0: one piece
};
inline Range rows_of(const void* p, long long rows, long long ld, size_t cols, size_t es) {
  return Range{p, ((size_t)(rows - 1) * ld + cols) * es, (size_t)ld * es, cols * es};
}
inline bool meet(const Range& a, const Range& b) {
  if (!a.p || !b.p) return false;
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  if (x >= y + b.bytes || y >= x + a.bytes) return false;
  if (a.pitch == 0 || a.pitch != b.pitch) return true;
  const size_t at = y >= x ? (y - x) % a.pitch : (a.pitch - (x - y) % a.pitch) % a.pitch;      // columns of one buffer are apart
  return at < a.row || at + b.row > a.pitch;
}
// `results` are written (the workspace among them), `inputs` read: no result may meet another or an input
template <size_t R, size_t I>
inline aa_status check_ranges(const Range (&results)[R], const Range (&inputs)[I], size_t elem) {
  for (size_t i = 0; i < R; ++i) {
    if ((uintptr_t)results[i].p % elem) return AA_ERR_SHAPE;
    for (size_t j = 0; j < i; ++j)
      if (meet(results[i], results[j])) return AA_ERR_ALIAS;
    for (const Range& in : inputs)
      if (meet(results[i], in)) return AA_ERR_ALIAS;
  }
  for (const Range& in : inputs)
    if ((uintptr_t)in.p % elem) return AA_ERR_SHAPE;
  return AA_OK;
}

}  // namespace aa
