// C-ABI layer of the gated feed-forward block: argument validation and workspace checks.
#include "../../include/agent_attn.h"

#include "kernels.h"
#include "row_ranges.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int kMaxWidth = 1 << 20, kMaxRows = 1 << 30;

aa_status check_ffn(const aa_ffn* d) {
  if (!d) return AA_ERR_NULL;
  if (d->dtype != AA_F32 && d->dtype != AA_F16 && d->dtype != AA_BF16) return AA_ERR_DTYPE;
  if (d->rows <= 0 || d->width <= 0 || d->hidden <= 0) return AA_ERR_SHAPE;
  if (d->activation < AA_SILU || d->activation > AA_SIGMOID) return AA_ERR_SHAPE;
  for (int64_t s : {d->x_stride, d->y_stride, d->dx_stride}) {
    if (s != 0 && s < d->width) return AA_ERR_SHAPE;
    if (s > 2 * kMaxWidth) return AA_ERR_UNSUPPORTED;
  }
  if (d->width > kMaxWidth || d->hidden > kMaxWidth || d->rows > kMaxRows) return AA_ERR_UNSUPPORTED;
  if ((int64_t)d->rows * (d->width > d->hidden ? d->width : d->hidden) >= (int64_t)1 << 40) return AA_ERR_UNSUPPORTED;
  return AA_OK;
}

aa::FfnBlock block_of(const aa_ffn* d) {
  aa::FfnBlock b{};
  b.T = d->rows, b.C = d->width, b.F = d->hidden, b.dtype = d->dtype, b.activation = d->activation;
  b.ldx = d->x_stride ? d->x_stride : d->width;
  b.ldy = d->y_stride ? d->y_stride : d->width;
  b.lddx = d->dx_stride ? d->dx_stride : d->width;
  return b;
}

using aa::Range;
using aa::check_ranges;
using aa::rows_of;

}  // namespace

extern "C" {

size_t agent_gated_ffn_workspace_bytes(const aa_ffn* desc) {
  return check_ffn(desc) == AA_OK ? aa::ffn_fwd_workspace(block_of(desc)) : 0;
}
size_t agent_gated_ffn_saved_bytes(const aa_ffn* desc) {
  return check_ffn(desc) == AA_OK ? aa::ffn_saved_bytes(block_of(desc)) : 0;
}
size_t agent_gated_ffn_bwd_workspace_bytes(const aa_ffn* desc) {
  return check_ffn(desc) == AA_OK ? aa::ffn_bwd_workspace(block_of(desc)) : 0;
}

aa_status agent_gated_ffn_fwd(const aa_ffn* desc, const void* x, const aa_ffn_weights* w, void* saved, void* workspace,
                              size_t workspace_bytes, void* y, void* hip_stream) {
  const aa_status st = check_ffn(desc);
  if (st != AA_OK) return st;
  if (!x || !w || !w->w_gate || !w->w_up || !w->w_down || !y) return AA_ERR_NULL;
  aa::FfnBlock b = block_of(desc);
  if (!workspace || ((uintptr_t)workspace % kAlign) != 0) return AA_ERR_WORKSPACE;
  if (((uintptr_t)saved % kAlign) != 0) return AA_ERR_WORKSPACE;
  const size_t es = b.es(), C = b.C, F = b.F, in = C * F * es;
  const Range results[] = {rows_of(y, b.T, b.ldy, C, es), {workspace, workspace_bytes}, {saved, aa::ffn_saved_bytes(b)}};
  const Range inputs[] = {rows_of(x, b.T, b.ldx, C, es), {w->w_gate, in}, {w->w_up, in}, {w->w_down, in},
                          {w->b_gate, F * es}, {w->b_up, F * es}, {w->b_down, C * es}};
  const aa_status at = check_ranges(results, inputs, es);
  if (at != AA_OK) return at;
  b.x = x, b.w_gate = w->w_gate, b.b_gate = w->b_gate, b.w_up = w->w_up, b.b_up = w->b_up;
  b.w_down = w->w_down, b.b_down = w->b_down, b.y = y;
  bool room;
  const hipError_t err = aa::launch_ffn_fwd(b, saved, workspace, workspace_bytes, &room, (hipStream_t)hip_stream);
  return !room ? AA_ERR_WORKSPACE : err == hipSuccess ? AA_OK : AA_ERR_HIP;
}

aa_status agent_gated_ffn_bwd(const aa_ffn* desc, const void* x, const aa_ffn_weights* w, const void* saved, const void* dy,
                              void* workspace, size_t workspace_bytes, void* dx, const aa_ffn_grads* g, void* hip_stream) {
  const aa_status st = check_ffn(desc);
  if (st != AA_OK) return st;
  if (!x || !w || !w->w_gate || !w->w_up || !w->w_down || !saved || !dy) return AA_ERR_NULL;
  aa::FfnBlock b = block_of(desc);
  if (!workspace || ((uintptr_t)workspace % kAlign) != 0) return AA_ERR_WORKSPACE;
  if (((uintptr_t)saved % kAlign) != 0) return AA_ERR_WORKSPACE;
  const aa_ffn_grads none{}, *to = g ? g : &none;
  const size_t es = b.es(), C = b.C, F = b.F, in = C * F * es;
  const Range results[] = {rows_of(dx, b.T, b.lddx, C, es), {workspace, workspace_bytes}, {to->dw_gate, in}, {to->dw_up, in},
                           {to->dw_down, in}, {to->db_gate, F * es}, {to->db_up, F * es}, {to->db_down, C * es}};
  const Range inputs[] = {rows_of(x, b.T, b.ldx, C, es), rows_of(dy, b.T, b.ldy, C, es), {w->w_gate, in},
                          {w->w_up, in}, {w->w_down, in}, {saved, aa::ffn_saved_bytes(b)}};
  const aa_status at = check_ranges(results, inputs, es);
  if (at != AA_OK) return at;
  b.x = x, b.w_gate = w->w_gate, b.w_up = w->w_up, b.w_down = w->w_down, b.dy = dy, b.dx = dx;
  b.dw_gate = to->dw_gate, b.dw_up = to->dw_up, b.dw_down = to->dw_down;
  b.db_gate = to->db_gate, b.db_up = to->db_up, b.db_down = to->db_down;
  bool room;
  const hipError_t err = aa::launch_ffn_bwd(b, saved, workspace, workspace_bytes, &room, (hipStream_t)hip_stream);
  return !room ? AA_ERR_WORKSPACE : err == hipSuccess ? AA_OK : AA_ERR_HIP;
}

}  // extern "C"
