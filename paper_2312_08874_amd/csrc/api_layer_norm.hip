// C-ABI layer of the layer norm: argument validation, workspace checks and launches.
#include "../../include/agent_attn.h"

#include <math.h>

#include "kernels.h"
#include "row_ranges.h"

namespace {

using aa::NormArgs;
using aa::Range;
using aa::rows_of;

constexpr size_t kAlign = 256;

int elem_bytes(const aa_layer_norm* d) { return d->dtype == AA_F32 ? 4 : 2; }
size_t weight_bytes(const aa_layer_norm* d) { return (size_t)d->width * (d->weight_dtype == AA_F32 ? 4 : 2); }

aa_status check_desc(const aa_layer_norm* d) {
  if (!d) return AA_ERR_NULL;
  if (d->dtype != AA_F32 && d->dtype != AA_F16 && d->dtype != AA_BF16) return AA_ERR_DTYPE;
  if (d->weight_dtype != AA_F32 && d->weight_dtype != d->dtype) return AA_ERR_DTYPE;
  if (d->rows <= 0 || d->width <= 0) return AA_ERR_SHAPE;
  if (!(d->eps >= 0.0f) || !isfinite(d->eps)) return AA_ERR_SHAPE;
  if (d->width > aa::kNormWidth || d->rows > (1 << 30)) return AA_ERR_UNSUPPORTED;
  return AA_OK;
}

// rows of one tensor (v null or without data: there is none), and their place for the kernel
aa_status take(const aa_layer_norm* d, const aa_rows* v, bool needed, Range* range, aa::NormRows* to) {
  *range = Range{nullptr, 0};
  *to = aa::NormRows{nullptr, 0};
  if (!v || !v->data) return needed ? AA_ERR_NULL : AA_OK;
  const int64_t stride = v->stride ? v->stride : d->width;
  if (stride < d->width && d->rows > 1) return AA_ERR_SHAPE;
  if (stride > (1 << 21)) return AA_ERR_UNSUPPORTED;
  *range = rows_of(v->data, d->rows, stride, d->width, elem_bytes(d));
  *to = aa::NormRows{(char*)v->data, stride};
  return AA_OK;
}

bool same(const Range& a, const Range& b) { return a.p == b.p && a.pitch == b.pitch; }

NormArgs args_of(const aa_layer_norm* d) {
  NormArgs a{};
  a.rows = d->rows, a.width = d->width, a.eps = d->eps, a.inv = 1.0f / (float)d->width;
  a.wide_weights = d->weight_dtype == AA_F32;
  return a;
}

aa_status launch(const aa_layer_norm* d, NormArgs& a, bool back, void* dw, void* db, void* stream) {
  const aa::NormShape s = aa::norm_shape(elem_bytes(d), d->width, back);
  a.blocks = aa::norm_blocks(s, d->rows, back);
  const auto fn = d->dtype == AA_F32 ? aa::launch_layer_norm_f32 : d->dtype == AA_F16 ? aa::launch_layer_norm_f16 : aa::launch_layer_norm_bf16;
  return fn(a, s, back, dw, db, (hipStream_t)stream) == hipSuccess ? AA_OK : AA_ERR_HIP;
}

}  // namespace

extern "C" {

size_t agent_layer_norm_bwd_workspace_bytes(const aa_layer_norm* desc) {
  if (check_desc(desc) != AA_OK) return 0;
  const int blocks = aa::norm_blocks(aa::norm_shape(elem_bytes(desc), desc->width, true), desc->rows, true);
  return ((size_t)blocks * 2 * desc->width * 4 + kAlign - 1) / kAlign * kAlign;
}

aa_status agent_layer_norm_fwd(const aa_layer_norm* desc, const aa_rows* x, const aa_rows* residual, const void* weight, const void* bias,
                               const aa_rows* y, const aa_rows* sum, float* saved, void* hip_stream) {
  aa_status st = check_desc(desc);
  if (st != AA_OK) return st;
  NormArgs a = args_of(desc);
  Range in[2], out[2];
  if ((st = take(desc, x, true, &in[0], &a.x)) != AA_OK) return st;
  if ((st = take(desc, residual, false, &in[1], &a.r)) != AA_OK) return st;
  if ((st = take(desc, y, true, &out[0], &a.y)) != AA_OK) return st;
  if ((st = take(desc, sum, false, &out[1], &a.sum)) != AA_OK) return st;
  const size_t es = elem_bytes(desc), ws = desc->weight_dtype == AA_F32 ? 4 : 2;
  for (const Range& r : {in[0], in[1], out[0], out[1]})
    if ((uintptr_t)r.p % es) return AA_ERR_SHAPE;
  if ((uintptr_t)weight % ws || (uintptr_t)bias % ws || (uintptr_t)saved % 8) return AA_ERR_SHAPE;
  const Range stats{saved, (size_t)8 * desc->rows}, weights[2] = {{weight, weight_bytes(desc)}, {bias, weight_bytes(desc)}};
  for (const Range& o : out) {      // a result may be an input's own rows
    for (const Range& i : in)
      if (aa::meet(o, i) && !same(o, i)) return AA_ERR_ALIAS;
    if (aa::meet(o, stats) || aa::meet(o, weights[0]) || aa::meet(o, weights[1])) return AA_ERR_ALIAS;
  }
  if (aa::meet(out[0], out[1])) return AA_ERR_ALIAS;
  for (const Range& i : {in[0], in[1], weights[0], weights[1]})
    if (aa::meet(stats, i)) return AA_ERR_ALIAS;
  a.w = weight, a.b = bias, a.stats = (float2*)saved;
  return launch(desc, a, false, nullptr, nullptr, hip_stream);
}

aa_status agent_layer_norm_bwd(const aa_layer_norm* desc, const aa_rows* x, const aa_rows* residual, const aa_rows* dy, const float* saved,
                               const void* weight, const aa_rows* dsum, void* workspace, size_t workspace_bytes, const aa_rows* dx, void* dweight,
                               void* dbias, void* hip_stream) {
  aa_status st = check_desc(desc);
  if (st != AA_OK) return st;
  if (!saved) return AA_ERR_NULL;
  NormArgs a = args_of(desc);
  Range in[4], out;
  if ((st = take(desc, x, true, &in[0], &a.x)) != AA_OK) return st;
  if ((st = take(desc, dy, true, &in[1], &a.dy)) != AA_OK) return st;
  if ((st = take(desc, dsum, false, &in[2], &a.dsum)) != AA_OK) return st;
  if ((st = take(desc, residual, false, &in[3], &a.r)) != AA_OK) return st;
  if ((st = take(desc, dx, false, &out, &a.dx)) != AA_OK) return st;
  const size_t es = elem_bytes(desc), ws = desc->weight_dtype == AA_F32 ? 4 : 2;
  for (const Range& r : {in[0], in[1], in[2], in[3], out})
    if ((uintptr_t)r.p % es) return AA_ERR_SHAPE;
  if ((uintptr_t)weight % ws || (uintptr_t)dweight % ws || (uintptr_t)dbias % ws || (uintptr_t)saved % 8) return AA_ERR_SHAPE;
  const bool sums = dweight || dbias;
  const size_t need = sums ? agent_layer_norm_bwd_workspace_bytes(desc) : 0;
  if (sums && (!workspace || ((uintptr_t)workspace % kAlign) != 0 || workspace_bytes < need)) return AA_ERR_WORKSPACE;
  const Range written[] = {{sums ? workspace : nullptr, need}, {dweight, weight_bytes(desc)}, {dbias, weight_bytes(desc)}};
  const Range read[] = {in[0], in[1], in[2], in[3], {saved, (size_t)8 * desc->rows}, {weight, weight_bytes(desc)}};
  for (size_t i = 0; i < 3; ++i) {
    for (size_t j = 0; j < i; ++j)
      if (aa::meet(written[i], written[j])) return AA_ERR_ALIAS;
    for (const Range& r : read)
      if (aa::meet(written[i], r)) return AA_ERR_ALIAS;
    if (aa::meet(written[i], out)) return AA_ERR_ALIAS;
  }
  for (const Range& r : read)      // dx may be the rows of x, residual, dy or dsum
    if (aa::meet(out, r) && !(r.pitch != 0 && same(out, r))) return AA_ERR_ALIAS;
  if (!sums && !a.dx.data) return AA_OK;
  a.w = weight, a.stats = (float2*)const_cast<float*>(saved), a.partial = sums ? (float*)workspace : nullptr;
  return launch(desc, a, true, dweight, dbias, hip_stream);
}

}  // extern "C"
