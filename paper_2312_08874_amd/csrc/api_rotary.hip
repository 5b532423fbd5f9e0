// C-ABI layer of the rotary positions and of the norms of queries and keys: argument validation and launches.
#include "../../include/agent_attn.h"

#include <math.h>

#include "kernels.h"
#include "token_views.h"

namespace {

using aa::RotaryArgs;
using aa::RotaryMode;

constexpr size_t kAlign = 256;

using Span = aa::TokenSpan;
using aa::bytes_meet;

aa_status check_rotary(const aa_rotary* r) {
  if (!r) return AA_ERR_NULL;
  if (r->dtype != AA_F32 && r->dtype != AA_F16 && r->dtype != AA_BF16) return AA_ERR_DTYPE;
  if (r->batch <= 0 || r->tokens <= 0 || r->heads_q <= 0 || r->heads_k < 0 || r->d <= 0) return AA_ERR_SHAPE;
  if (r->axes < 0 || r->axes > aa::kRotaryAxes) return AA_ERR_SHAPE;
  if (r->d > 2 * aa::kRotaryPairs) return AA_ERR_UNSUPPORTED;
  if ((int64_t)r->batch * r->tokens >= (int64_t)1 << 31 || (int64_t)r->heads_q + r->heads_k > 65535) return AA_ERR_UNSUPPORTED;
  if (r->axes == 0) return AA_OK;
  if (r->pairing < AA_ROPE_ADJACENT || r->pairing > AA_ROPE_AXIS_HALVES) return AA_ERR_SHAPE;
  int64_t pairs = 0, cells = 1;
  bool any = false, all = true;
  for (int x = 0; x < r->axes; ++x) {
    if (r->pairs[x] <= 0 || r->pairs[x] > aa::kRotaryPairs) return AA_ERR_SHAPE;
    pairs += r->pairs[x];
    if (r->grid[x] < 0) return AA_ERR_SHAPE;
    any = any || r->grid[x] > 0;
    all = all && r->grid[x] > 0;
    if (all && cells <= r->tokens) cells *= r->grid[x];
  }
  if (2 * pairs > r->d) return AA_ERR_SHAPE;
  if (any ? !all || cells != r->tokens || r->positions : !r->positions) return any ? AA_ERR_SHAPE : AA_ERR_NULL;
  if (r->positions && ((uintptr_t)r->positions & 3)) return AA_ERR_SHAPE;
  if (!r->freq) return AA_ERR_NULL;
  for (int64_t j = 0; j < pairs; ++j)
    if (!isfinite(r->freq[j])) return AA_ERR_SHAPE;
  return AA_OK;
}

int elem_bytes(const aa_rotary* r) { return r->dtype == AA_F32 ? 4 : 2; }

aa_status check_view(const aa_rotary* r, const aa_view* v, int heads, bool result, Span* out) {
  *out = Span{nullptr, 0, 0, 0, r->batch, heads, r->tokens, r->d, elem_bytes(r)};
  return aa::check_token_view(v, result, out);
}

void place(aa::TokenView* v, const Span& s) { *v = aa::TokenView{s.data, s.sb, s.sh, s.sn}; }

// Validates the views of one call and fills the kernel's arguments; groups: the inputs, the gradients (or null), the results.
aa_status make_args(const aa_rotary* r, const aa_view* const in[2], const aa_view* const grad[2], const aa_view* const out[2],
                    RotaryArgs* a, aa::RotaryShape* shape) {
  *a = RotaryArgs{};
  a->batch = r->batch, a->tokens = r->tokens, a->heads[0] = r->heads_q, a->heads[1] = r->heads_k, a->d = r->d;
  a->axes = r->axes, a->pairing = r->pairing, a->sign = 1.0f;
  const int es = elem_bytes(r), tensors = r->heads_k > 0 ? 2 : 1;
  Span spans[6];
  int n = 0;
  unsigned long long align = 0;
  for (int g = 0; g < 3; ++g) {
    const aa_view* const* group = g == 0 ? in : g == 1 ? grad : out;
    if (!group) continue;
    for (int i = 0; i < tensors; ++i) {
      Span s;
      const aa_status st = check_view(r, group[i], a->heads[i], g == 2, &s);
      if (st != AA_OK) return st;
      align |= (uintptr_t)s.data | (unsigned long long)((s.sb | s.sh | s.sn) * es);
      place(g == 0 ? &a->in[i] : g == 1 ? &a->grad[i] : &a->out[i], s);
      spans[n++] = s;
    }
  }
  // results: their own input or gradient, or apart from everything
  const int results = n - tensors;
  for (int o = results; o < n; ++o)
    for (int i = 0; i < n; ++i) {
      if (i == o || (i < results && i % tensors == o - results && spans[i].same_place(spans[o]))) continue;
      if (aa::spans_meet(spans[i], spans[o])) return AA_ERR_ALIAS;
    }
  if (r->axes > 0) {
    for (int x = 0; x < aa::kRotaryAxes; ++x) {
      a->first[x + 1] = a->first[x] + (x < r->axes ? r->pairs[x] : 0);
      a->grid[x] = x < r->axes && !r->positions ? r->grid[x] : 0;
    }
    a->pairs = a->first[r->axes];
    for (int j = 0; j < a->pairs; ++j) a->turn[j] = r->freq[j] / 6.283185307179586476925;
    if (r->positions) {
      a->positions = r->positions;
      a->positions_float = r->positions_float != 0;
      a->positions_batch = r->positions_shared ? 0 : (long long)r->tokens * r->axes;
      const size_t bytes = (size_t)4 * r->axes * r->tokens * (r->positions_shared ? 1 : r->batch);
      for (int o = results; o < n; ++o)
        if (bytes_meet(spans[o].data, spans[o].bytes(), r->positions, bytes)) return AA_ERR_ALIAS;
    }
  }
  *shape = aa::rotary_shape(es, r->d, r->pairing, r->axes, a->first, align);
  return AA_OK;
}

aa_status check_norm(const aa_rotary* r, const aa_qk_norm* norm) {
  if (!norm) return AA_ERR_NULL;
  if (!(norm->eps >= 0.0f) || !isfinite(norm->eps)) return AA_ERR_SHAPE;
  if (((uintptr_t)norm->w_q & 3) || (r->heads_k > 0 && ((uintptr_t)norm->w_k & 3))) return AA_ERR_SHAPE;
  return AA_OK;
}

// without keys w_k may be anything: waves without heads would read it
const float* weight_of(const aa_rotary* r, const aa_qk_norm* norm, int which) {
  return which == 0 ? norm->w_q : r->heads_k > 0 ? norm->w_k : nullptr;
}

size_t weight_bytes(const aa_rotary* r, const aa_qk_norm* norm, int which) {
  return (size_t)4 * r->d * (norm->per_head ? (which ? r->heads_k : r->heads_q) : 1);
}

// whether the bytes meet one of the results
bool results_meet(const aa_rotary* r, const RotaryArgs& a, const void* p, size_t bytes) {
  for (int i = 0; i < (r->heads_k > 0 ? 2 : 1); ++i) {
    const aa::TokenView& v = a.out[i];
    const long long n = (r->batch - 1) * v.sb + (a.heads[i] - 1) * v.sh + (r->tokens - 1) * v.sn + r->d;
    if (bytes_meet(v.data, (size_t)n * elem_bytes(r), p, bytes)) return true;
  }
  return false;
}

aa_status rotate(const aa_rotary* desc, const aa_view* q, const aa_view* k, const aa_view* q_out, const aa_view* k_out, float sign,
                 void* hip_stream) {
  aa_status st = check_rotary(desc);
  if (st != AA_OK) return st;
  if (desc->axes == 0) return AA_ERR_SHAPE;
  RotaryArgs a;
  aa::RotaryShape shape;
  const aa_view *in[2] = {q, k}, *out[2] = {q_out, k_out};
  st = make_args(desc, in, nullptr, out, &a, &shape);
  if (st != AA_OK) return st;
  a.sign = sign;
  return aa::launch_rotary(desc->dtype, a, shape, RotaryMode::kRotate, nullptr, nullptr, (hipStream_t)hip_stream) == hipSuccess
             ? AA_OK : AA_ERR_HIP;
}

}  // namespace

extern "C" {

aa_status agent_rope_fwd(const aa_rotary* desc, const aa_view* q, const aa_view* k, const aa_view* q_out, const aa_view* k_out,
                         void* hip_stream) {
  return rotate(desc, q, k, q_out, k_out, 1.0f, hip_stream);
}

aa_status agent_rope_bwd(const aa_rotary* desc, const aa_view* dq_out, const aa_view* dk_out, const aa_view* dq, const aa_view* dk,
                         void* hip_stream) {
  return rotate(desc, dq_out, dk_out, dq, dk, -1.0f, hip_stream);
}

aa_status agent_qk_norm_fwd(const aa_rotary* desc, const aa_qk_norm* norm, const aa_view* q, const aa_view* k, const aa_view* q_out,
                            const aa_view* k_out, void* hip_stream) {
  aa_status st = check_rotary(desc);
  if (st != AA_OK) return st;
  st = check_norm(desc, norm);
  if (st != AA_OK) return st;
  RotaryArgs a;
  aa::RotaryShape shape;
  const aa_view *in[2] = {q, k}, *out[2] = {q_out, k_out};
  st = make_args(desc, in, nullptr, out, &a, &shape);
  if (st != AA_OK) return st;
  for (int i = 0; i < 2; ++i) {
    a.weight[i] = weight_of(desc, norm, i);
    if (results_meet(desc, a, a.weight[i], weight_bytes(desc, norm, i))) return AA_ERR_ALIAS;
  }
  a.weight_heads = norm->per_head != 0, a.eps = norm->eps;
  return aa::launch_rotary(desc->dtype, a, shape, RotaryMode::kNorm, nullptr, nullptr, (hipStream_t)hip_stream) == hipSuccess
             ? AA_OK : AA_ERR_HIP;
}

size_t agent_qk_norm_bwd_workspace_bytes(const aa_rotary* desc, const aa_qk_norm* norm) {
  if (check_rotary(desc) != AA_OK || check_norm(desc, norm) != AA_OK) return 0;
  RotaryArgs a{};
  a.heads[0] = desc->heads_q, a.heads[1] = desc->heads_k, a.d = desc->d, a.weight_heads = norm->per_head != 0;
  return (aa::rotary_partial_floats(a) * 4 + kAlign - 1) / kAlign * kAlign;
}

aa_status agent_qk_norm_bwd(const aa_rotary* desc, const aa_qk_norm* norm, const aa_view* q, const aa_view* k, const aa_view* dq_out,
                            const aa_view* dk_out, void* workspace, size_t workspace_bytes, const aa_view* dq, const aa_view* dk,
                            float* dw_q, float* dw_k, void* hip_stream) {
  aa_status st = check_rotary(desc);
  if (st != AA_OK) return st;
  st = check_norm(desc, norm);
  if (st != AA_OK) return st;
  RotaryArgs a;
  aa::RotaryShape shape;
  const aa_view *in[2] = {q, k}, *grad[2] = {dq_out, dk_out}, *out[2] = {dq, dk};
  st = make_args(desc, in, grad, out, &a, &shape);
  if (st != AA_OK) return st;
  if (desc->heads_k == 0) dw_k = nullptr;
  float* dw[2] = {dw_q, dw_k};
  const bool sums = dw_q || dw_k;
  if (sums && (!workspace || ((uintptr_t)workspace % kAlign) != 0 || workspace_bytes < agent_qk_norm_bwd_workspace_bytes(desc, norm)))
    return AA_ERR_WORKSPACE;
  if (!sums) workspace_bytes = 0;
  const int es = elem_bytes(desc), tensors = desc->heads_k > 0 ? 2 : 1;
  if (results_meet(desc, a, workspace, workspace_bytes)) return AA_ERR_ALIAS;
  for (int i = 0; i < 2; ++i) {
    const size_t bytes = weight_bytes(desc, norm, i);
    a.weight[i] = weight_of(desc, norm, i);
    if ((uintptr_t)dw[i] & 3) return AA_ERR_SHAPE;
    if (results_meet(desc, a, a.weight[i], bytes) || results_meet(desc, a, dw[i], bytes)) return AA_ERR_ALIAS;
    if (bytes_meet(workspace, workspace_bytes, a.weight[i], bytes) || bytes_meet(workspace, workspace_bytes, dw[i], bytes)) return AA_ERR_ALIAS;
    for (int j = 0; j < 2; ++j)
      if (bytes_meet(dw[i], bytes, weight_of(desc, norm, j), weight_bytes(desc, norm, j))) return AA_ERR_ALIAS;
    for (int j = 0; j < tensors; ++j)
      for (const aa::TokenView* v : {&a.in[j], &a.grad[j]}) {
        const long long n = (desc->batch - 1) * v->sb + (a.heads[j] - 1) * v->sh + (desc->tokens - 1) * v->sn + desc->d;
        if (bytes_meet(v->data, (size_t)n * es, dw[i], bytes) || bytes_meet(v->data, (size_t)n * es, workspace, workspace_bytes))
          return AA_ERR_ALIAS;
      }
  }
  if (bytes_meet(dw_q, weight_bytes(desc, norm, 0), dw_k, weight_bytes(desc, norm, 1))) return AA_ERR_ALIAS;
  a.weight_heads = norm->per_head != 0, a.eps = norm->eps, a.partial = (float*)workspace;
  return aa::launch_rotary(desc->dtype, a, shape, RotaryMode::kNormBackward, dw_q, dw_k, (hipStream_t)hip_stream) == hipSuccess
             ? AA_OK : AA_ERR_HIP;
}

}  // extern "C"
