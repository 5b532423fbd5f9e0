// C-ABI layer of softmax attention: argument validation and workspace checks.
#include "../../include/agent_attn.h"

#include <math.h>

#include "kernels.h"
#include "token_views.h"

namespace {

using aa::SoftmaxArgs;
using aa::TokenSpan;

constexpr size_t kAlign = 256;

aa_status check_desc(const aa_softmax_attn* d) {
  if (!d) return AA_ERR_NULL;
  if (d->dtype != AA_F32 && d->dtype != AA_F16 && d->dtype != AA_BF16) return AA_ERR_DTYPE;
  if (d->batch <= 0 || d->heads_q <= 0 || d->heads_k <= 0 || d->tokens_q <= 0 || d->tokens_k <= 0 || d->d <= 0) return AA_ERR_SHAPE;
  if (d->heads_q % d->heads_k != 0 || d->sequences < 0) return AA_ERR_SHAPE;
  if (!(d->scale >= 0.0f) || !isfinite(d->scale * 1.4426950408889634f)) return AA_ERR_SHAPE;
  if (d->sequences > 0) {
    if (d->batch != 1 || d->lengths_q || d->lengths_k) return AA_ERR_SHAPE;
    if (!d->starts_q || !d->starts_k) return AA_ERR_NULL;
  } else if (d->starts_q || d->starts_k) {
    return AA_ERR_SHAPE;
  }
  for (const int32_t* p : {d->starts_q, d->starts_k, d->lengths_q, d->lengths_k})
    if ((uintptr_t)p & 3) return AA_ERR_SHAPE;
  if (d->d > aa::kSoftmaxWidth || d->heads_q > 65535 || d->tokens_q > (1 << 30) || d->tokens_k > (1 << 30) || d->sequences > (1 << 28))
    return AA_ERR_UNSUPPORTED;
  const int64_t lim = (int64_t)1 << 40, heads = d->heads_q;
  if ((int64_t)d->batch * d->tokens_q > lim / (heads * d->d) || (int64_t)d->batch * d->tokens_k > lim / (heads * d->d)) return AA_ERR_UNSUPPORTED;
  return AA_OK;
}

SoftmaxArgs args_of(const aa_softmax_attn* d) {
  SoftmaxArgs a{};
  a.batch = d->batch, a.heads_q = d->heads_q, a.heads_k = d->heads_k, a.tokens_q = d->tokens_q, a.tokens_k = d->tokens_k, a.d = d->d;
  a.sequences = d->sequences, a.starts_q = d->starts_q, a.starts_k = d->starts_k, a.lengths_q = d->lengths_q, a.lengths_k = d->lengths_k;
  a.causal = d->causal != 0;
  a.scale = d->scale > 0.0f ? d->scale : 1.0f / sqrtf((float)d->d);
  a.c = a.scale * 1.4426950408889634f;
  return a;
}

aa_status take(const aa_softmax_attn* d, const aa_view* v, bool keys, bool result, TokenSpan* s, aa::TokenView* to) {
  *s = TokenSpan{nullptr, 0, 0, 0, d->batch, keys ? d->heads_k : d->heads_q, keys ? d->tokens_k : d->tokens_q, d->d, d->dtype == AA_F32 ? 4 : 2};
  const aa_status st = aa::check_token_view(v, result, s);
  if (st == AA_OK) *to = aa::TokenView{s->data, s->sb, s->sh, s->sn};
  return st;
}

struct Bytes {
  const void* p;
  size_t n;
};

// whether something that is written meets anything else of the call
template <size_t R, size_t I, size_t W, size_t P>
bool any_meet(const TokenSpan (&results)[R], const TokenSpan (&inputs)[I], const Bytes (&written)[W], const Bytes (&read)[P]) {
  for (size_t i = 0; i < R; ++i) {
    for (size_t j = 0; j < i; ++j)
      if (aa::spans_meet(results[i], results[j])) return true;
    for (const TokenSpan& s : inputs)
      if (aa::spans_meet(results[i], s)) return true;
    for (const Bytes& b : written)
      if (aa::bytes_meet(results[i].data, results[i].bytes(), b.p, b.n)) return true;
    for (const Bytes& b : read)
      if (aa::bytes_meet(results[i].data, results[i].bytes(), b.p, b.n)) return true;
  }
  for (size_t i = 0; i < W; ++i) {
    for (size_t j = 0; j < i; ++j)
      if (aa::bytes_meet(written[i].p, written[i].n, written[j].p, written[j].n)) return true;
    for (const TokenSpan& s : inputs)
      if (aa::bytes_meet(s.data, s.bytes(), written[i].p, written[i].n)) return true;
    for (const Bytes& b : read)
      if (aa::bytes_meet(written[i].p, written[i].n, b.p, b.n)) return true;
  }
  return false;
}

// what the forward pass keeps: its place
void keep(const aa_softmax_attn* d, const void* saved, SoftmaxArgs* a) {
  a->lse = (float*)const_cast<void*>(saved);
  a->low = saved && aa::softmax_keeps_low(d->dtype, *a) ? (char*)const_cast<void*>(saved) + aa::softmax_saved_lse(*a) : nullptr;
}

}  // namespace

extern "C" {

size_t agent_softmax_attn_saved_bytes(const aa_softmax_attn* desc) {
  return check_desc(desc) == AA_OK ? aa::softmax_saved_bytes(desc->dtype, args_of(desc)) : 0;
}

size_t agent_softmax_attn_workspace_bytes(const aa_softmax_attn* desc, const aa_view* q, const aa_view* k, const aa_view* v) {
  if (check_desc(desc) != AA_OK) return 0;
  SoftmaxArgs a = args_of(desc);
  TokenSpan s;
  if (q && take(desc, q, false, false, &s, &a.q) != AA_OK) return 0;
  if (k && take(desc, k, true, false, &s, &a.k) != AA_OK) return 0;
  if (v && take(desc, v, true, false, &s, &a.v) != AA_OK) return 0;
  return aa::softmax_fwd_workspace(desc->dtype, a);
}

size_t agent_softmax_attn_bwd_workspace_bytes(const aa_softmax_attn* desc, const aa_view* q, const aa_view* k, const aa_view* v,
                                              const aa_view* dout) {
  if (check_desc(desc) != AA_OK) return 0;
  SoftmaxArgs a = args_of(desc);
  TokenSpan s;
  if (q && take(desc, q, false, false, &s, &a.q) != AA_OK) return 0;
  if (k && take(desc, k, true, false, &s, &a.k) != AA_OK) return 0;
  if (v && take(desc, v, true, false, &s, &a.v) != AA_OK) return 0;
  if (dout && take(desc, dout, false, false, &s, &a.dout) != AA_OK) return 0;
  return aa::softmax_bwd_workspace(desc->dtype, a);
}

aa_status agent_softmax_attn_fwd(const aa_softmax_attn* desc, const aa_view* q, const aa_view* k, const aa_view* v, void* workspace,
                                 size_t workspace_bytes, const aa_view* out, void* saved, void* hip_stream) {
  aa_status st = check_desc(desc);
  if (st != AA_OK) return st;
  SoftmaxArgs a = args_of(desc);
  TokenSpan in[3], res[1];
  if ((st = take(desc, q, false, false, &in[0], &a.q)) != AA_OK) return st;
  if ((st = take(desc, k, true, false, &in[1], &a.k)) != AA_OK) return st;
  if ((st = take(desc, v, true, false, &in[2], &a.v)) != AA_OK) return st;
  if ((st = take(desc, out, false, true, &res[0], &a.out)) != AA_OK) return st;
  if (!aa::softmax_fits(desc->dtype, a)) return AA_ERR_UNSUPPORTED;
  if ((uintptr_t)saved % kAlign) return AA_ERR_WORKSPACE;
  const size_t need = aa::softmax_fwd_workspace(desc->dtype, a);
  if (need > 0 && (!workspace || ((uintptr_t)workspace % kAlign) != 0 || workspace_bytes < need)) return AA_ERR_WORKSPACE;
  const size_t ns = desc->sequences > 0 ? (size_t)4 * (desc->sequences + 1) : 0, nl = (size_t)4 * desc->batch;
  const Bytes written[] = {{workspace, need}, {saved, aa::softmax_saved_bytes(desc->dtype, a)}};
  const Bytes read[] = {{desc->starts_q, ns}, {desc->starts_k, ns}, {desc->lengths_q, nl}, {desc->lengths_k, nl}};
  if (any_meet(res, in, written, read)) return AA_ERR_ALIAS;
  keep(desc, saved, &a);
  return aa::launch_softmax_fwd(desc->dtype, a, workspace, (hipStream_t)hip_stream) == hipSuccess ? AA_OK : AA_ERR_HIP;
}

aa_status agent_softmax_attn_bwd(const aa_softmax_attn* desc, const aa_view* q, const aa_view* k, const aa_view* v, const aa_view* out,
                                 const void* saved, const aa_view* dout, void* workspace, size_t workspace_bytes, const aa_view* dq,
                                 const aa_view* dk, const aa_view* dv, void* hip_stream) {
  aa_status st = check_desc(desc);
  if (st != AA_OK) return st;
  if (!saved) return AA_ERR_NULL;
  if ((uintptr_t)saved % kAlign) return AA_ERR_WORKSPACE;
  SoftmaxArgs a = args_of(desc);
  TokenSpan in[5], res[3];
  if ((st = take(desc, q, false, false, &in[0], &a.q)) != AA_OK) return st;
  if ((st = take(desc, k, true, false, &in[1], &a.k)) != AA_OK) return st;
  if ((st = take(desc, v, true, false, &in[2], &a.v)) != AA_OK) return st;
  if ((st = take(desc, out, false, false, &in[3], &a.out)) != AA_OK) return st;
  if ((st = take(desc, dout, false, false, &in[4], &a.dout)) != AA_OK) return st;
  if ((st = take(desc, dq, false, true, &res[0], &a.dq)) != AA_OK) return st;
  if ((st = take(desc, dk, true, true, &res[1], &a.dk)) != AA_OK) return st;
  if ((st = take(desc, dv, true, true, &res[2], &a.dv)) != AA_OK) return st;
  if (!aa::softmax_fits(desc->dtype, a)) return AA_ERR_UNSUPPORTED;
  const size_t need = aa::softmax_bwd_workspace(desc->dtype, a);
  if (!workspace || ((uintptr_t)workspace % kAlign) != 0 || workspace_bytes < need) return AA_ERR_WORKSPACE;
  const size_t ns = desc->sequences > 0 ? (size_t)4 * (desc->sequences + 1) : 0, nl = (size_t)4 * desc->batch;
  const Bytes written[] = {{workspace, need}};
  const Bytes read[] = {{saved, aa::softmax_saved_bytes(desc->dtype, a)}, {desc->starts_q, ns}, {desc->starts_k, ns}, {desc->lengths_q, nl}, {desc->lengths_k, nl}};
  if (any_meet(res, in, written, read)) return AA_ERR_ALIAS;
  keep(desc, saved, &a);
  return aa::launch_softmax_bwd(desc->dtype, a, workspace, (hipStream_t)hip_stream) == hipSuccess ? AA_OK : AA_ERR_HIP;
}

}  // extern "C"
