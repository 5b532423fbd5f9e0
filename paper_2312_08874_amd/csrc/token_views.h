// Token tensors [batch][heads][tokens][d] as the C-ABI layer checks them: strides, extents, and whether two of them meet.
#pragma once
#include "../../include/agent_attn.h"

#include <algorithm>
#include <utility>

namespace aa {

struct TokenSpan {      // sizes and strides in elements, es bytes each
  char* data;
  long long sb, sh, sn;
  int batch, heads, tokens, d, es;
  long long extent() const {      // elements from the first to behind the last
    return (batch - 1) * sb + (heads - 1) * sh + (tokens - 1) * sn + d;
  }
  size_t bytes() const { return (size_t)(extent() * es); }
  bool same_place(const TokenSpan& o) const { return data == o.data && sb == o.sb && sh == o.sh && sn == o.sn && heads == o.heads; }
};

// Strides all 0: dense.  result: no element twice.  Sizes are filled in already.
inline aa_status check_token_view(const aa_view* v, bool result, TokenSpan* s) {
  if (!v || !v->data) return AA_ERR_NULL;
  if ((uintptr_t)v->data % s->es) return AA_ERR_SHAPE;
  s->data = (char*)v->data, s->sb = v->stride_b, s->sh = v->stride_h, s->sn = v->stride_n;
  if (s->sb < 0 || s->sh < 0 || s->sn < 0) return AA_ERR_SHAPE;
  if (s->sb == 0 && s->sh == 0 && s->sn == 0) s->sn = s->d, s->sh = (long long)s->tokens * s->d, s->sb = s->sh * s->heads;
  const long long lim = 1ll << 40;
  if (s->sb > lim || s->sh > lim || s->sn > lim) return AA_ERR_UNSUPPORTED;
  std::pair<long long, long long> axis[3] = {{s->sb, s->batch}, {s->sh, s->heads}, {s->sn, s->tokens}};
  std::sort(axis, axis + 3);
  long long extent = s->d;
  for (const auto& a : axis) {
    if (a.second == 1) continue;
    if (result && a.first < extent) return AA_ERR_SHAPE;
    if (a.first > (lim - extent) / a.second) return AA_ERR_UNSUPPORTED;
    extent += a.first * (a.second - 1);
  }
  return AA_OK;
}

inline bool bytes_meet(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b || !na || !nb) return false;
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}

// Elements that a tensor takes of every `period`: those along axes whose strides are whole periods lie at the same place of theirs.
inline long long part_of_period(const TokenSpan& s, long long period) {
  long long extent = s.d;
  const std::pair<long long, long long> axes[3] = {{s.sb, s.batch}, {s.sh, s.heads}, {s.sn, s.tokens}};
  for (const auto& a : axes)
    if (a.first % period != 0) extent += (a.second - 1) * a.first;
  return extent;
}

// Tensors whose extents meet are apart all the same where both repeat with one period (a head's, token's or sequence's stride)
// and take different parts of it, as the slices of a fused projection do.
inline bool spans_meet(const TokenSpan& a, const TokenSpan& b) {
  if (!bytes_meet(a.data, a.bytes(), b.data, b.bytes())) return false;
  const long long es = a.es, diff = (long long)((intptr_t)b.data - (intptr_t)a.data);
  for (const long long period : {a.sh, a.sn, a.sb, b.sh, b.sn, b.sb}) {
    if (period <= 0) continue;
    const long long wa = part_of_period(a, period), wb = part_of_period(b, period), p = period * es, at = (diff % p + p) % p;
    if (wa <= period && at >= wa * es && at + wb * es <= p) return false;
  }
  return true;
}

}  // namespace aa
